// Attention's backward pass for gfx950 (CDNA4): the gradients of attn_fwd_ex.
//
// With S = Q K^T, P = exp(scale S - lse) (recomputed from the forward pass's row
// log-sum-exp) and dO the gradient of the output,
//     dV = P^T dO,   dP = dO V^T,   dS = P o (dP - delta),   delta = rowsum(dO o O) - dlse,
//     dQ = scale dS K,   dK = scale dS^T Q.
//
// Three kernels, and no atomics, so that every call gives the same bits:
//   bwd_rows_kernel   delta and the base-2 log-sum-exp of every row (HBM bound);
//   bwd_dkdv_kernel   a wave keeps 32*KB keys: K and V as operands and dK, dV as
//                     accumulators in registers, and walks the query tiles (of all query
//                     heads of the group): S, dP, dV, dK, four products;
//   bwd_dq_kernel     a wave keeps 32*QB queries: Q, dO and dQ in registers, and walks the
//                     key tiles: S, dP, dQ, three products.
// Seven products instead of the five of the definition: dQ and dK sum over different
// axes, and one kernel for both would have to add one of them up across workgroups,
// either by atomics, whose order changes the result, or through partials of the size of
// (key blocks) x Q in memory.
//
// Orientation.  All products are v_mfma_f32_32x32x16_bf16.  Its accumulator holds column
// l%32 in lane l and rows 8*(r/4) + 4*(l/32) + r%4 in registers r.  The score blocks are
// laid out so that the axis the next product sums over lies in the registers: queries in
// the dK/dV kernel (S = Q K^T, one key per lane), keys in the dQ kernel (S^T = K Q^T, one
// query per lane).  Registers 8s..8s+7, rounded to bf16, are then the operand of that
// product's step s as they stand, with the step's 16 positions in the order
//     16s + 4*(l/32) + i%4 + 8*(i/4),  i = 0..7,
// and the other operand, read transposed from LDS, takes the same order: two
// ds_read_b64_tr_b16 of four rows each.
//
// LDS.  A streamed tile is 32 rows of D values without padding, read both by rows
// (ds_read_b128) and transposed.  Its 16-byte pieces are exchanged within each row so
// that both are free of bank conflicts (64 banks): 16 rows of one column hit 16
// different pieces of the bank line, and so do the four rows x four pieces of a
// transposed read (tile_swizzle).
//
// Roundings: P and dS to bf16, as operands; everything else is fp32 until the result.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fwd_kernel.h"

namespace attn {
namespace {

constexpr int kBwdThreads = 256;
constexpr int kBwdWaves = kBwdThreads / 64;

// Which 16-byte piece of a row holds piece c: c ^ tile_swizzle(row).
template <int D>
__device__ __forceinline__ int tile_swizzle(int row) {
    return D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
}

// One operand tile (32 rows of D) from a head's slab into LDS; the four waves share
// its 1 KiB pieces.  Rows past the slab re-read its last row (finite, and weighted 0).
template <int D>
struct TileLoad {
    static constexpr int PIECES = 32 * D * 2 / 1024;
    static constexpr int NJ = PIECES / kBwdWaves;
    static constexpr int ROWS = 512 / D;  // of one piece
    int off[NJ];  // this lane's source bytes within a tile

    __device__ __forceinline__ void init(int wave, int lane) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int r = (wave + j * kBwdWaves) * ROWS + lane / (D / 8);
            off[j] = r * (D * 2) + ((lane % (D / 8)) ^ tile_swizzle<D>(r)) * 16;
        }
    }
    __device__ __forceinline__ void issue(dma_rsrc_t rsrc, uint32_t lds, int row0, int n_rows,
                                          int wave) const {
        if (row0 + 32 <= n_rows) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                lds_dma16(rsrc, lds + (wave + j * kBwdWaves) * 1024, off[j], row0 * (D * 2));
        } else {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int r = min(row0 + off[j] / (D * 2), n_rows - 1);
                lds_dma16(rsrc, lds + (wave + j * kBwdWaves) * 1024,
                          r * (D * 2) + off[j] % (D * 2), 0);
            }
        }
    }
};

// Operands of one streamed tile at LDS address `tile`.  By rows: lane l holds row l%32,
// values 16*ks + 8*(l/32) ..+7.  Transposed: column 32*cb + l%32, rows of step t in the
// order above.  The exchanged piece of an address is an XOR, so each kind has one
// per-lane base and a compile-time XOR and offset for each operand.
template <int D>
struct TileRead {
    uint32_t row, col;

    __device__ __forceinline__ void init(int lane) {
        const int hh = lane >> 5, i = lane & 15, r = lane & 31;
        row = r * (D * 2) + ((hh ^ tile_swizzle<D>(r)) << 4);
        const int rr = 4 * hh + (i >> 2);
        col = rr * (D * 2) + (((2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) ^ tile_swizzle<D>(rr)) << 4) +
              8 * (i & 1);
    }
    // of a tile whose bases are row + tile and col + tile
    template <int KS>
    static __device__ __forceinline__ bf16x8 by_row(uint32_t base, int offset) {
        return *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)((base ^ (KS << 5)) +
                                                                            offset);
    }
    template <int CB, int T>
    static __device__ __forceinline__ bf16x8 by_col(uint32_t base, int offset) {
        s16x8 x;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t at =
                (base ^ ((4 * CB ^ 2 * j) << 4)) + offset + (16 * T + 8 * j) * (D * 2);
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(uintptr_t)at);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * j + e] = y[e];
        }
        return __builtin_bit_cast(bf16x8, x);
    }
};

__device__ __forceinline__ f32x4 lds_quad(uint32_t at) {
    return *(const __attribute__((address_space(3))) f32x4*)(uintptr_t)at;
}

// Two values rounded to bf16, as one register of an operand.
__device__ __forceinline__ uint32_t round2(float a, float b) {
    bf16x2 y;
    y[0] = (__bf16)a;
    y[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, y);
}

// A value that is formed at this place and not sunk to where it is used, in a later block.
template <typename T>
__device__ __forceinline__ void here(T& x) {
    asm volatile("" : "+v"(x));
}

// The loop bodies are written slot by slot (an operand, its products, a share of the
// other work); nothing moves from one slot to another.
__device__ __forceinline__ void slot_end() { __builtin_amdgcn_sched_barrier(0); }

constexpr int kRing = 4;  // operands in registers: read three slots ahead

// The gradients' accumulators fill the accumulation registers, and the scores must stay
// out of them: the VALU cannot read those, and the compiler, left to itself, puts every
// product's result there and moves accumulators out and back in on every tile (192 moves
// in the dK/dV kernel).  So the scores' products are written out, with plain registers.
// The compiler does not see the waits that they need, which the assembly therefore
// holds itself: two wait states before each (a VALU result read by it), and settle(),
// twenty, between the last product of a block and its first other use.  (A product that
// adds to the one before needs none.)
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void score_first(f32x16& d, bf16x8 a, bf16x8 b) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0"
                 : "=&v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void score_from(f32x16& d, bf16x8 a, bf16x8 b, const f32x16& c) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %3"
                 : "=&v"(d) : "v"(a), "v"(b), "v"(c));
}
__device__ __forceinline__ void score_add(f32x16& d, bf16x8 a, bf16x8 b) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0"
                 : "+v"(d) : "v"(a), "v"(b));
}
template <int N>
__device__ __forceinline__ void settle(f32x16 (&d)[N]) {
    static_assert(N == 1 || N == 2, "");
    if constexpr (N == 2)
        asm volatile("s_nop 15\n\ts_nop 3" : "+v"(d[0]), "+v"(d[1]));
    else
        asm volatile("s_nop 15\n\ts_nop 3" : "+v"(d[0]));
}

// Row of accumulator register r in lane half hh.
__device__ __forceinline__ int acc_row(int r, int hh) { return 8 * (r >> 2) + 4 * hh + (r & 3); }

// Logical workgroup of this one: the hardware deals workgroups round-robin to the XCDs,
// so each XCD gets a contiguous range (of few heads, whose tiles stay in its L2).
__device__ __forceinline__ int logical_wg(int wg, int n_wg, int num_xcds) {
    const int per = n_wg / num_xcds, rem = n_wg % num_xcds;
    const int xcd = wg % num_xcds, slot = wg / num_xcds;
    return (xcd < rem ? xcd * (per + 1) : rem * (per + 1) + (xcd - rem) * per) + slot;
}

// A 32 x 32 block of accumulators (one result row per lane, its columns c0 + acc_row) out.
__device__ __forceinline__ void store_block(const f32x16& x, void* out, long long at, int bf16,
                                            int hh, float factor) {
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
        const long long p = at + 8 * r4 + 4 * hh;
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x[4 * r4 + e] * factor;
        if (bf16) {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            bf16x4 z;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = (__bf16)y[e];
            *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(out) + p) = z;
        } else {
            *reinterpret_cast<f32x4*>(static_cast<float*>(out) + p) = y;
        }
    }
}

// ------------------------------------------------------------- row values --
// For each tile of 32 query rows 64 floats: -lse * log2(e) of its rows, then -delta.
// Rows past Sq get -inf and 0: their weights come out as exactly 0.  D/8 lanes to a row.
template <int D, bool O_BF16>
__global__ __launch_bounds__(256) void bwd_rows_kernel(const BwdArgs a) {
    constexpr int L = D / 8;
    const int n_qt = (a.Sq + 31) / 32;
    const long long slot = ((long long)blockIdx.x * 256 + threadIdx.x) / L;  // row of a tile
    const int lc = threadIdx.x % L;
    const long long tile = slot / 32;
    const long long bh = tile / n_qt;
    if (bh >= a.q_heads) return;  // whole lane groups
    const int i = (int)(slot % 32);
    const int q = (int)(tile - bh * n_qt) * 32 + i;
    const long long row = bh * a.Sq + min(q, a.Sq - 1);
    const u32x4 g = *reinterpret_cast<const u32x4*>(a.d_o + row * D + lc * 8);
    float o[8];
    if constexpr (O_BF16) {
        const u32x4 u =
            *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.o) + row * D + lc * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[2 * e] = __uint_as_float(u[e] << 16);
            o[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
        }
    } else {
        const f32x4* p =
            reinterpret_cast<const f32x4*>(static_cast<const float*>(a.o) + row * D + lc * 8);
        const f32x4 x = p[0], y = p[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[e] = x[e];
            o[4 + e] = y[e];
        }
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        s = fmaf(__uint_as_float(g[e] << 16), o[2 * e], s);
        s = fmaf(__uint_as_float(g[e] & 0xffff0000u), o[2 * e + 1], s);
    }
#pragma unroll
    for (int m = L / 2; m > 0; m /= 2) s += __shfl_xor(s, m, L);
    if (lc == 0) {
        const bool live = q < a.Sq;
        const float l = a.lse[row];
        a.rows[tile * 64 + i] = live ? -l * 1.4426950408889634f : -INFINITY;
        a.rows[tile * 64 + 32 + i] = live ? (a.dlse ? a.dlse[row] - s : -s) : 0.f;
    }
}

// ------------------------------------------------------------------ dK, dV --
template <int D, int KB, bool CAUSAL>
__global__ __launch_bounds__(kBwdThreads, 1) void bwd_dkdv_kernel(const BwdArgs a) {
    constexpr int KD = D / 16, CB = D / 32, TILE = 32 * D;
    constexpr int BK = kBwdWaves * 32 * KB;  // keys of a workgroup
    __shared__ __attribute__((aligned(1024))) uint16_t lds[2 * 2 * TILE];  // [slot][Q, dO]
    __shared__ __attribute__((aligned(16))) float rows[2][64];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    const int logical = logical_wg(blockIdx.x, gridDim.x, a.num_xcds);
    const int per_head = a.blocks * a.splits;
    const int bh = logical / per_head;
    const int split = (logical - bh * per_head) / a.blocks;
    const int k0 = (logical - bh * per_head - split * a.blocks) * BK;  // heavy blocks first
    const int wk0 = k0 + wave * 32 * KB;  // first key of the wave

    bf16x8 kf[KB][KD], vf[KB][KD];  // B operands: lane l holds key l%32
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const long long at =
            ((long long)bh * a.Skv + min(wk0 + kb * 32 + l32, a.Skv - 1)) * D + hh * 8;
#pragma unroll
        for (int ks = 0; ks < KD; ++ks) {
            kf[kb][ks] = *reinterpret_cast<const bf16x8*>(a.k + at + ks * 16);
            vf[kb][ks] = *reinterpret_cast<const bf16x8*>(a.v + at + ks * 16);
        }
    }
    f32x16 dk[KB][CB] = {}, dv[KB][CB] = {};

    // steps of this workgroup: query tiles of every head of the group, from the first
    // that reaches the block's first key
    const int diag = a.Skv - a.Sq;
    const int n_qt = (a.Sq + 31) / 32;
    const int qt0 = CAUSAL ? max(0, k0 - diag) / 32 : 0;
    const int per_q = max(0, n_qt - qt0);
    const long long steps = (long long)per_q * a.group;
    const int begin = (int)(steps * split / a.splits), end = (int)(steps * (split + 1) / a.splits);

    TileLoad<D> load;
    load.init(wave, lane);
    TileRead<D> read;
    read.init(lane);
    const uint32_t lds0 = lds_address(lds), rows0 = lds_address(rows);
    const uint32_t slab = (uint32_t)a.Sq * D * 2;
    auto issue = [&](int step, int slot) __attribute__((always_inline)) {
        const int g = step / per_q, qt = qt0 + step - g * per_q;
        const long long head = (long long)bh * a.group + g;
        const uint32_t dst = lds0 + slot * (2 * TILE * 2);
        load.issue(make_dma_rsrc(a.q + head * a.Sq * D, slab), dst, qt * 32, a.Sq, wave);
        load.issue(make_dma_rsrc(a.d_o + head * a.Sq * D, slab), dst + TILE * 2, qt * 32, a.Sq,
                   wave);
        if (wave == 0)
            lds_dma4(make_dma_rsrc(a.rows + (head * n_qt + qt) * 64, 256), rows0 + slot * 256,
                     lane * 4);
    };

    // Operand i of a tile, in the order of use: Q by rows (S), dO by rows (dP), dO
    // transposed (dV), Q transposed (dK); KD of each.
    constexpr int OPS = 4 * KD;
    bf16x8 ring[kRing];
    uint32_t row_base, col_base, nl_base;  // of the tile that is read
    auto tile_bases = [&](int slot) __attribute__((always_inline)) {
        row_base = read.row + lds0 + slot * (2 * TILE * 2);
        col_base = read.col + lds0 + slot * (2 * TILE * 2);
        nl_base = rows0 + slot * 256 + 16 * hh;
        // opaque, so that the XORed addresses are formed where they are used instead of
        // being kept in registers over the whole loop
        asm volatile("" : "+v"(row_base), "+v"(col_base), "+v"(nl_base));
    };
    auto fetch = [&](auto i_tag) __attribute__((always_inline)) {
        constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
        if constexpr (ph == 0) ring[i % kRing] = TileRead<D>::template by_row<j>(row_base, 0);
        if constexpr (ph == 1)
            ring[i % kRing] = TileRead<D>::template by_row<j>(row_base, TILE * 2);
        if constexpr (ph == 2)
            ring[i % kRing] = TileRead<D>::template by_col<j % CB, j / CB>(col_base, TILE * 2);
        if constexpr (ph == 3)
            ring[i % kRing] = TileRead<D>::template by_col<j % CB, j / CB>(col_base, 0);
    };
    struct Scores {
        f32x16 s[KB], dp[KB];  // S, then P; dP - delta, then dS
        f32x4 nl[2];           // -lse log2 e of eight rows
        uint32_t pk[KB][8];    // P as operand
    };
    uint32_t dsk[KB][8];  // dS as operand
    auto product = [&](auto i_tag, auto kb_tag, Scores& x_) __attribute__((always_inline)) {
        f32x16(&s)[KB] = x_.s;
        f32x16(&dp)[KB] = x_.dp;
        uint32_t(&pk)[KB][8] = x_.pk;
        constexpr int i = decltype(i_tag)::value, kb = decltype(kb_tag)::value;
        constexpr int ph = i / KD, j = i % KD, t = j / CB, cb = j % CB;
        const bf16x8 x = ring[i % kRing];
        if constexpr (ph == 0 && j == 0) score_first(s[kb], x, kf[kb][j]);
        if constexpr (ph == 0 && j > 0) score_add(s[kb], x, kf[kb][j]);
        if constexpr (ph == 1) score_add(dp[kb], x, vf[kb][j]);
        if constexpr (ph >= 2) {
            const uint32_t* o = ph == 2 ? pk[kb] : dsk[kb];
            const u32x4 y = {o[4 * t], o[4 * t + 1], o[4 * t + 2], o[4 * t + 3]};
            f32x16& acc = ph == 2 ? dv[kb][cb] : dk[kb][cb];
            acc = mfma(x, __builtin_bit_cast(bf16x8, y), acc);
        }
    };
    // The weights (two values of each block) follow S during the products of dP and of the
    // first half of dV; dS during those of dV.
    auto weight = [&](auto r_tag, Scores& x_) __attribute__((always_inline)) {
        f32x16(&s)[KB] = x_.s;
        f32x4(&nl)[2] = x_.nl;
        uint32_t(&pk)[KB][8] = x_.pk;
        constexpr int r = decltype(r_tag)::value;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb][r] =
                __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale_log2, nl[(r / 4) % 2][r % 4]));
            if constexpr (r % 2 == 1) pk[kb][r / 2] = round2(s[kb][r - 1], s[kb][r]);
        }
        if constexpr (r % 4 == 3 && r + 5 < 16) nl[(r / 4) % 2] = lds_quad(nl_base + 8 * (r + 5));
    };
    // Scores of hidden pairs: their weights come out as exactly 0.
    auto hide = [&](int q0, Scores& x_) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int lim = wk0 + kb * 32 + l32 - q0 - diag - 4 * hh;
#pragma unroll
            for (int r = 0; r < 16; ++r) x_.s[kb][r] = acc_row(r, 0) >= lim ? x_.s[kb][r] : a.hidden;
        }
    };
    auto grad = [&](auto r_tag, Scores& x_) __attribute__((always_inline)) {
        f32x16(&s)[KB] = x_.s;
        f32x16(&dp)[KB] = x_.dp;
        constexpr int r = decltype(r_tag)::value;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            dp[kb][r] *= s[kb][r];
            if constexpr (r % 2 == 1) dsk[kb][r / 2] = round2(dp[kb][r - 1], dp[kb][r]);
        }
    };
    // -delta, from which the products of dP start
    auto start_dp = [&](auto r4_tag, Scores& x_) __attribute__((always_inline)) {
        f32x16(&dp)[KB] = x_.dp;
        constexpr int r4 = decltype(r4_tag)::value;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const f32x4 x = lds_quad(nl_base + 128 + 32 * r4);
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[kb][4 * r4 + e] = x[e];
        }
    };
    constexpr int TAIL = OPS - (kRing - 1);  // the last slots, behind the barrier
    auto body = [&](int q0) __attribute__((always_inline)) {
        Scores x;
        static_for<0, TAIL>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
            fetch(std::integral_constant<int, i + kRing - 1>{});
            if constexpr (ph == 0 && j >= KD - 4) 
                start_dp(std::integral_constant<int, j - (KD - 4)>{}, x);
            if constexpr (ph == 0 && j == KD - 1) {
                x.nl[0] = lds_quad(nl_base);
                x.nl[1] = lds_quad(nl_base + 32);
            }
            static_for<0, KB>([&](auto kb_tag) __attribute__((always_inline)) {
                product(i_tag, kb_tag, x);
                // 12 of the 16 rows' weights in the gaps of dP (but for the first slot's,
                // when S settles), 4 in the first half of dV's; dS in dV's
                constexpr int n = KB * KD, gap = j * KB + decltype(kb_tag)::value;
                auto w = [&](auto r) __attribute__((always_inline)) {
                    weight(r, x);
                };
                if constexpr (ph == 1 && j > 0)
                    static_for<(gap - KB) * 12 / (n - KB), (gap - KB + 1) * 12 / (n - KB)>(w);
                if constexpr (ph == 2 && gap < n / 2)
                    static_for<12 + gap * 4 / (n / 2), 12 + (gap + 1) * 4 / (n / 2)>(w);
                if constexpr (ph == 2 && j > 0)
                    static_for<(gap - KB) * 16 / (n - KB), (gap - KB + 1) * 16 / (n - KB)>(
                        [&](auto r) __attribute__((always_inline)) { grad(r, x); });
            });
            if constexpr (ph == 1 && j == 0) {
                settle(x.s);
                if (CAUSAL && q0 + diag < wk0 + 32 * KB - 1) hide(q0, x);
            }
            if constexpr (ph == 2 && j == 0) settle(x.dp);
            slot_end();
        });
    };

    if (begin < end) {
        issue(begin, 0);
        if (begin + 1 < end) issue(begin + 1, 1);
        publish_barrier<0>();
        tile_bases(0);
        static_for<0, kRing - 1>(fetch);
    }
    for (int step = begin; step < end; ++step) {
        const int slot = (step - begin) & 1;
        // (a wave whose keys are all hidden computes zeros: it would only wait)
        body(CAUSAL ? (qt0 + step % per_q) * 32 : 0);
        // Every operand of this tile has been read: its slot is free behind the barrier,
        // which also publishes the next tile.
        publish_barrier<0>();
        if (step + 2 < end) issue(step + 2, slot);
        tile_bases(slot ^ 1);
        Scores none;  // (dK's products read dsk alone)
        static_for<TAIL, OPS>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value;
            static_for<0, KB>(
                [&](auto kb_tag) __attribute__((always_inline)) { product(i_tag, kb_tag, none); });
            fetch(std::integral_constant<int, i + kRing - 1 - OPS>{});
            slot_end();
        });
    }

#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const int key = wk0 + kb * 32 + l32;
        if (key >= a.Skv) continue;
        long long at = ((long long)bh * a.Skv + key) * D;
        if (a.splits > 1) at += (long long)split * a.part_stride;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            store_block(dk[kb][cb], a.out0, at + cb * 32, a.out_bf16, hh, a.scale);
            store_block(dv[kb][cb], a.out1, at + cb * 32, a.out_bf16, hh, 1.f);
        }
    }
}

// ---------------------------------------------------------------------- dQ --
template <int D, int QB, bool CAUSAL>
__global__ __launch_bounds__(kBwdThreads, 1) void bwd_dq_kernel(const BwdArgs a) {
    constexpr int KD = D / 16, CB = D / 32, TILE = 32 * D;
    constexpr int BQ = kBwdWaves * 32 * QB;  // queries of a workgroup
    constexpr int SLOT = 2 * TILE * 2;  // bytes of a tile of K and one of V
    __shared__ __attribute__((aligned(1024))) uint16_t lds[3 * 2 * TILE];  // [slot][K, V]
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    const int logical = logical_wg(blockIdx.x, gridDim.x, a.num_xcds);
    const int per_head = a.blocks * a.splits;
    const int bh = logical / per_head;
    const int split = (logical - bh * per_head) / a.blocks;
    // heavy blocks first
    const int q0 = (a.blocks - 1 - (logical - bh * per_head - split * a.blocks)) * BQ;
    const int wq0 = q0 + wave * 32 * QB;

    const int n_qt = (a.Sq + 31) / 32;
    bf16x8 qf[QB][KD], gf[QB][KD];  // B operands: lane l holds query l%32
    float nl[QB];
    f32x16 nd[QB];  // -delta, from which the products of dP start
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int q = wq0 + qb * 32 + l32;
        const long long at = ((long long)bh * a.Sq + min(q, a.Sq - 1)) * D + hh * 8;
#pragma unroll
        for (int ks = 0; ks < KD; ++ks) {
            qf[qb][ks] = *reinterpret_cast<const bf16x8*>(a.q + at + ks * 16);
            gf[qb][ks] = *reinterpret_cast<const bf16x8*>(a.d_o + at + ks * 16);
        }
        // (queries past Sq: the last tile's padding, or the last row of all)
        const long long tile = (long long)bh * n_qt + min(q, n_qt * 32 - 1) / 32;
        nl[qb] = a.rows[tile * 64 + l32];
        const float x = a.rows[tile * 64 + 32 + l32];
#pragma unroll
        for (int r = 0; r < 16; ++r) nd[qb][r] = x;
    }
    f32x16 dq[QB][CB] = {};

    const int diag = a.Skv - a.Sq;
    const int last_q = min(q0 + BQ, a.Sq) - 1;
    const int n_keys = CAUSAL ? min(a.Skv, last_q + diag + 1) : a.Skv;
    const long long steps = (n_keys + 31) / 32;
    const int begin = (int)(steps * split / a.splits), end = (int)(steps * (split + 1) / a.splits);

    TileLoad<D> load;
    load.init(wave, lane);
    TileRead<D> read;
    read.init(lane);
    const uint32_t lds0 = lds_address(lds);
    const uint32_t slab = (uint32_t)a.Skv * D * 2;
    const long long head = bh / a.group;
    const dma_rsrc_t k_rsrc = make_dma_rsrc(a.k + head * a.Skv * D, slab);
    const dma_rsrc_t v_rsrc = make_dma_rsrc(a.v + head * a.Skv * D, slab);
    auto issue = [&](int step, int slot) __attribute__((always_inline)) {
        const uint32_t dst = lds0 + slot * SLOT;
        load.issue(k_rsrc, dst, step * 32, a.Skv, wave);
        load.issue(v_rsrc, dst + TILE * 2, step * 32, a.Skv, wave);
    };

    // Operand i of a step: K by rows (S of this tile), K transposed (dQ of the tile before:
    // its dS is formed during the products of S), V by rows (dP of this tile); KD of each.
    constexpr int OPS = 3 * KD;
    bf16x8 ring[kRing];
    uint32_t row_base, col_base;
    auto fetch = [&](auto i_tag) __attribute__((always_inline)) {
        constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
        if constexpr (ph == 0) ring[i % kRing] = TileRead<D>::template by_row<j>(row_base, 0);
        if constexpr (ph == 1)
            ring[i % kRing] = TileRead<D>::template by_col<j % CB, j / CB>(col_base, 0);
        if constexpr (ph == 2)
            ring[i % kRing] = TileRead<D>::template by_row<j>(row_base, TILE * 2);
    };
    f32x16 s[QB], p[QB] = {}, dp[QB] = {};  // (no tile before the first: its dS is 0)
    uint32_t dsk[QB][8];  // dS as operands
    auto product = [&](auto i_tag, auto qb_tag) __attribute__((always_inline)) {
        constexpr int i = decltype(i_tag)::value, qb = decltype(qb_tag)::value;
        constexpr int ph = i / KD, j = i % KD, t = j / CB, cb = j % CB;
        const bf16x8 x = ring[i % kRing];
        if constexpr (ph == 0 && j == 0) score_first(s[qb], x, qf[qb][j]);
        if constexpr (ph == 0 && j > 0) score_add(s[qb], x, qf[qb][j]);
        if constexpr (ph == 1) {
            const u32x4 y = {dsk[qb][4 * t], dsk[qb][4 * t + 1], dsk[qb][4 * t + 2],
                             dsk[qb][4 * t + 3]};
            dq[qb][cb] = mfma(x, __builtin_bit_cast(bf16x8, y), dq[qb][cb]);
        }
        if constexpr (ph == 2 && j == 0) score_from(dp[qb], x, gf[qb][j], nd[qb]);
        if constexpr (ph == 2 && j > 0) score_add(dp[qb], x, gf[qb][j]);
    };
    auto weight = [&](auto r_tag) __attribute__((always_inline)) {
        constexpr int r = decltype(r_tag)::value;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float x = __builtin_amdgcn_exp2f(fmaf(s[qb][r], a.scale_log2, nl[qb]));
            here(x);
            p[qb][r] = x;
        }
    };
    // Scores of hidden pairs and of keys past Skv: their weights come out as exactly 0.
    auto hide = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int last =
                CAUSAL ? min(a.Skv - 1, wq0 + qb * 32 + l32 + diag) : a.Skv - 1;
            const int lim = last - k0 - 4 * hh;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[qb][r] = acc_row(r, 0) <= lim ? s[qb][r] : a.hidden;
        }
    };
    auto grad = [&](auto r_tag) __attribute__((always_inline)) {
        constexpr int r = decltype(r_tag)::value;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            dp[qb][r] *= p[qb][r];
            if constexpr (r % 2 == 1) {
                dsk[qb][r / 2] = round2(dp[qb][r - 1], dp[qb][r]);
                here(dsk[qb][r / 2]);
            }
        }
    };
    constexpr int N = QB * KD;  // products, and the gaps behind them, of one kind
    constexpr int TAIL = OPS - (kRing - 1);  // the last slots, behind the barrier
    auto body = [&](int k0) __attribute__((always_inline)) {
        static_for<0, TAIL>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
            fetch(std::integral_constant<int, i + kRing - 1>{});
            static_for<0, QB>([&](auto qb_tag) __attribute__((always_inline)) {
                product(i_tag, qb_tag);
                // dS of the tile before in the gaps of S; 12 of the 16 rows' weights in those
                // of dQ, 4 in those of dP; the first slots are left to settle
                constexpr int gap = j * QB + decltype(qb_tag)::value;
                constexpr int M = N - QB, B = N - QB * (kRing - 1);
                if constexpr (ph == 0 && j > 0)
                    static_for<(gap - QB) * 16 / M, (gap - QB + 1) * 16 / M>(grad);
                if constexpr (ph == 1 && j > 0)
                    static_for<(gap - QB) * 12 / M, (gap - QB + 1) * 12 / M>(weight);
                if constexpr (ph == 2) static_for<12 + gap * 4 / B, 12 + (gap + 1) * 4 / B>(weight);
            });
            if constexpr (ph == 0 && j == 0) settle(dp);
            if constexpr (ph == 1 && j == 0) {
                settle(s);
                if (k0 + 32 > a.Skv || (CAUSAL && k0 + 31 > wq0 + diag)) hide(k0);
            }
            slot_end();
        });
    };
    // dQ of the wave's last tile.
    auto drain = [&]() __attribute__((always_inline)) {
        settle(dp);
        static_for<0, 16>(grad);
        static_for<KD, KD + kRing - 1>(fetch);
        static_for<KD, 2 * KD>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value;
            if constexpr (i + kRing - 1 < 2 * KD)
                fetch(std::integral_constant<int, i + kRing - 1>{});
            static_for<0, QB>(
                [&](auto qb_tag) __attribute__((always_inline)) { product(i_tag, qb_tag); });
            slot_end();
        });
    };

    int slot = 0;
    if (begin < end) {
        issue(begin, 0);
        if (begin + 1 < end) issue(begin + 1, 1);
        publish_barrier<0>();
        row_base = read.row + lds0;
        static_for<0, kRing - 1>(fetch);
    }
    for (int step = begin; step < end; ++step) {
        // (before the first tile: itself, with a dS of 0)
        const int prev = slot == 0 ? 2 : slot - 1, next = slot == 2 ? 0 : slot + 1;
        // opaque, so that the XORed addresses are formed where they are used instead of
        // being kept in registers over the whole loop
        row_base = read.row + lds0 + slot * SLOT;
        col_base = read.col + lds0 + (step == begin ? slot : prev) * SLOT;
        asm volatile("" : "+v"(row_base), "+v"(col_base));
        // (a wave whose pairs are all hidden computes zeros: it would only wait)
        body(step * 32);
        // The tile before has been read for good: its slot is free behind the barrier,
        // which also publishes the next tile.
        publish_barrier<0>();
        if (step + 2 < end) issue(step + 2, prev);
        row_base = read.row + lds0 + next * SLOT;
        asm volatile("" : "+v"(row_base));
        static_for<TAIL, OPS>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value;
            static_for<0, QB>(
                [&](auto qb_tag) __attribute__((always_inline)) { product(i_tag, qb_tag); });
            fetch(std::integral_constant<int, i + kRing - 1 - OPS>{});
            slot_end();
        });
        slot = next;
    }
    if (begin < end) {
        col_base = read.col + lds0 + (slot == 0 ? 2 : slot - 1) * SLOT;
        drain();
    }

#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int q = wq0 + qb * 32 + l32;
        if (q >= a.Sq) continue;
        long long at = ((long long)bh * a.Sq + q) * D;
        if (a.splits > 1) at += (long long)split * a.part_stride;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
            store_block(dq[qb][cb], a.out0, at + cb * 32, a.out_bf16, hh, a.scale);
    }
}

// out[i] = sum of n partials at i, i + stride, ..., in their order; four values to a
// thread.  HBM bound.
__global__ __launch_bounds__(256) void bwd_sum_kernel(const float* part, long long stride, int n,
                                                      void* out, int out_bf16, long long quads) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= quads) return;
    f32x4 s = {};
    for (int j = 0; j < n; ++j) s += *reinterpret_cast<const f32x4*>(part + j * stride + i * 4);
    if (out_bf16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (__bf16)s[e];
        *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(out) + i * 4) = z;
    } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(out) + i * 4) = s;
    }
}

template <int D>
hipError_t launch_d(const BwdPlan& p, BwdArgs a, int causal, int o_bf16, int out_bf16, void* dq,
                    void* dk, void* dv, float* part, hipStream_t stream) {
    const long long slots = a.q_heads * ((a.Sq + 31) / 32) * 32 * (D / 8);
    const dim3 row_grid((unsigned)((slots + 255) / 256));
    if (o_bf16)
        bwd_rows_kernel<D, true><<<row_grid, 256, 0, stream>>>(a);
    else
        bwd_rows_kernel<D, false><<<row_grid, 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long long kv_values = a.kv_heads * a.Skv * D, q_values = a.q_heads * a.Sq * D;
    auto sum = [&](const float* from, void* to, int n, long long values) {
        bwd_sum_kernel<<<(unsigned)((values / 4 + 255) / 256), 256, 0, stream>>>(
            from, values, n, to, out_bf16, values / 4);
        return hipGetLastError();
    };

    a.blocks = p.kv_blocks;
    a.splits = p.kv_splits;
    a.part_stride = kv_values;
    a.out_bf16 = p.kv_splits > 1 ? 0 : out_bf16;
    a.out0 = p.kv_splits > 1 ? part : dk;
    a.out1 = p.kv_splits > 1 ? part + p.kv_splits * kv_values : dv;
    const dim3 kv_grid((unsigned)(a.kv_heads * a.blocks * a.splits));
    if (causal)
        bwd_dkdv_kernel<D, 2, true><<<kv_grid, kBwdThreads, 0, stream>>>(a);
    else
        bwd_dkdv_kernel<D, 2, false><<<kv_grid, kBwdThreads, 0, stream>>>(a);
    e = hipGetLastError();
    if (e == hipSuccess && p.kv_splits > 1) e = sum(part, dk, p.kv_splits, kv_values);
    if (e == hipSuccess && p.kv_splits > 1)
        e = sum(part + p.kv_splits * kv_values, dv, p.kv_splits, kv_values);
    if (e != hipSuccess) return e;

    a.blocks = p.q_blocks;
    a.splits = p.q_splits;
    a.part_stride = q_values;
    a.out_bf16 = p.q_splits > 1 ? 0 : out_bf16;
    a.out0 = p.q_splits > 1 ? part : dq;
    const dim3 q_grid((unsigned)(a.q_heads * a.blocks * a.splits));
    if (causal)
        bwd_dq_kernel<D, 2, true><<<q_grid, kBwdThreads, 0, stream>>>(a);
    else
        bwd_dq_kernel<D, 2, false><<<q_grid, kBwdThreads, 0, stream>>>(a);
    e = hipGetLastError();
    if (e == hipSuccess && p.q_splits > 1) e = sum(part, dq, p.q_splits, q_values);
    return e;
}

}  // namespace

hipError_t launch_bwd(const BwdPlan& p, const BwdArgs& a, int d, int causal, int o_bf16,
                      int out_bf16, void* dq, void* dk, void* dv, float* part,
                      hipStream_t stream) {
    return d == 64 ? launch_d<64>(p, a, causal, o_bf16, out_bf16, dq, dk, dv, part, stream)
                   : launch_d<128>(p, a, causal, o_bf16, out_bf16, dq, dk, dv, part, stream);
}

}  // namespace attn
