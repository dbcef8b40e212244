// Attention's backward pass for gfx950 (CDNA4): the gradients of attn_fwd_ex.
//
// With S = Q K^T, P = exp(scale S - lse) (recomputed from the forward pass's row
// log-sum-exp) and dO the gradient of the output,
//     dV = P^T dO,   dP = dO V^T,   dS = P o (dP - delta),   delta = rowsum(dO o O) - dlse,
//     dQ = scale dS K,   dK = scale dS^T Q.
//
// No atomics, so that every call gives the same bits.  bwd_rows_kernel computes delta and
// the base-2 log-sum-exp of every row (HBM bound); bwd_kernel holds two kinds of
// workgroups:
//   dkdv_block        a wave keeps 32*KB keys: K and V as operands and dK, dV as
//                     accumulators in registers, and walks the query tiles (of all query
//                     heads of the group): S, dP, dV, dK, four products;
//   dq_block          a wave keeps 32*QB queries: Q, dO and dQ in registers, and walks the
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
// Roundings: P and dS to bf16, since the matrix instruction takes no more (as P in the forward
// pass); everything else is fp32 until the result.  In norm the gradients are 0.0024 off the
// exact ones with both, 0.0017 from the rounding of bf16 results alone.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <type_traits>

#include "fwd_kernel.h"

namespace attn {
namespace {

// Waves of a workgroup, and 32-row blocks that each keeps.  With D = 128 one wave to a SIMD
// and two blocks to a wave: every operand read from LDS serves two products (with one, LDS
// would be as busy as the matrix cores).  With D = 64 the weights, as many for half the
// products, take as long as those do, and two waves to a SIMD overlap the two kinds of
// work better than one does (B4 H16 S2048 4% faster, side by side); in two workgroups of 128
// rows, they leave out more of a causal diagonal (causal 4% again).
template <int D>
struct BwdShape {
    static constexpr int ROWS = bwd_block_rows(D), BLOCKS = D == 64 ? 1 : 2;
    static constexpr int WAVES = ROWS / (32 * BLOCKS), THREADS = 64 * WAVES;
    static constexpr int WAVES_PER_SIMD = WAVES * bwd_wgs_per_cu(D) / 4;
};

// Which 16-byte piece of a row holds piece c: c ^ tile_swizzle(row).
template <int D>
__device__ __forceinline__ int tile_swizzle(int row) {
    return D == 128 ? (row & 3) << 2 | ((row >> 2) & 3) : ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
}

// A pair of tiles (32 rows of D each), the same rows of two slabs, into LDS one behind the
// other; the waves share their 1 KiB pieces.  Rows past the slabs re-read the last row
// (finite, and weighted 0).
template <int D>
struct TileLoad {
    static constexpr int W = BwdShape<D>::WAVES, PIECES = 32 * D * 2 / 1024;
    static constexpr int NJ = 2 * PIECES / W, NO = PIECES / W;
    static_assert(PIECES % W == 0, "a wave's pieces of each tile");
    static constexpr int ROWS = 512 / D;  // of one piece
    int off[NO];  // this lane's source bytes within a tile

    __device__ __forceinline__ void init(int wave, int lane) {
#pragma unroll
        for (int j = 0; j < NO; ++j) {
            // (a wave's number is less than PIECES: it is written so because without the
            // remainder the folded d = 128 kernel spills five registers, with it one)
            const int r = (wave % PIECES + j * W) * ROWS + lane / (D / 8);
            off[j] = r * (D * 2) + ((lane % (D / 8)) ^ tile_swizzle<D>(r)) * 16;
        }
    }
    __device__ __forceinline__ void issue(dma_rsrc_t slab0, dma_rsrc_t slab1, uint32_t lds,
                                          int row0, int n_rows, int wave) const {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int piece = wave + j * W;
            const dma_rsrc_t slab = j < NJ / 2 ? slab0 : slab1;
            if (row0 + 32 <= n_rows) {
                lds_dma16(slab, lds + piece * 1024, off[j % NO], row0 * (D * 2));
            } else {
                const int r = min(row0 + off[j % NO] / (D * 2), n_rows - 1);
                lds_dma16(slab, lds + piece * 1024, r * (D * 2) + off[j % NO] % (D * 2), 0);
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

// Operands are read into a ring of registers, some slots ahead.  ahead: operands that
// have been asked for by the end of the reads of slot i.
template <int D>
struct KvRing {
    static constexpr int SIZE = D == 64 ? 8 : 4, OPS = D / 4;
    static constexpr int ahead(int i) { return i + (D == 64 ? 5 : 4); }
    static_assert(OPS - ahead(0) + 1 >= 3 * D / 16, "dS is done before the last slots");
};
template <int D>
struct QRing {
    static constexpr int SIZE = D == 64 ? 4 : 8, OPS = 3 * D / 16;
    static constexpr int ahead(int i) { return i + (D == 64 ? 4 : 7); }
    static_assert(OPS - ahead(0) + 1 > 2 * D / 16, "and the weights");
};

// The gradients' accumulators fill the accumulation registers, and the scores must stay
// out of them: the VALU cannot read those, and the compiler, left to itself, puts every
// product's result there and moves accumulators out and back in on every tile (192 moves
// a tile for dK, dV).  So the scores' products are written out, with plain registers.
// The compiler does not see the wait states that these need.  Between the last product of
// a block and its first other use (12) settle() holds them; between a VALU result and the
// product that reads it (2) none are held, because no operand of these products is one:
// they come from LDS, from registers that the loop does not write, or from the product
// before.  tests/test_bwd_hazards.py checks both in the generated code.
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// ACC: b lies in accumulation registers, where the kernel has some to spare.
#define ATTN_SCORE_MFMA(C) "v_mfma_f32_32x32x16_bf16 %0, %1, %2, " C
template <bool ACC>
__device__ __forceinline__ void score_first(f32x16& d, bf16x8 a, bf16x8 b) {
    if constexpr (ACC)
        asm volatile(ATTN_SCORE_MFMA("0") : "=&v"(d) : "v"(a), "a"(b));
    else
        asm volatile(ATTN_SCORE_MFMA("0") : "=&v"(d) : "v"(a), "v"(b));
}
template <bool ACC>
__device__ __forceinline__ void score_from(f32x16& d, bf16x8 a, bf16x8 b, const f32x16& c) {
    if constexpr (ACC)
        asm volatile(ATTN_SCORE_MFMA("%3") : "=&v"(d) : "v"(a), "a"(b), "v"(c));
    else
        asm volatile(ATTN_SCORE_MFMA("%3") : "=&v"(d) : "v"(a), "v"(b), "v"(c));
}
template <bool ACC>
__device__ __forceinline__ void score_add(f32x16& d, bf16x8 a, bf16x8 b) {
    if constexpr (ACC)
        asm volatile(ATTN_SCORE_MFMA("%0") : "+v"(d) : "v"(a), "a"(b));
    else
        asm volatile(ATTN_SCORE_MFMA("%0") : "+v"(d) : "v"(a), "v"(b));
}
#undef ATTN_SCORE_MFMA
template <int FROM, int TO, int N>
__device__ __forceinline__ void settle(f32x16 (&d)[N]) {
    static_assert(TO <= N && TO - FROM <= 2 && TO > FROM, "");
    if constexpr (TO - FROM == 2)
        asm volatile("s_nop 11" : "+v"(d[FROM]), "+v"(d[FROM + 1]));
    else
        asm volatile("s_nop 11" : "+v"(d[FROM]));
}

// Masks: none, causal, and causal with the heads of a group in one.  (Apart: at d = 128 the
// causal kernel has no register to spare for finding each row's position, it would spill 27;
// the folded one spills one, outside of the loops.)
constexpr int kNoMask = 0, kCausalMask = 1, kFoldedMask = 2;

// Position of a row of a folded problem.  (Exact: rows are fewer than 2^32 / period.)
__device__ __forceinline__ int position(const BwdArgs& a, int row) {
    return row - a.period * (int)__umulhi((uint32_t)row, a.period_inverse);
}

// Row of accumulator register r in lane half hh.
__device__ __forceinline__ int acc_row(int r, int hh) { return 8 * (r >> 2) + 4 * hh + (r & 3); }

// 32 result rows of a wave (row l%32 in lane l, columns 32*cb + acc_row) to out, rows from
// row0 up to n_rows.  Through LDS: stored from the registers, an instruction would write
// 8 or 16 bytes to each of 32 rows; staged, it writes whole lines (a workgroup's results
// in 4 us instead of 13, with all workgroups storing at once).  The stage, the wave's
// own, is 32 rows of half the fp32 values, or of all bf16 ones, padded by 16 bytes.
template <int D>
constexpr int stage_bytes() { return 32 * (D * 2 + 16); }

template <int D>
__device__ __forceinline__ void store_rows(const f32x16 (&x)[D / 32], char* stage, void* out,
                                           long long row0, long long n_rows, int bf16,
                                           float factor) {
    constexpr int STRIDE = D * 2 + 16, L = D * 2 / 16, RPI = 64 / L;  // lanes to a row, rows at once
    // (counted anew: taken from the thread's number it would be kept over the loops)
    const int lane = __lane_id(), l32 = lane & 31, hh = lane >> 5;
    auto flush = [&](char* base, long long row_bytes) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 32 / RPI; ++i) {
            const int r = i * RPI + lane / L;
            const u32x4 y = *reinterpret_cast<const u32x4*>(stage + r * STRIDE + (lane % L) * 16);
            if (row0 + r < n_rows)
                *reinterpret_cast<u32x4*>(base + (row0 + r) * row_bytes + (lane % L) * 16) = y;
        }
    };
    if (bf16) {
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                uint32_t y[2];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    y[e] = round2(x[cb][4 * r4 + 2 * e] * factor, x[cb][4 * r4 + 2 * e + 1] * factor);
                *reinterpret_cast<uint64_t*>(stage + l32 * STRIDE +
                                             (32 * cb + 8 * r4 + 4 * hh) * 2) =
                    (uint64_t)y[1] << 32 | y[0];
            }
        flush(static_cast<char*>(out), D * 2);
        return;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = x[half * (D / 64) + c][4 * r4 + e] * factor;
                *reinterpret_cast<f32x4*>(stage + l32 * STRIDE + (32 * c + 8 * r4 + 4 * hh) * 4) = y;
            }
        flush(static_cast<char*>(out) + half * D * 2, D * 4);
    }
}

// LDS of a workgroup, in bytes: row values, then slots of a pair of tiles each (Q and dO:
// 2, K and V: 3).  At the start the waves' own rows of both their operands come through
// the place from the second slot on; at the end the results through the stages.
template <int D>
struct BwdLds {
    static constexpr int TILE = 32 * D * 2, SLOT = 2 * TILE;
    static constexpr int SLOTS = 1024, OWN = SLOTS + SLOT;
    static constexpr int OWN_WAVE = 2 * BwdShape<D>::BLOCKS * TILE;
    static constexpr int STAGES = BwdShape<D>::WAVES * stage_bytes<D>();
    static constexpr int BYTES = OWN + BwdShape<D>::WAVES * OWN_WAVE;
    static_assert(BYTES >= SLOTS + 3 * SLOT && BYTES >= STAGES, "");
};

// A wave's own rows of a head's slab as operand registers: op[b][ks] holds row l%32 of
// the wave's b-th block, values 16*ks + 8*(l/32) ..+7.  Loaded straight into registers, an
// instruction touches 32 rows, 32 bytes each, and the operands of a workgroup took 5.8 us;
// through LDS in whole rows they take 3.  own_load issues the loads of a block, own_read
// reads the blocks that have landed.
template <int D>
__device__ __forceinline__ void own_load(dma_rsrc_t rsrc, uint32_t lds, int row0, int n_rows,
                                         int lane) {
    constexpr int ROWS = 512 / D;
#pragma unroll
    for (int p = 0; p < 32 / ROWS; ++p) {
        const int r = p * ROWS + lane / (D / 8);
        const int c = (lane % (D / 8)) ^ tile_swizzle<D>(r);
        lds_dma16(rsrc, lds + p * 1024, min(row0 + r, n_rows - 1) * (D * 2) + c * 16, 0);
    }
}
template <int D>
__device__ __forceinline__ void own_read(bf16x8 (&op)[BwdShape<D>::BLOCKS][D / 16],
                                         const TileRead<D>& read, uint32_t lds) {
    static_for<0, BwdShape<D>::BLOCKS>([&](auto b) __attribute__((always_inline)) {
        static_for<0, D / 16>([&](auto ks) __attribute__((always_inline)) {
            op[b][ks] = TileRead<D>::template by_row<decltype(ks)::value>(
                read.row + lds, decltype(b)::value * BwdLds<D>::TILE);
        });
    });
}

// ------------------------------------------------------------- row values --
// For each tile of 32 query rows 64 floats: -lse * log2(e) of its rows, then -delta.
// Rows past Sq get -inf and 0: their weights come out as exactly 0.  D/8 lanes to a row.
// HBM bound, one read of O and dO: B4 H16 S2048 d128, 102 MB, 19 us (5.4 TB/s).
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
// One block of keys (kv head bh, over the batch), part `split` of `splits` of its sum.
template <int D, int MASK>
__device__ __forceinline__ void dkdv_block(const BwdArgs& a, char* lds, int bh, int block,
                                           int split, int splits) {
    constexpr bool CAUSAL = MASK != kNoMask, FOLDED = MASK == kFoldedMask;
    constexpr int KB = BwdShape<D>::BLOCKS, KD = D / 16, CB = D / 32;
    typedef BwdLds<D> L;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int k0 = block * BwdShape<D>::ROWS;
    // the wave's blocks of 32 keys are KSTEP apart, so that near a causal diagonal all
    // waves have their second block hidden at the same time
    constexpr int KSTEP = 32 * BwdShape<D>::WAVES;
    const int wk0 = k0 + wave * 32;  // first key of the wave's first block

    bf16x8 kf[KB][KD], vf[KB][KD];  // B operands: lane l holds key l%32
    f32x16 dk[KB][CB] = {}, dv[KB][CB] = {};

    // steps: query tiles of every head of the group, from the first that reaches the
    // block's first key
    const int diag = a.diag;
    const int n_qt = (a.Sq + 31) / 32;
    const int qt0 = CAUSAL ? max(0, k0 - diag) / 32 : 0;
    const int per_q = n_qt - qt0;
    const int steps = a.units.size.kv_steps(block);
    const int begin = (int)((long long)steps * split / splits);
    const int end = (int)((long long)steps * (split + 1) / splits);

    TileLoad<D> load;
    load.init(wave, lane);
    TileRead<D> read;
    read.init(lane);
    const uint32_t rows0 = lds_address(lds), lds0 = rows0 + L::SLOTS;
    const uint32_t slab = (uint32_t)a.Sq * D * 2;
    // of the next load: its head's slabs, its tile
    int load_g = begin / per_q, load_qt = qt0 + begin % per_q;
    dma_rsrc_t q_rsrc, g_rsrc, row_rsrc;
    auto load_head = [&]() __attribute__((always_inline)) {
        const long long head = (long long)bh * a.group + load_g;
        q_rsrc = make_dma_rsrc(a.q + head * a.Sq * D, slab);
        g_rsrc = make_dma_rsrc(a.d_o + head * a.Sq * D, slab);
        row_rsrc = make_dma_rsrc(a.rows + head * n_qt * 64, n_qt * 256);
    };
    load_head();
    auto issue = [&](int slot) __attribute__((always_inline)) {
        const uint32_t dst = lds0 + slot * L::SLOT;
        load.issue(q_rsrc, g_rsrc, dst, load_qt * 32, a.Sq, wave);
        if (wave == 0) lds_dma4(row_rsrc, rows0 + slot * 256, __lane_id() * 4, load_qt * 256);
        if (++load_qt == n_qt) {
            load_qt = qt0;
            ++load_g;
            if (load_g < a.group) load_head();
        }
    };

    // Operand i of a tile, in the order of use: Q by rows (S), dO by rows (dP), dO
    // transposed (dV), Q transposed (dK); KD of each.
    typedef KvRing<D> Ring;
    constexpr int OPS = Ring::OPS, RING = Ring::SIZE;
    static_assert(OPS == 4 * KD && OPS % RING == 0, "");
    bf16x8 ring[RING];
    uint32_t row_base, col_base, nl_base;  // of the tile that is read
    auto tile_bases = [&](int slot) __attribute__((always_inline)) {
        row_base = read.row + lds0 + slot * L::SLOT;
        col_base = read.col + lds0 + slot * L::SLOT;
        nl_base = rows0 + slot * 256 + 16 * hh;
        // opaque, so that the XORed addresses are formed where they are used instead of
        // being kept in registers over the whole loop
        asm volatile("" : "+v"(row_base), "+v"(col_base), "+v"(nl_base));
    };
    auto fetch = [&](auto i_tag) __attribute__((always_inline)) {
        constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
        if constexpr (ph == 0) ring[i % RING] = TileRead<D>::template by_row<j>(row_base, 0);
        if constexpr (ph == 1)
            ring[i % RING] = TileRead<D>::template by_row<j>(row_base, L::TILE);
        if constexpr (ph == 2)
            ring[i % RING] = TileRead<D>::template by_col<j % CB, j / CB>(col_base, L::TILE);
        if constexpr (ph == 3)
            ring[i % RING] = TileRead<D>::template by_col<j % CB, j / CB>(col_base, 0);
    };
    struct Scores {
        f32x16 s[KB], dp[KB];  // S, then P; dP - delta, then dS
        f32x16 nd;             // -delta, from which the products of dP start
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
        const bf16x8 x = ring[i % RING];
        if constexpr (ph == 0 && j == 0) score_first<D == 64>(s[kb], x, kf[kb][j]);
        if constexpr (ph == 0 && j > 0) score_add<D == 64>(s[kb], x, kf[kb][j]);
        if constexpr (ph == 1 && j == 0) score_from<D == 64>(dp[kb], x, vf[kb][j], x_.nd);
        if constexpr (ph == 1 && j > 0) score_add<D == 64>(dp[kb], x, vf[kb][j]);
        if constexpr (ph >= 2) {
            const uint32_t* o = ph == 2 ? pk[kb] : dsk[kb];
            const u32x4 y = {o[4 * t], o[4 * t + 1], o[4 * t + 2], o[4 * t + 3]};
            f32x16& acc = ph == 2 ? dv[kb][cb] : dk[kb][cb];
            acc = mfma(x, __builtin_bit_cast(bf16x8, y), acc);
        }
    };
    // The weights (two values of each block) follow S during the products of dP and of the
    // first half of dV; dS during those of dV.
    // (NA: the blocks at work, the first ones)
    auto weight = [&](auto r_tag, auto na, Scores& x_) __attribute__((always_inline)) {
        constexpr int NA = decltype(na)::value;
        f32x16(&s)[KB] = x_.s;
        f32x4(&nl)[2] = x_.nl;
        uint32_t(&pk)[KB][8] = x_.pk;
        constexpr int r = decltype(r_tag)::value;
#pragma unroll
        for (int kb = 0; kb < NA; ++kb) {
            s[kb][r] =
                __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale_log2, nl[(r / 4) % 2][r % 4]));
            if constexpr (r % 2 == 1) pk[kb][r / 2] = round2(s[kb][r - 1], s[kb][r]);
        }
        if constexpr (r % 4 == 3 && r + 5 < 16) nl[(r / 4) % 2] = lds_quad(nl_base + 8 * (r + 5));
    };
    // Scores of hidden pairs: their weights come out as exactly 0.
    auto hide = [&](int q0, auto na, Scores& x_) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < decltype(na)::value; ++kb) {
            if constexpr (FOLDED) {
                const int lim = wk0 + kb * KSTEP + l32 - diag;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x_.s[kb][r] = position(a, q0 + acc_row(r, hh)) >= lim ? x_.s[kb][r] : a.hidden;
                continue;
            }
            const int lim = wk0 + kb * KSTEP + l32 - q0 - diag - 4 * hh;
#pragma unroll
            for (int r = 0; r < 16; ++r) x_.s[kb][r] = acc_row(r, 0) >= lim ? x_.s[kb][r] : a.hidden;
        }
    };
    auto grad = [&](auto r_tag, auto na, Scores& x_) __attribute__((always_inline)) {
        f32x16(&s)[KB] = x_.s;
        f32x16(&dp)[KB] = x_.dp;
        constexpr int r = decltype(r_tag)::value;
#pragma unroll
        for (int kb = 0; kb < decltype(na)::value; ++kb) {
            dp[kb][r] *= s[kb][r];
            if constexpr (r % 2 == 1) {
                dsk[kb][r / 2] = round2(dp[kb][r - 1], dp[kb][r]);
                here(dsk[kb][r / 2]);
            }
        }
    };
    auto start_dp = [&](auto r4_tag, Scores& x_) __attribute__((always_inline)) {
        constexpr int r4 = decltype(r4_tag)::value;
        const f32x4 x = lds_quad(nl_base + 128 + 32 * r4);
#pragma unroll
        for (int e = 0; e < 4; ++e) x_.nd[4 * r4 + e] = x[e];
    };
    constexpr int TAIL = OPS - Ring::ahead(0) + 1;  // the last slots, behind the barrier
    auto body = [&](int q0, auto na) __attribute__((always_inline)) {
        constexpr int NA = decltype(na)::value;
        Scores x;
        static_for<0, TAIL>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
            static_for<Ring::ahead(i - 1), Ring::ahead(i)>(fetch);
            if constexpr (ph == 0 && j >= KD - 4)
                start_dp(std::integral_constant<int, j - (KD - 4)>{}, x);
            if constexpr (ph == 0 && j == KD - 1) {
                x.nl[0] = lds_quad(nl_base);
                x.nl[1] = lds_quad(nl_base + 32);
            }
            static_for<0, NA>([&](auto kb_tag) __attribute__((always_inline)) {
                product(i_tag, kb_tag, x);
                // 12 of the 16 rows' weights in the gaps of dP (but for the first slot's,
                // when S settles), 4 in the first half of dV's; dS in dV's
                constexpr int n = NA * KD, gap = j * NA + decltype(kb_tag)::value;
                auto w = [&](auto r) __attribute__((always_inline)) { weight(r, na, x); };
                if constexpr (ph == 1 && j > 0)
                    static_for<(gap - NA) * 12 / (n - NA), (gap - NA + 1) * 12 / (n - NA)>(w);
                if constexpr (ph == 2 && gap < n / 2)
                    static_for<12 + gap * 4 / (n / 2), 12 + (gap + 1) * 4 / (n / 2)>(w);
                if constexpr (ph == 2 && j > 0)
                    static_for<(gap - NA) * 16 / (n - NA), (gap - NA + 1) * 16 / (n - NA)>(
                        [&](auto r) __attribute__((always_inline)) { grad(r, na, x); });
                slot_end();
            });
            if constexpr (ph == 1 && j == 0) {
                settle<0, NA>(x.s);
                if (CAUSAL && (FOLDED ? 0 : q0) + diag < wk0 + (NA - 1) * KSTEP + 31)
                    hide(q0, na, x);
            }
            if constexpr (ph == 2 && j == 0) settle<0, NA>(x.dp);
            slot_end();
        });
    };

    int qt = load_qt;
    issue(0);  // (a part has at least one step)
    {
        const uint32_t own = rows0 + L::OWN + wave * L::OWN_WAVE;
        const uint32_t slab = (uint32_t)a.Skv * D * 2;
        const long long at = (long long)bh * a.Skv * D;
        const dma_rsrc_t k_rsrc = make_dma_rsrc(a.k + at, slab);
        const dma_rsrc_t v_rsrc = make_dma_rsrc(a.v + at, slab);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int row = wk0 + kb * KSTEP;
            own_load<D>(k_rsrc, own + kb * L::TILE, row, a.Skv, lane);
            own_load<D>(v_rsrc, own + L::OWN_WAVE / 2 + kb * L::TILE, row, a.Skv, lane);
        }
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        own_read<D>(kf, read, own);
        own_read<D>(vf, read, own + L::OWN_WAVE / 2);
    }
    publish_barrier<0>();  // (all have read their own: its place is free)
    if (begin + 1 < end) issue(1);
    tile_bases(0);
    static_for<0, Ring::ahead(-1)>(fetch);
    int slot = 0, step = begin;
    auto tile = [&](auto na) __attribute__((always_inline)) {
        // (a wave whose keys are all hidden computes zeros: it would only wait)
        body(qt * 32, na);
        if (CAUSAL && ++qt == n_qt) qt = qt0;
        // Every operand of this tile has been read: its slot is free behind the barrier,
        // which also publishes the next tile.
        publish_barrier<0>();
        if (step + 2 < end) issue(slot);
        slot ^= 1;
        tile_bases(slot);
        Scores none;  // (dK's products read dsk alone)
        static_for<TAIL, OPS>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value;
            static_for<0, decltype(na)::value>(
                [&](auto kb_tag) __attribute__((always_inline)) { product(i_tag, kb_tag, none); });
            static_for<Ring::ahead(i - 1) - OPS, Ring::ahead(i) - OPS>(fetch);
            slot_end();
        });
        ++step;
    };
    // every wave's second block hidden (four of a diagonal's eight tiles) or past the keys
    const int second = k0 + KSTEP < a.Skv ? k0 + KSTEP : INT_MAX;
    auto half = [&]() __attribute__((always_inline)) {
        return KB == 2 && (MASK == kCausalMask ? qt * 32 + 31 + diag < second : second == INT_MAX);
    };
    while (step < end) {
        if constexpr (KB == 2)
            while (step < end && half()) tile(std::integral_constant<int, 1>{});
        while (step < end && !half()) tile(std::integral_constant<int, KB>{});
    }

    __syncthreads();  // the stages overlay the tiles
    const bool part = splits > 1;
    const long long rows = a.kv_heads * a.Skv, row0 = (long long)bh * a.Skv + wk0;
    void* dk_out = part ? a.part_k + split * rows * D : a.dk;
    void* dv_out = part ? a.part_v + split * rows * D : a.dv;
    const long long last = (long long)(bh + 1) * a.Skv;
    char* stage = lds + wave * stage_bytes<D>();
    const int bf16 = part ? 0 : a.out_bf16;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        store_rows<D>(dk[kb], stage, dk_out, row0 + kb * KSTEP, last, bf16, a.scale);
        store_rows<D>(dv[kb], stage, dv_out, row0 + kb * KSTEP, last, bf16, 1.f);
    }
}

// ---------------------------------------------------------------------- dQ --
// One block of queries (of the group of kv head kvh, over the batch), part `split` of
// `splits` of its sum.
template <int D, int MASK>
__device__ __forceinline__ void dq_block(const BwdArgs& a, char* lds, int kvh, int block,
                                         int split, int splits) {
    constexpr bool CAUSAL = MASK != kNoMask, FOLDED = MASK == kFoldedMask;
    constexpr int QB = BwdShape<D>::BLOCKS, KD = D / 16, CB = D / 32;
    typedef BwdLds<D> L;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // The wave's tiles of 32 queries are WAVES apart in the block, as the keys in
    // dkdv_block; where the block has a tile to a wave at most, they are the second ones.
    // (Outside of the block's tiles: the nearest one again, and nothing stored.)
    constexpr int WAVES = BwdShape<D>::WAVES;
    const int n_qt = (a.Sq + 31) / 32, tiles = n_qt * a.group;
    const int block0 = block * (BwdShape<D>::ROWS / 32);
    const bool one = QB == 2 && block0 + WAVES >= tiles;
    const int tile0 = one ? block0 - WAVES : block0;
    int wq0[QB];         // first query
    long long head[QB];  // of which head, over the batch
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int t = min(max(tile0 + qb * WAVES + wave, block0), tiles - 1);
        const int qt = __builtin_amdgcn_readfirstlane(t / a.group);
        wq0[qb] = qt * 32;
        head[qb] = (long long)kvh * a.group + (t - qt * a.group);
    }
    bf16x8 qf[QB][KD], gf[QB][KD];  // B operands: lane l holds query l%32
    float nl[QB];
    f32x16 nd[QB];  // -delta, from which the products of dP start
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float* rows = a.rows + (head[qb] * n_qt + wq0[qb] / 32) * 64;
        nl[qb] = rows[l32];
        const float x = rows[32 + l32];
#pragma unroll
        for (int r = 0; r < 16; ++r) nd[qb][r] = x;
    }
    f32x16 dq[QB][CB] = {};

    const int diag = a.diag;
    const int steps = a.units.size.q_steps(block);
    const int begin = (int)((long long)steps * split / splits);
    const int end = (int)((long long)steps * (split + 1) / splits);

    TileLoad<D> load;
    load.init(wave, lane);
    TileRead<D> read;
    read.init(lane);
    const uint32_t lds0 = lds_address(lds) + L::SLOTS;
    const uint32_t slab = (uint32_t)a.Skv * D * 2;
    const dma_rsrc_t k_rsrc = make_dma_rsrc(a.k + (long long)kvh * a.Skv * D, slab);
    const dma_rsrc_t v_rsrc = make_dma_rsrc(a.v + (long long)kvh * a.Skv * D, slab);
    auto issue = [&](int step, int slot) __attribute__((always_inline)) {
        const uint32_t dst = lds0 + slot * L::SLOT;
        load.issue(k_rsrc, v_rsrc, dst, step * 32, a.Skv, wave);
    };

    // Operand i of a step: K by rows (S of this tile), K transposed (dQ of the tile before:
    // its dS is formed during the products of S), V by rows (dP of this tile); KD of each.
    typedef QRing<D> Ring;
    constexpr int OPS = Ring::OPS, RING = Ring::SIZE;
    static_assert(OPS == 3 * KD && OPS % RING == 0, "");
    bf16x8 ring[RING];
    uint32_t row_base, col_base;
    auto fetch = [&](auto i_tag) __attribute__((always_inline)) {
        constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
        if constexpr (ph == 0) ring[i % RING] = TileRead<D>::template by_row<j>(row_base, 0);
        if constexpr (ph == 1)
            ring[i % RING] = TileRead<D>::template by_col<j % CB, j / CB>(col_base, 0);
        if constexpr (ph == 2)
            ring[i % RING] = TileRead<D>::template by_row<j>(row_base, L::TILE);
    };
    f32x16 s[QB], p[QB] = {}, dp[QB] = {};  // (no tile before the first: its dS is 0)
    uint32_t dsk[QB][8];  // dS as operands
    auto product = [&](auto i_tag, auto qb_tag) __attribute__((always_inline)) {
        constexpr int i = decltype(i_tag)::value, qb = decltype(qb_tag)::value;
        constexpr int ph = i / KD, j = i % KD, t = j / CB, cb = j % CB;
        const bf16x8 x = ring[i % RING];
        if constexpr (ph == 0 && j == 0) score_first<true>(s[qb], x, qf[qb][j]);
        if constexpr (ph == 0 && j > 0) score_add<true>(s[qb], x, qf[qb][j]);
        if constexpr (ph == 1) {
            const u32x4 y = {dsk[qb][4 * t], dsk[qb][4 * t + 1], dsk[qb][4 * t + 2],
                             dsk[qb][4 * t + 3]};
            dq[qb][cb] = mfma(x, __builtin_bit_cast(bf16x8, y), dq[qb][cb]);
        }
        if constexpr (ph == 2 && j == 0) score_from<true>(dp[qb], x, gf[qb][j], nd[qb]);
        if constexpr (ph == 2 && j > 0) score_add<true>(dp[qb], x, gf[qb][j]);
    };
    // (QF: the first of the blocks at work, the last ones; the others' weights are 0)
    auto weight = [&](auto r_tag, auto qf_tag) __attribute__((always_inline)) {
        constexpr int r = decltype(r_tag)::value, QF = decltype(qf_tag)::value;
#pragma unroll
        for (int qb = 0; qb < QF; ++qb) p[qb][r] = 0.f;
#pragma unroll
        for (int qb = QF; qb < QB; ++qb) {
            float x = __builtin_amdgcn_exp2f(fmaf(s[qb][r], a.scale_log2, nl[qb]));
            here(x);
            p[qb][r] = x;
        }
    };
    // Scores of hidden pairs and of keys past Skv: their weights come out as exactly 0.
    auto hide = [&](int k0, auto qf_tag) __attribute__((always_inline)) {
#pragma unroll
        for (int qb = decltype(qf_tag)::value; qb < QB; ++qb) {
            const int q = wq0[qb] + l32;
            const int last =
                CAUSAL ? min(a.Skv - 1, (FOLDED ? position(a, q) : q) + diag) : a.Skv - 1;
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
    constexpr int TAIL = OPS - Ring::ahead(0) + 1;  // the last slots, behind the barrier
    auto body = [&](int k0, auto qf_tag) __attribute__((always_inline)) {
        constexpr int QF = decltype(qf_tag)::value;
        static_for<0, TAIL>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value, ph = i / KD, j = i % KD;
            static_for<Ring::ahead(i - 1), Ring::ahead(i)>(fetch);
            // dS of the tile before in the gaps of S; 12 of the 16 rows' weights in those
            // of dQ, 4 in those of dP; the first slots are left to settle
            constexpr int Q0 = ph == 1 ? 0 : QF, NQ = QB - Q0;  // (dQ: of all blocks)
            static_for<Q0, QB>([&](auto qb_tag) __attribute__((always_inline)) {
                product(i_tag, qb_tag);
                constexpr int gap = j * NQ + decltype(qb_tag)::value - Q0;
                constexpr int M = NQ * (KD - 1), B = NQ * (KD - (OPS - TAIL));
                auto w = [&](auto r) __attribute__((always_inline)) { weight(r, qf_tag); };
                if constexpr (ph == 0 && j > 0)
                    static_for<(gap - NQ) * 16 / M, (gap - NQ + 1) * 16 / M>(grad);
                if constexpr (ph == 1 && j > 0)
                    static_for<(gap - NQ) * 12 / M, (gap - NQ + 1) * 12 / M>(w);
                if constexpr (ph == 2) static_for<12 + gap * 4 / B, 12 + (gap + 1) * 4 / B>(w);
                slot_end();
            });
            if constexpr (ph == 0 && j == 0) settle<0, QB>(dp);
            if constexpr (ph == 1 && j == 0) {
                settle<QF, QB>(s);
                if (k0 + 32 > a.Skv || (CAUSAL && k0 + 31 > (FOLDED ? 0 : wq0[QF]) + diag))
                    hide(k0, qf_tag);
            }
            slot_end();
        });
    };
    // dQ of the wave's last tile.
    auto drain = [&]() __attribute__((always_inline)) {
        settle<0, QB>(dp);
        static_for<0, 16>(grad);
        static_for<KD, KD + 3>(fetch);
        static_for<KD, 2 * KD>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value;
            if constexpr (i + 3 < 2 * KD) fetch(std::integral_constant<int, i + 3>{});
            static_for<0, QB>(
                [&](auto qb_tag) __attribute__((always_inline)) { product(i_tag, qb_tag); });
            slot_end();
        });
    };

    int slot = 0;
    issue(begin, 0);  // (a part has at least one step)
    {
        const uint32_t own = lds_address(lds) + L::OWN + wave * L::OWN_WAVE;
        const uint32_t slab = (uint32_t)a.Sq * D * 2;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const long long at = head[qb] * a.Sq * D;
            own_load<D>(make_dma_rsrc(a.q + at, slab), own + qb * L::TILE, wq0[qb], a.Sq, lane);
            own_load<D>(make_dma_rsrc(a.d_o + at, slab), own + L::OWN_WAVE / 2 + qb * L::TILE,
                        wq0[qb], a.Sq, lane);
        }
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        own_read<D>(qf, read, own);
        own_read<D>(gf, read, own + L::OWN_WAVE / 2);
    }
    publish_barrier<0>();  // (all have read their own: its place is free)
    if (begin + 1 < end) issue(begin + 1, 1);
    row_base = read.row + lds0;
    static_for<0, Ring::ahead(-1)>(fetch);
    int step = begin;
    auto tile = [&](auto qf_tag) __attribute__((always_inline)) {
        // (before the first tile: itself, with a dS of 0)
        const int prev = slot == 0 ? 2 : slot - 1, next = slot == 2 ? 0 : slot + 1;
        // opaque, so that the XORed addresses are formed where they are used instead of
        // being kept in registers over the whole loop
        row_base = read.row + lds0 + slot * L::SLOT;
        col_base = read.col + lds0 + (step == begin ? slot : prev) * L::SLOT;
        asm volatile("" : "+v"(row_base), "+v"(col_base));
        // (a wave whose pairs are all hidden computes zeros: it would only wait)
        body(step * 32, qf_tag);
        // The tile before has been read for good: its slot is free behind the barrier,
        // which also publishes the next tile.
        publish_barrier<0>();
        if (step + 2 < end) issue(step + 2, prev);
        row_base = read.row + lds0 + next * L::SLOT;
        asm volatile("" : "+v"(row_base));
        static_for<TAIL, OPS>([&](auto i_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(i_tag)::value;
            static_for<decltype(qf_tag)::value, QB>(
                [&](auto qb_tag) __attribute__((always_inline)) { product(i_tag, qb_tag); });
            static_for<Ring::ahead(i - 1) - OPS, Ring::ahead(i) - OPS>(fetch);
            slot_end();
        });
        slot = next;
        ++step;
    };
    // every wave's first block hidden: four of a diagonal's eight tiles, the last ones
    const int half =
        one ? begin
        : MASK == kCausalMask && QB == 2
            ? min(end, (min(tile0 + WAVES, tiles) - 1) / a.group + (31 + diag) / 32 + 1)
            : end;
    while (step < half) tile(std::integral_constant<int, 0>{});
    if constexpr (QB == 2)
        while (step < end) tile(std::integral_constant<int, 1>{});
    col_base = read.col + lds0 + (slot == 0 ? 2 : slot - 1) * L::SLOT;
    drain();

    __syncthreads();  // the stages overlay the tiles
    const bool part = splits > 1;
    void* out = part ? a.part_q + split * a.q_heads * a.Sq * D : a.dq;
    char* stage = lds + wave * stage_bytes<D>();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int t = tile0 + qb * WAVES + wave;
        const long long last = t >= block0 && t < tiles ? (head[qb] + 1) * a.Sq : 0;
        store_rows<D>(dq[qb], stage, out, head[qb] * a.Sq + wq0[qb], last,
                      part ? 0 : a.out_bf16, a.scale);
    }
}

// ------------------------------------------------------------------ kernel --
// Workgroups: for every key/value head, the parts of its blocks of keys and of its group's
// blocks of queries, in one launch, so that the one kind fills the other's gaps.
// The hardware deals workgroups round-robin to the XCDs; each XCD gets whole heads, whose
// tiles stay in its L2, where they can be dealt evenly.
//
// Bound by the matrix cores, and in long calls by the clock that they run at: B1 H32 S8192
// d128 2.93 ms, 1.31 PFLOP/s in the seven products, MFMA busy 62% at 2.0 of 2.4 GHz (a large
// GEMM of this library reaches 1.24 on the same card).  Short causal calls also show a
// workgroup's start and end, some 7 us each, which nothing overlaps with one wave to a SIMD:
// B4 H16 S2048 d128 244 us in counter passes, 280 traced back to back: 0.99 and 0.86 PFLOP/s
// over the pairs that are not hidden.  Few queries are bound by HBM: both kinds of blocks read
// all of K and V (causal B2 Hq64 Hkv8 Sq6 Skv18702 d128 108 us, 453 MB for the necessary 307).
template <int D, int MASK>
__global__ __launch_bounds__(
    BwdShape<D>::THREADS, BwdShape<D>::WAVES_PER_SIMD) void bwd_kernel(
    const BwdArgs a, const typename std::conditional<(MASK > 0), BwdOrder, int>::type order) {
    __shared__ __attribute__((aligned(1024))) char lds[BwdLds<D>::BYTES];
    const int heads = (int)a.kv_heads;
    const bool even = heads % a.num_xcds == 0;
    const int first = even ? (int)(blockIdx.x % a.num_xcds) * (heads / a.num_xcds) : 0;
    const BwdUnit* named = nullptr;
    if constexpr (MASK != kNoMask) named = order.unit;
    const BwdWork w = bwd_work(a.units, named, even ? heads / a.num_xcds : heads,
                               even ? (int)(blockIdx.x / a.num_xcds) : (int)blockIdx.x);
    const int head = first + w.head;
    if (w.kv)
        dkdv_block<D, MASK>(a, lds, head, w.block, w.split, w.splits);
    else
        dq_block<D, MASK>(a, lds, head, w.block, w.split, w.splits);
}

// Adds up the parts of the blocks that have several, in their order, four values to a
// thread: dK and dV (z = 0, 1), dQ (2).  HBM bound: B2 Hq32 Hkv8 S1777 d128 8.2 us.
template <int D>
__global__ __launch_bounds__(256) void bwd_sum_kernel(const BwdArgs a) {
    const bool q = blockIdx.z == 2;
    const int S = q ? a.Sq : a.Skv;
    const long long rows = (q ? a.q_heads : a.kv_heads) * S;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = i / (D / 4);
    if (row >= rows) return;
    const int at = (int)(row % S), g = (int)(row / S % a.group);  // (g: of a query)
    const int n = a.units.parts(!q, q ? (at / 32 * a.group + g) / (BwdShape<D>::ROWS / 32)
                                      : at / BwdShape<D>::ROWS);
    if (n == 1) return;
    const float* part = (q ? a.part_q : blockIdx.z ? a.part_v : a.part_k) + i * 4;
    void* out = q ? a.dq : blockIdx.z ? a.dv : a.dk;
    f32x4 s = *reinterpret_cast<const f32x4*>(part);
#pragma unroll 4
    for (int j = 1; j < n; ++j) s += *reinterpret_cast<const f32x4*>(part + j * rows * D);
    if (a.out_bf16) {
        const uint64_t y = (uint64_t)round2(s[2], s[3]) << 32 | round2(s[0], s[1]);
        *reinterpret_cast<uint64_t*>(static_cast<uint16_t*>(out) + i * 4) = y;
    } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(out) + i * 4) = s;
    }
}

template <int D>
hipError_t launch_d(const BwdPlan& p, const BwdArgs& a, int o_bf16, hipStream_t stream) {
    const long long slots = a.q_heads * ((a.Sq + 31) / 32) * 32 * (D / 8);
    const dim3 row_grid((unsigned)((slots + 255) / 256));
    if (o_bf16)
        bwd_rows_kernel<D, true><<<row_grid, 256, 0, stream>>>(a);
    else
        bwd_rows_kernel<D, false><<<row_grid, 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)p.grid);
    if (a.period)
        bwd_kernel<D, kFoldedMask><<<grid, BwdShape<D>::THREADS, 0, stream>>>(a, p.order);
    else if (a.causal)
        bwd_kernel<D, kCausalMask><<<grid, BwdShape<D>::THREADS, 0, stream>>>(a, p.order);
    else
        bwd_kernel<D, kNoMask><<<grid, BwdShape<D>::THREADS, 0, stream>>>(a, 0);
    e = hipGetLastError();
    if (e != hipSuccess || (!p.kv_chunk && !p.q_chunk)) return e;
    const long long kv_rows = p.kv_chunk ? a.kv_heads * a.Skv : 0;
    const long long q_rows = p.q_chunk ? a.q_heads * a.Sq : 0;
    const long long quads = (kv_rows > q_rows ? kv_rows : q_rows) * (D / 4);
    bwd_sum_kernel<D><<<dim3((unsigned)((quads + 255) / 256), 1, p.q_chunk ? 3 : 2), 256, 0,
                        stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_bwd(const BwdPlan& p, const BwdArgs& args, int d, int o_bf16,
                      hipStream_t stream) {
    BwdArgs a = args;
    a.units = {{bwd_block_rows(d), a.Sq, a.Skv, a.group, a.causal, a.diag},
               p.kv_blocks, p.q_blocks, p.kv_units, p.q_units, p.kv_chunk, p.q_chunk, p.ordered};
    // the parts follow the row values
    const long long kv_values = a.kv_heads * a.Skv * d;
    a.part_k = a.rows + a.q_heads * ((a.Sq + 31) / 32) * 64;
    a.part_v = a.part_k + p.kv_parts * kv_values;
    a.part_q = a.part_v + p.kv_parts * kv_values;
    return d == 64 ? launch_d<64>(p, a, o_bf16, stream) : launch_d<128>(p, a, o_bf16, stream);
}

}  // namespace attn
