// Attention of requests with few new tokens over a paged cache.
//
// For request r, new token i (position pos = kv - n + i) and query head h, over the keys j that
// the token sees (j <= pos under a causal mask, j > pos - window with a window):
//     x_j = scale q.k_j,  capped: cap tanh(x_j / cap),  with slopes: x_j - slope_h |pos - j|,
//     o = sum_j exp(x_j) v_j / sum_j exp(x_j),  lse = log sum_j exp(x_j),
// o = 0 and lse = -inf where a token sees no key.
//
// The new tokens of all query heads that share a key/value head are the rows of one product, 16 MT
// at most, token by token (row = token * group + head of the group), so that each key is read
// once for all of them.  Products on v_mfma_f32_16x16x32_bf16: S^T = K Q^T and
// O^T += V^T P^T, both operands through a wave's own tiles in LDS, V read transposed.  A step is
// 32 keys to each of four or eight waves; what a lane gets of S^T, eight keys of one row, is the
// operand that its P^T has to be.  A wave's 32 keys are four aligned runs of eight, each in one
// page, whose number is read a step ahead.
//
// Bound: HBM, 4 D bytes a key.  All items (request, key/value head) one behind another
// are one line of steps, which the workgroups share out evenly whatever the requests'
// lengths are; no length is known to the host.  Each workgroup finds its part by summing the
// lengths itself (one launch less than a plan of its own).  An item that lies in several
// workgroups leaves partial sums (unnormalised, with their maximum), which a second kernel adds in
// order: no atomics, the same bits every call.  A workgroup has two of them at most, one for an
// item that began before it and one for an item that goes on behind it.  Short items stay whole,
// without a second launch.
//
// Memory.  Whole rows, 1 KiB to an instruction, straight into LDS and past the caches: 6.5 TB/s
// over a long batch (16 requests of 8192 keys, 32 heads: 332 us for 2.1 GB).  With the cache 6.0;
// loads of K's operands as they are needed, 64 bytes of 16 rows each, 5.4 to 5.8.  Where the
// workgroups have a few steps each, their start (3 us) and the adding up (4 us) count: 16 tokens
// over 73k keys of 8 heads 55 us, 5.4 TB/s; one over 512 keys 9 us.
//
// Only the aligned runs of eight rows that hold a key in [lo, kv) are read, lo being the first that
// any of the request's tokens sees: a run past these is the nearest of them again.  The scores of
// keys outside [lo, kv) are masked, and their rows of V become zeros in LDS, whatever the page
// holds there.  A page number outside the cache is replaced by 0 and makes the request's results
// NaN.
//
// The scalars of a workgroup's share, of its item and of both descriptors are more than there are
// scalar registers: 76 to 86 of them lie in lanes of a vector register, most through the loop.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "lds_dma.h"
#include "paged.h"
#include "paged_device.h"

namespace attn {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int kNT = 256;  // of the sum kernel
constexpr float kLn2 = 0.69314718055994531f;

// max / sum of x over the four 16-lane rows (lanes l, l^16, l^32, l^48)
__device__ __forceinline__ float rows4_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows4_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// o / l and the log-sum-exp of 4 of a row's values; a row without keys (l = 0) is 0, -inf.
template <int D>
__device__ __forceinline__ void store_row(const PagedArgs& a, long long token, int head, int col,
                                          f32x4 acc, float M, float L) {
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const long long at = (token * a.Hq + head) * D + col;
    if (a.out_bf16) {
        const bf16x4 y = {(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv),
                          (__bf16)(acc[3] * inv)};
        *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(a.o) + at) = y;
    } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at) = acc * inv;
    }
    if (a.lse && col == 0)
        a.lse[token * a.Hq + head] = L == 0.f ? -INFINITY : (M + __builtin_log2f(L)) * kLn2;
}

// A step's 32 keys of a wave in LDS: whole rows, 1 KiB (4 or 8 rows) to a load, K's pieces 16
// bytes apart.  A row's 16-byte pieces are exchanged inside it (by the source address of each
// lane), so that K's reads (16 rows of one piece) and V's (8 rows of 32 bytes) are free of bank
// conflicts.
template <int D>
struct RowLds {
    static constexpr int PIECE_ROWS = 512 / D, PIECES = 32 / PIECE_ROWS;
    static constexpr int K_PIECE = 1024 + 16, V_PIECE = 1024;
    static constexpr int K_BYTES = PIECES * K_PIECE, V_BYTES = PIECES * V_PIECE;
    static constexpr int WAVE = K_BYTES + V_BYTES;
    __device__ static constexpr int k_swap(int row) {
        return D == 128 ? 4 * (row & 3) : 2 * ((row >> 1) & 3);
    }
    __device__ static constexpr int v_swap(int row) {
        return D == 128 ? 4 * (row & 3) ^ 2 * ((row >> 2) & 1) : 2 * ((row >> 1) & 3);
    }
};

// Past the caches: each row is read once.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_past(dma_rsrc_t rsrc, uint32_t dst, int voffset, int soffset) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, %3 offen nt lds"
        :
        : "s"(dst), "v"(voffset), "s"(rsrc), "s"(soffset)
        : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

template <int D, int MT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void paged_rows_kernel(const PagedArgs a) {
    using L = RowLds<D>;
    constexpr int NT = NW * 64;
    constexpr int KEYS = 32 * NW;    // of a step
    constexpr int KS = D / 32;       // MFMA steps over a row
    constexpr int DB = D / 16;       // 16-column blocks of O^T
    constexpr int OST = D + 4;       // floats to a row where the waves meet
    constexpr int BLOCK = 16 * MT;
    constexpr int LOADS = L::PIECES; // of an operand and step
    __shared__ __attribute__((aligned(16))) uint8_t lds[NW * L::WAVE];
    __shared__ float sm[NW][BLOCK], sl[NW][BLOCK];
    __shared__ int found[2];
    static_assert(NW * 16 * OST * 4 <= (int)sizeof(lds), "");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    int* const meta = a.meta + (long long)blockIdx.x * kPagedMeta;
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };

    // ---- this workgroup's part of the line of all units ------------------------
    // (less than 2^31 of them: the host chose their size)  Up to 64 requests: each wave by itself.
    auto units_of = [&](const PagedRequest& x) {
        const Share s = share_of(a, x, KEYS);
        return s.items * s.units;
    };
    const bool alone = a.R <= 64;
    const int first_r = alone ? lane : tid;
    PagedRequest x = {0, 0, 0, 0, 0, 0};
    int mine = 0, sum = 0;  // (up to NT requests: this thread's alone)
    for (int r = first_r; r < a.R; r += NT) {
        x = paged_request(a, r);
        mine = units_of(x);
        sum += mine;
    }
    int total, upto;
    if (alone) {
        upto = wave_scan(sum);
        total = __builtin_amdgcn_readlane(upto, 63);
    } else {
        upto = block_scan<NT>(sum, &total);
    }
    const int n_wg = min(a.n_wg, total), wg = blockIdx.x;
    if (a.meta && tid == 0) meta[0] = 0;
    if (wg >= n_wg) return;
    // the first `more` workgroups have a unit more than the others
    const int per = (uint32_t)total / (uint32_t)n_wg, more = total - per * n_wg;
    const int u0 = per * wg + min(wg, more), u1 = u0 + per + (wg < more);
    int r, r_first;  // request, its first unit
    if (alone) {
        const unsigned long long here = __ballot(u0 >= upto - mine && u0 < upto);
        r = __ffsll((long long)here) - 1;
        auto from = [&](int v) { return __builtin_amdgcn_readlane(v, r); };
        r_first = from(upto - mine);
        x = {from(x.q0), from(x.qn), from(x.pos0), from(x.kv), from(x.lo), from(x.bad)};
    } else {
        int before = 0;
        for (int r0 = 0; r0 < a.R; r0 += NT) {
            int all = total;
            if (a.R > NT) {
                mine = 0;
                if (r0 + tid < a.R) {
                    x = paged_request(a, r0 + tid);
                    mine = units_of(x);
                }
                upto = block_scan<NT>(mine, &all);
            }
            if (u0 < before + all) {
                const int first = before + upto - mine;
                if (u0 >= first && u0 < first + mine) {
                    found[0] = r0 + tid;
                    found[1] = first;
                }
                break;
            }
            before += all;
        }
        __syncthreads();
        r = uniform(found[0]);
        r_first = uniform(found[1]);
        x = paged_request(a, r);
    }

    const int page_mask = (1 << a.page_log2) - 1;
    const uint32_t k_lds = lds_address(lds) + wave * L::WAVE, v_lds = k_lds + L::K_BYTES;
    uint8_t* const k_tile = lds + wave * L::WAVE;
    uint8_t* const v_tile = k_tile + L::K_BYTES;
    // this lane's place in a 1 KiB piece, and its source (V: in even and in odd pieces)
    const int p_row = lane / (D / 8), p_chunk = lane % (D / 8);
    const int k_off = p_row * (int)a.k.row16 * 16 + (p_chunk ^ L::k_swap(p_row)) * 16;
    const int v_off0 = p_row * (int)a.v.row16 * 16 + (p_chunk ^ L::v_swap(p_row)) * 16;
    const int v_off1 =
        p_row * (int)a.v.row16 * 16 + (p_chunk ^ L::v_swap(p_row + L::PIECE_ROWS)) * 16;
    // operands: K row l16 (and + 16), piece 4 s + g4; V rows 4 g4 + l16 / 4 (and + 16), column
    // 16 db + 4 (l16 % 4)
    const int k_row = (l16 / L::PIECE_ROWS) * L::K_PIECE + (l16 % L::PIECE_ROWS) * (D * 2);
    constexpr int K_16 = 16 / L::PIECE_ROWS * L::K_PIECE;
    const int tr_row = 4 * g4 + (l16 >> 2);
    const int v_row = tr_row * (D * 2) + 8 * (l16 & 1);
    for (int u = u0; u < u1;) {
        const Share share = share_of(a, x, KEYS);
        const int mine_here = share.items * share.units;
        if (u >= r_first + mine_here) {  // the next request that has any
            r_first += mine_here;
            for (++r;; r += 64) {
                const int rr = min(r + lane, a.R - 1);
                const Share s = share_of(a, paged_request(a, rr), KEYS);
                const unsigned long long any = __ballot(s.items > 0 && r + lane < a.R);
                if (any) {
                    r += __ffsll((long long)any) - 1;
                    break;
                }
                if (r + 64 >= a.R) return;  // (never: u1 <= total)
            }
            r = uniform(r);
            x = paged_request(a, r);
            continue;
        }
        const int head = (uint32_t)(u - r_first) / (uint32_t)share.units;
        const int unit0 = u - r_first - head * share.units;
        const int unit1 = min(share.units, unit0 + (u1 - u));
        const int t0 = unit0 << a.unit_log2, t1 = min(share.steps, unit1 << a.unit_log2);
        const int item_first = u - unit0;  // of the line
        u += unit1 - unit0;
        const int n_rows = x.qn * a.group;  // (few at most, which is no more than BLOCK)
        const GroupDiv rows(a, 0);

        // ---- loads of a step: a wave's 32 keys, in aligned runs of eight ------------------
        const uint16_t* const k_head = a.k.ptr + head * a.k.head;
        const uint16_t* const v_head = a.v.ptr + head * a.v.head;
        const int* const table = a.table + (long long)r * a.table_stride;
        int bad = x.bad;
        const bool any_keys = x.kv > x.lo;
        const int key0 = x.lo / KEYS * KEYS + 32 * wave;
        // first key of a run, clamped to the runs that hold a key that some row sees
        auto run_of = [&](int t, int i) __attribute__((always_inline)) {
            return max(min(key0 + t * KEYS + 8 * i, (x.kv - 1) & ~7), x.lo & ~7);
        };
        // page numbers of a step's runs, in lanes 0 to 3
        auto entries = [&](int t) __attribute__((always_inline)) {
            int e = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int p = table[run_of(t, i) >> a.page_log2];
                if ((uint32_t)p >= (uint32_t)a.n_pages) {
                    p = 0;
                    bad = 1;
                }
                e = lane == i ? p : e;
            }
            return e;
        };
        auto load = [&](const PagedSide& side, const uint16_t* base, uint32_t dst, int piece,
                        int off0, int off1, int t, int e) __attribute__((always_inline)) {
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                const uint64_t at =
                    (uint64_t)(uint32_t)__builtin_amdgcn_readlane(e, i) * side.page16 +
                    (uint64_t)(uint32_t)(run_of(t, i) & page_mask) * side.row16;
                const dma_rsrc_t rsrc = make_dma_rsrc(base + at * 8, 0x7fffffffu);
                load_past(rsrc, uniform(dst), off0, 0);
                if constexpr (L::PIECE_ROWS == 4)
                    load_past(rsrc, uniform(dst + piece), off1, uniform(4 * side.row16 * 16));
                dst += piece * (8 / L::PIECE_ROWS);
            }
        };
        auto load_k = [&](int t, int e) __attribute__((always_inline)) {
            load(a.k, k_head, k_lds, L::K_PIECE, k_off, k_off, t, e);
        };
        auto load_v = [&](int t, int e) __attribute__((always_inline)) {
            load(a.v, v_head, v_lds, L::V_PIECE, v_off0, v_off1, t, e);
        };
        int entry = 0;

        // ---- this lane's queries: Q^T, dims 32 s + 8 g4 .. + 7 of row l16 -----------
        bf16x8 qf[MT][KS];
        int hi[MT], lo[MT], pos[MT];
        float slope[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            int h;
            const int tok = rows.token(min(mt * 16 + l16, n_rows - 1), &h);
            h += head * a.group;
            const uint16_t* qp = a.q + (x.q0 + tok) * a.q_row + h * a.q_head + 8 * g4;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 w = *reinterpret_cast<const u32x4*>(qp + 32 * s);
                w ^= a.q_sign;
                qf[mt][s] = __builtin_bit_cast(bf16x8, w);
            }
            pos[mt] = x.pos0 + tok;
            hi[mt] = a.causal ? min(pos[mt], x.kv - 1) : x.kv - 1;
            lo[mt] = a.window ? pos[mt] - a.window + 1 : 0;
            slope[mt] = a.slopes ? a.slopes[h] * 1.4426950408889634f : 0.f;
        }
        // keys from here to there are seen by every row
        int unused;
        const int all_hi = a.causal ? min(x.pos0 + rows.token(0, &unused), x.kv - 1) : x.kv - 1;
        const int all_lo =
            a.window ? x.pos0 + rows.token(n_rows - 1, &unused) - a.window + 1 : 0;

        float m[MT], l[MT];
        f32x4 oacc[MT][DB];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt] = -INFINITY;
            l[mt] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) oacc[mt][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        // One slot to an operand: K's next rows are asked for as soon as its operands are in
        // registers, V's likewise, so that a wave's 16 KiB are on their way nearly always.  (The
        // first step's loads are those of a step -1 without work: one copy of the code.)
        if (any_keys) entry = entries(t0);
        for (int t = any_keys ? t0 - 1 : t1; t < t1; ++t) {
            const int kb = key0 + t * KEYS;
            const bool work = t >= t0, more_steps = t + 1 < t1;
            bf16x8 kf[2][KS];
            if (work) {
                wait_loads<LOADS>();  // K's have landed (V's are newer)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        kf[b][s] = *reinterpret_cast<const bf16x8*>(
                            k_tile + b * K_16 + k_row + (((4 * s + g4) ^ L::k_swap(l16)) * 16));
                wait_lds();
            }
            if (more_steps) load_k(t + 1, entry);
            f32x4 sa[MT], sb[MT];
            if (work) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                sa[mt] = sb[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    sa[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0][s], qf[mt][s], sa[mt],
                                                                    0, 0, 0);
                    sb[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1][s], qf[mt][s], sb[mt],
                                                                    0, 0, 0);
                }
            }
            bf16x8 pf[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                // lane (row l16, g4) has keys kb + 4 g4 + e and, from e = 4 on, 12 further
                float sc[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[i] = sa[mt][i];
                    sc[4 + i] = sb[mt][i];
                }
                // log2 units; for |u| < 1 by tanh's series in y (the first term left out is
                // 2^-26 of it), so that small scores keep their bits: here is time for it
                if (a.cap_out != 0.f) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float u = sc[e] * a.cap_in;
                        const float y = u * 0.34657359028f, z = y * y;
                        float t = fmaf(z, -1382.f / 155925.f, 62.f / 2835.f);
                        t = fmaf(z, t, -17.f / 315.f);
                        t = fmaf(z, t, 2.f / 15.f);
                        t = fmaf(z, t, -1.f / 3.f);
                        t = fmaf(y * z, t, y) * a.cap_out;
                        sc[e] = fabsf(u) < 1.f ? t : capped(u, a.cap_out);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) sc[e] *= a.scale_log2;
                }
                const int kl = kb + 4 * g4;
                if (a.slopes) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sc[e] = fmaf(-slope[mt], (float)abs(pos[mt] - (kl + 12 * (e / 4) + e)),
                                     sc[e]);
                }
                if (kb + 31 > all_hi || kb < all_lo) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int key = kl + 12 * (e / 4) + e;
                        if (key > hi[mt] || key < lo[mt]) sc[e] = -INFINITY;
                    }
                }
                float mx = sc[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sc[e]);
                mx = rows4_max(mx);
                const float m_new = fmaxf(m[mt], mx);
                const float ref = m_new == -INFINITY ? 0.f : m_new;  // no key seen yet
                const float alpha = __builtin_amdgcn_exp2f(m[mt] - ref);
                l[mt] *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db) oacc[mt][db] *= alpha;
                m[mt] = m_new;
                // P is rounded to bf16 (at most 2^-8 of each weight) as the operand it has to
                // be; its sum takes the weights as they are, so that the log-sum-exp is fp32's
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = __builtin_amdgcn_exp2f(sc[e] - ref);
                    l[mt] += p;
                    pf[mt][e] = (__bf16)p;
                }
            }
                // O^T += V^T P^T, 16 columns at a time: lane i of 16 reads 4 values of row i / 4 of
                // four, and receives column i of these four keys
                if (more_steps)
                    wait_loads<LOADS>();  // V's have landed (K's next are newer)
                else
                    wait_loads<0>();
                if (kb < x.lo || kb + 32 > x.kv) {
                    // rows that no query sees hold what the page does: weights of 0 need numbers
#pragma unroll 1
                    for (int p = 0; p < L::PIECES; ++p) {
                        const int key = kb + p * L::PIECE_ROWS + p_row;
                        if (key < x.lo || key >= x.kv)
                            *reinterpret_cast<u32x4*>(v_tile + p * L::V_PIECE + lane * 16) =
                                u32x4{0u, 0u, 0u, 0u};
                    }
                    wait_lds();
                }
                bf16x8 vf[DB];
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const int chunk = 2 * db + ((l16 >> 1) & 1);
                    const uint8_t* const at = v_tile + v_row + (chunk ^ L::v_swap(tr_row)) * 16;
                    const s16x4 w0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(at));
                    const s16x4 w1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(at + 16 * D * 2));
                    const s16x8 w = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
                    vf[db] = __builtin_bit_cast(bf16x8, w);
                }
                wait_lds();
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        oacc[mt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            vf[db], pf[mt], oacc[mt][db], 0, 0, 0);
            }
            if (more_steps) {
                load_v(t + 1, entry);
                entry = entries(min(t + 2, t1 - 1));
            }
        }

        // ---- the waves meet, 16 rows at a time -----------------------------------
        bad = __syncthreads_or(bad);
        const bool whole = unit0 == 0 && unit1 == share.units;
        const int part = unit0 == 0 ? 1 : 0;
        if (!whole && tid == 0 && unit0 == 0) {  // the first part of an item: its others follow
            const int end = item_first + share.units - 1;  // its last unit, and whose it is
            const int big = more * (per + 1);
            const int last = end < big ? (uint32_t)end / (uint32_t)(per + 1)
                                       : more + (uint32_t)(end - big) / (uint32_t)per;
            meta[1] = x.q0;
            meta[2] = head * a.group;
            meta[3] = 0;
            meta[4] = n_rows;
            meta[0] = last - wg + 1;
        }
        // (addresses from an opaque copy of the thread's number: else they are computed before
        // the loop and kept in registers through it)
        int etid = tid;
        asm volatile("" : "+v"(etid));
        const int e16 = etid & 15, eg4 = (etid >> 4) & 3;
        float* const so = reinterpret_cast<float*>(lds);  // [wave][16][OST]
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt > 0) __syncthreads();
            const float lsum = rows4_sum(l[mt]);  // the lane groups have different keys
            if (eg4 == 0) {
                sm[wave][mt * 16 + e16] = m[mt];
                sl[wave][mt * 16 + e16] = bad ? NAN : lsum;
            }
#pragma unroll
            for (int db = 0; db < DB; ++db)
                *reinterpret_cast<f32x4*>(so + (wave * 16 + e16) * OST + 16 * db + 4 * eg4) =
                    oacc[mt][db];
            __syncthreads();
            for (int i = etid; i < 16 * D / 4; i += NT) {
                const int row = mt * 16 + i / (D / 4), col = i % (D / 4) * 4;
                if (row >= n_rows) break;
                float M = sm[0][row];
#pragma unroll
                for (int w = 1; w < NW; ++w) M = fmaxf(M, sm[w][row]);
                const float ref = M == -INFINITY ? 0.f : M;
                float L0 = 0.f;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float wt = __builtin_amdgcn_exp2f(sm[w][row] - ref);
                    L0 = fmaf(wt, sl[w][row], L0);
                    acc += wt * *reinterpret_cast<const f32x4*>(
                                    so + (w * 16 + row - mt * 16) * OST + col);
                }
                if (whole) {
                    int h;
                    const int tok = rows.token(row, &h);
                    store_row<D>(a, x.q0 + tok, head * a.group + h, col, acc, M, L0);
                } else {
                    const long long at = ((long long)wg * 2 + part) * BLOCK + row;
                    *reinterpret_cast<f32x4*>(a.ws_o + at * D + col) = acc;
                    if (col == 0) {
                        a.ws_m[at] = M;
                        a.ws_l[at] = L0;
                    }
                }
            }
        }
        __syncthreads();  // the tiles are V's again
    }
}

// Adds parts of rows, ROWS rows of an item to a workgroup.  After the row kernel (TILES false)
// item g is the one that begins in its workgroup g and does not end there: its first part is that
// workgroup's second one, the others are the following workgroups' first.  After the tile kernel
// item g is a block of a head, its splits one behind another.
//
// Bound by latency after the row kernel: few rows of many parts, just written by other CUs.  The
// lane groups of a row take every GP-th part, four on their way, and meet in LDS: 4.5 us after 16
// tokens over 73k keys.  After the tile kernel there are many rows of few parts (bound: HBM), and
// each lane group has its own: 7.8 us for the 34 MB of a chunk of 512 tokens in four splits.
template <int D, bool TILES>
constexpr int kSumRows = TILES ? kNT / (D / 4) : 256 / D;
template <int D, bool TILES>
__device__ __forceinline__ void sum_rows(const PagedArgs& a, int index, int block, int per) {
    constexpr int ROWS = kSumRows<D, TILES>;
    constexpr int LANES = D / 4, GROUPS = kNT / LANES, GP = GROUPS / ROWS, U = 4;
    const int g = (uint32_t)index / (uint32_t)per, row0 = (index - g * per) * ROWS;
    const int4* const meta = reinterpret_cast<const int4*>(TILES ? a.tile_meta : a.meta) +
                             (long long)g * (kPagedMeta / 4);
    const float* const ws_m = TILES ? a.tile_m : a.ws_m;
    const float* const ws_l = TILES ? a.tile_l : a.ws_l;
    const float* const ws_o = TILES ? a.tile_o : a.ws_o;
    const int4 item = meta[0];
    const int n_rows = meta[1].x, n = item.x;
    if (n == 0 || row0 >= n_rows) return;
    const int grp = threadIdx.x / LANES, lane = threadIdx.x % LANES, col = lane * 4;
    const int row = min(row0 + grp / GP, n_rows - 1);
    auto at = [&](int i) {  // part i
        const long long part = TILES ? (long long)g * a.splits + i : ((long long)g + i) * 2 + (i == 0);
        return part * block + row;
    };
    float M = -INFINITY, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = grp % GP; i0 < n; i0 += U * GP) {
        float m[U], l[U];
        f32x4 o[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {  // (past the end the last part's, unused)
            const long long p = at(min(i0 + u * GP, n - 1));
            m[u] = ws_m[p];
            l[u] = ws_l[p];
            o[u] = *reinterpret_cast<const f32x4*>(ws_o + p * D + col);
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < U; ++u) top = i0 + u * GP < n ? fmaxf(top, m[u]) : top;
        const float ref = top == -INFINITY ? 0.f : top;
        const float w0 = __builtin_amdgcn_exp2f(M - ref);
        L *= w0;
        acc *= w0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * GP >= n) break;
            const float w = __builtin_amdgcn_exp2f(m[u] - ref);
            L = fmaf(w, l[u], L);
            acc += w * o[u];
        }
        M = top;
    }
    if constexpr (GP > 1) {
        __shared__ f32x4 so[GROUPS][LANES];
        __shared__ float sm[GROUPS], sl[GROUPS];
        so[grp][lane] = acc;
        if (lane == 0) {
            sm[grp] = M;
            sl[grp] = L;
        }
        __syncthreads();
        if (grp % GP != 0) return;
#pragma unroll
        for (int q = 1; q < GP; ++q) M = fmaxf(M, sm[grp + q]);
        const float ref = M == -INFINITY ? 0.f : M;
        L = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < GP; ++q) {
            const float w = __builtin_amdgcn_exp2f(sm[grp + q] - ref);
            L = fmaf(w, sl[grp + q], L);
            acc += w * so[grp + q][lane];
        }
    }
    if (row0 + grp / GP >= n_rows) return;
    const int rr = item.w + row, tok = (uint32_t)rr / (uint32_t)a.group;
    store_row<D>(a, item.y + tok, item.z + rr - tok * a.group, col, acc, M, L);
}

// The first row_wgs workgroups add the row kernel's parts, row_per of them to an item, the others
// the tile kernel's.
template <int D>
__global__ __launch_bounds__(kNT) void paged_sum_kernel(const PagedArgs a, int row_wgs,
                                                        int row_per, int row_block) {
    if ((int)blockIdx.x < row_wgs)
        sum_rows<D, false>(a, blockIdx.x, row_block, row_per);
    else
        sum_rows<D, true>(a, blockIdx.x - row_wgs, kPagedTileRows,
                          kPagedTileRows / kSumRows<D, true>);
}

template <int D>
hipError_t launch_sums(const PagedArgs& a, int row_block, hipStream_t stream) {
    constexpr int kRows = kSumRows<D, false>;
    const int row_per = (a.few + kRows - 1) / kRows;
    const long long rows = a.meta ? (long long)a.n_wg * row_per : 0;
    const long long tiles =
        a.splits > 1 ? a.tile_wgs / a.splits * (kPagedTileRows / kSumRows<D, true>) : 0;
    if (rows + tiles == 0) return hipSuccess;
    hipLaunchKernelGGL(paged_sum_kernel<D>, dim3((unsigned)(rows + tiles)), dim3(kNT), 0, stream,
                       a, (int)rows, row_per, row_block);
    return hipGetLastError();
}

template <int D, int MT>
hipError_t launch_rows(const PagedArgs& a, int waves, hipStream_t stream) {
    if (waves == 8)
        hipLaunchKernelGGL((paged_rows_kernel<D, MT, 8>), dim3(a.n_wg), dim3(512), 0, stream, a);
    else
        hipLaunchKernelGGL((paged_rows_kernel<D, MT, 4>), dim3(a.n_wg), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_sums(const PagedArgs& a, int d, int row_block, hipStream_t stream) {
    return d == 64 ? launch_sums<64>(a, row_block, stream)
                   : launch_sums<128>(a, row_block, stream);
}

hipError_t launch_paged_rows(const PagedArgs& a, int d, int block, int waves, hipStream_t stream) {
    if (d == 64 && block == 16) return launch_rows<64, 1>(a, waves, stream);
    if (d == 64 && block == 32) return launch_rows<64, 2>(a, waves, stream);
    if (d == 128 && block == 16) return launch_rows<128, 1>(a, waves, stream);
    if (d == 128 && block == 32) return launch_rows<128, 2>(a, waves, stream);
    return hipErrorInvalidValue;
}

hipError_t launch_paged_tiles(const PagedArgs& a, int d, int form, hipStream_t stream) {
    if (d == 64) return launch_paged_tiles_d64(a, form, stream);
    if (d == 128) return launch_paged_tiles_d128(a, form, stream);
    return hipErrorInvalidValue;
}

}  // namespace attn
