// Attention of requests with few new tokens over a paged cache.
//
// For request r, new token i (position pos = kv - n + i) and query head h, over the keys j that
// the token sees (j <= pos under a causal mask, j > pos - window with a window):
//     x_j = scale q.k_j,  capped: cap tanh(x_j / cap),  with slopes: x_j - slope_h |pos - j|,
//     o = sum_j exp(x_j) v_j / sum_j exp(x_j),  lse = log sum_j exp(x_j),
// o = 0 and lse = -inf where a token sees no key.
//
// The new tokens of all query heads that share a key/value head are the rows of one product, in
// blocks of 16 MT, token by token (row = token * group + head of the group), so that each key is
// read once for all of them.  Products on v_mfma_f32_16x16x32_bf16: S^T = K Q^T with K's rows
// straight from memory as operand A, O^T += V^T P^T with V through a wave's own LDS tile, read
// transposed.  A step is 128 keys, 32 to a wave; keys are permuted inside 32 so that the scores
// that a lane gets are the operand that its P^T has to be.  A lane's K and V rows lie in one
// aligned run of eight keys, hence in one page: one page number serves all its loads of a step,
// and is read a step ahead.
//
// Bound: HBM, 4 D bytes a key.  All items (request, key/value head, block of rows) one behind
// another are one line of steps, which the workgroups share out evenly whatever the requests'
// lengths are; no length is known to the host.  Each workgroup finds its part by summing the
// lengths itself (one launch less than a plan of its own).  An item that lies in several
// workgroups leaves partial sums (unnormalised, with their maximum), which a second kernel adds in
// order: no atomics, the same bits every call.  A workgroup has two of them at most, one for an
// item that began before it and one for an item that goes on behind it.
//
// Only keys in [lo, kv) are read, lo being the first that any of the request's tokens sees; rows
// of a tile outside it are copies of its first or last key with weight 0.  A page number outside
// the cache is replaced by 0 and makes the request's results NaN.
#include <hip/hip_runtime.h>
#include <stdint.h>

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

constexpr int kNT = 256, kNW = 4;
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

// Items of a request and steps of each, for blocks of `block` rows.
struct Share {
    int items, blocks, steps;
};
__device__ __forceinline__ Share share_of(const PagedArgs& a, const PagedRequest& x, int block) {
    Share s = {0, 0, 0};
    const long long rows = (long long)x.qn * a.group;
    if (rows == 0 || rows > a.few) return s;
    s.blocks = (int)((rows + block - 1) / block);
    s.items = s.blocks * a.Hkv;
    s.steps = x.kv > x.lo ? (x.kv + kPagedRowKeys - 1) / kPagedRowKeys - x.lo / kPagedRowKeys : 1;
    return s;
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

template <int D, int MT>
__global__ __launch_bounds__(kNT) void paged_rows_kernel(const PagedArgs a) {
    constexpr int KS = D / 32;       // MFMA steps over a row
    constexpr int DB = D / 16;       // 16-column blocks of O^T
    constexpr int VST = D + 32;      // bf16 to a row of V in LDS
    constexpr int OST = D + 4;       // floats to a row where the waves meet
    constexpr int BLOCK = 16 * MT;
    __shared__ __attribute__((aligned(16))) uint16_t vtile[kNW][32 * VST];
    __shared__ float sm[kNW][BLOCK], sl[kNW][BLOCK];
    __shared__ long long found[2];  // request, steps before it
    static_assert(kNW * 16 * OST * 4 <= (int)sizeof(vtile), "");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    int* const meta = a.meta + (long long)blockIdx.x * kPagedMeta;

    // ---- this workgroup's part of the line of all steps ------------------------
    long long mine = 0;  // up to kNT requests: this thread's
    long long sum = 0;
    for (int r = tid; r < a.R; r += kNT) {
        const Share s = share_of(a, paged_request(a, r), BLOCK);
        mine = (long long)s.items * s.steps;
        sum += mine;
    }
    long long total;
    long long upto = block_scan<kNT>(sum, &total);
    const int n_wg = (int)min((long long)a.n_wg, total);
    if (tid == 0) meta[0] = 0;
    if ((int)blockIdx.x >= n_wg) return;
    const long long u0 = total * blockIdx.x / n_wg, u1 = total * (blockIdx.x + 1) / n_wg;
    long long before = 0;
    for (int r0 = 0; r0 < a.R; r0 += kNT) {
        long long all = total;
        if (a.R > kNT) {
            const int r = r0 + tid;
            mine = 0;
            if (r < a.R) {
                const Share s = share_of(a, paged_request(a, r), BLOCK);
                mine = (long long)s.items * s.steps;
            }
            upto = block_scan<kNT>(mine, &all);
        }
        if (u0 < before + all) {
            const long long first = before + upto - mine;
            if (u0 >= first && u0 < first + mine) {
                found[0] = r0 + tid;
                found[1] = first;
            }
            break;
        }
        before += all;
    }
    __syncthreads();
    int r = __builtin_amdgcn_readfirstlane((int)found[0]);
    long long r_first = found[1];  // of the line, where request r begins

    const int rk = 8 * (l16 >> 2) + (l16 & 3);  // this lane's keys of a step: rk, rk + 4
    const int page_mask = (1 << a.page_log2) - 1;
    uint16_t* const vt = vtile[wave];
    for (long long u = u0; u < u1;) {
        const PagedRequest x = paged_request(a, r);
        const Share share = share_of(a, x, BLOCK);
        const long long mine_here = (long long)share.items * share.steps;
        if (u >= r_first + mine_here) {  // the next request that has any
            r_first += mine_here;
            for (++r;; r += 64) {
                const int rr = min(r + lane, a.R - 1);
                const Share s = share_of(a, paged_request(a, rr), BLOCK);
                const unsigned long long any = __ballot(s.items > 0 && r + lane < a.R);
                if (any) {
                    r += __ffsll((long long)any) - 1;
                    break;
                }
                if (r + 64 >= a.R) return;  // (never: u1 <= total)
            }
            r = __builtin_amdgcn_readfirstlane(r);
            continue;
        }
        const int item = (int)((u - r_first) / share.steps);
        const int t0 = (int)(u - r_first - (long long)item * share.steps);
        const int t1 = (int)min((long long)share.steps, t0 + (u1 - u));
        const long long item_first = u - t0;  // of the line
        u += t1 - t0;
        const int head = item / share.blocks, blk = item - head * share.blocks;
        const int n_rows = min(x.qn * a.group - blk * BLOCK, BLOCK);

        // ---- this lane's queries: Q^T, dims 32 s + 8 g4 .. + 7 of row l16 -----------
        bf16x8 qf[MT][KS];
        int hi[MT], lo[MT], pos[MT];
        float slope[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int row = blk * BLOCK + min(mt * 16 + l16, n_rows - 1);
            const int tok = row / a.group, h = head * a.group + row - tok * a.group;
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
        const int tok_last = (blk * BLOCK + n_rows - 1) / a.group;
        const int all_hi = a.causal ? x.pos0 + blk * BLOCK / a.group : x.kv - 1;
        const int all_lo = a.window ? x.pos0 + tok_last - a.window + 1 : 0;
        const uint16_t* const kp = a.k.ptr + head * a.k.head + 8 * g4;
        const uint16_t* const vp = a.v.ptr + head * a.v.head + 8 * g4;
        const int* const table = a.table + (long long)r * a.table_stride;

        float m[MT], l[MT];
        f32x4 oacc[MT][DB];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt] = -INFINITY;
            l[mt] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) oacc[mt][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        bool bad = x.bad;
        const int key0 = x.lo / kPagedRowKeys * kPagedRowKeys + 32 * wave;
        auto key_of = [&](int kb, int i) { return max(min(kb + i, x.kv - 1), x.lo); };
        int entry = 0;
        if (x.kv > x.lo) entry = table[key_of(key0 + t0 * kPagedRowKeys, rk) >> a.page_log2];
        for (int t = t0; t < t1; ++t) {
            const int kb = key0 + t * kPagedRowKeys;
            int next = 0;
            if (t + 1 < t1) next = table[key_of(kb + kPagedRowKeys, rk) >> a.page_log2];
            if (kb < x.kv && kb + 32 > x.lo) {
                const bool out = (uint32_t)entry >= (uint32_t)a.n_pages;
                bad |= out;
                const long long page = out ? 0 : entry;
                u32x4 kr[2][KS], vr[2][KS];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int s0 = key_of(kb, rk + 4 * b) & page_mask;
                    const uint16_t* const kk = kp + page * a.k.page + s0 * a.k.row;
                    const uint16_t* const vv = vp + page * a.v.page + s0 * a.v.row;
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        kr[b][s] = __builtin_nontemporal_load(
                            reinterpret_cast<const u32x4*>(kk + 32 * s));
                        vr[b][s] = __builtin_nontemporal_load(
                            reinterpret_cast<const u32x4*>(vv + 32 * s));
                    }
                }
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        *reinterpret_cast<u32x4*>(vt + (rk + 4 * b) * VST + 32 * s + 8 * g4) =
                            vr[b][s];
                bf16x8 pf[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    // lane (row l16, g4) gets keys kb + 8 g4 + e, e = 0..7
                    f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        sa = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, kr[0][s]), qf[mt][s], sa, 0, 0, 0);
                        sb = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, kr[1][s]), qf[mt][s], sb, 0, 0, 0);
                    }
                    float sc[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sc[i] = sa[i];
                        sc[4 + i] = sb[i];
                    }
                    // log2 units; tanh y = 1 - 2 / (1 + e^2y)
                    if (a.cap_out != 0.f) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float w = __builtin_amdgcn_exp2f(sc[e] * a.cap_in);
                            sc[e] = fmaf(-2.f * a.cap_out, __builtin_amdgcn_rcpf(1.f + w),
                                         a.cap_out);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) sc[e] *= a.scale_log2;
                    }
                    const int kl = kb + 8 * g4;
                    if (a.slopes) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            sc[e] = fmaf(-slope[mt], (float)abs(pos[mt] - (kl + e)), sc[e]);
                    }
                    if (kb + 31 > all_hi || kb < all_lo) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (kl + e > hi[mt] || kl + e < lo[mt]) sc[e] = -INFINITY;
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
                    // P is rounded to bf16 (2^-9 of each weight) as the operand it has to be; its
                    // sum takes the weights as they are, so that the log-sum-exp is fp32's
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float p = __builtin_amdgcn_exp2f(sc[e] - ref);
                        l[mt] += p;
                        pf[mt][e] = (__bf16)p;
                    }
                }
                // O^T += V^T P^T: lane (i, g) of a 16-lane group reads row 8 g + i / 4 (and
                // + 4) at column 16 db + 4 (i % 4) and receives column 16 db + i of keys
                // 8 g .. 8 g + 3 (and 8 g + 4 .. 8 g + 7)
                const uint16_t* const vs = vt + (8 * g4 + (l16 >> 2)) * VST + 4 * (l16 & 3);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const s16x4 w0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(vs + 16 * db));
                    const s16x4 w1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(vs + 4 * VST + 16 * db));
                    const s16x8 w = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        oacc[mt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, w), pf[mt], oacc[mt][db], 0, 0, 0);
                }
            }
            entry = next;
        }

        // ---- the waves meet, 16 rows at a time -----------------------------------
        bad = __syncthreads_or(bad);
        const bool whole = t0 == 0 && t1 == share.steps;
        const int part = t0 == 0 ? 1 : 0;
        if (!whole && tid == 0 && t0 == 0) {  // the first part of an item: its others follow
            const int last =
                (int)(((item_first + share.steps) * n_wg - 1) / total);  // who has its last step
            meta[1] = x.q0;
            meta[2] = head * a.group;
            meta[3] = blk * BLOCK;
            meta[4] = n_rows;
            meta[0] = last - (int)blockIdx.x + 1;
        }
        float* const so = reinterpret_cast<float*>(&vtile[0][0]);  // [wave][16][OST]
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt > 0) __syncthreads();
            const float lsum = rows4_sum(l[mt]);  // the lane groups have different keys
            if (g4 == 0) {
                sm[wave][mt * 16 + l16] = m[mt];
                sl[wave][mt * 16 + l16] = bad ? NAN : lsum;
            }
#pragma unroll
            for (int db = 0; db < DB; ++db)
                *reinterpret_cast<f32x4*>(so + (wave * 16 + l16) * OST + 16 * db + 4 * g4) =
                    oacc[mt][db];
            __syncthreads();
            for (int i = tid; i < 16 * D / 4; i += kNT) {
                const int row = mt * 16 + i / (D / 4), col = i % (D / 4) * 4;
                if (row >= n_rows) break;
                float M = sm[0][row];
#pragma unroll
                for (int w = 1; w < kNW; ++w) M = fmaxf(M, sm[w][row]);
                const float ref = M == -INFINITY ? 0.f : M;
                float L = 0.f;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kNW; ++w) {
                    const float wt = __builtin_amdgcn_exp2f(sm[w][row] - ref);
                    L = fmaf(wt, sl[w][row], L);
                    acc += wt * *reinterpret_cast<const f32x4*>(so + (w * 16 + row - mt * 16) * OST +
                                                                col);
                }
                if (whole) {
                    const int rr = blk * BLOCK + row, tok = rr / a.group;
                    store_row<D>(a, x.q0 + tok, head * a.group + rr - tok * a.group, col, acc, M,
                                 L);
                } else {
                    const long long at = ((long long)blockIdx.x * 2 + part) * BLOCK + row;
                    *reinterpret_cast<f32x4*>(a.ws_o + at * D + col) = acc;
                    if (col == 0) {
                        a.ws_m[at] = M;
                        a.ws_l[at] = L;
                    }
                }
            }
        }
        __syncthreads();  // the tiles are V's again
    }
}

// Adds parts of rows: workgroup (g, y) those of rows y * ROWS .. of the item g.  After the row
// kernel (TILES false) item g is the one that begins in its workgroup g and does not end there:
// its first part is that workgroup's second one, the others are the following workgroups' first.
// After the tile kernel item g is a block of a head, its splits one behind another.
template <int D, bool TILES>
__global__ __launch_bounds__(kNT) void paged_sum_kernel(const PagedArgs a, int block) {
    constexpr int LANES = D / 4, ROWS = kNT / LANES;
    const int* const meta = (TILES ? a.tile_meta : a.meta) + (long long)blockIdx.x * kPagedMeta;
    const float* const ws_m = TILES ? a.tile_m : a.ws_m;
    const float* const ws_l = TILES ? a.tile_l : a.ws_l;
    const float* const ws_o = TILES ? a.tile_o : a.ws_o;
    const int n = meta[0];
    const int row = blockIdx.y * ROWS + threadIdx.x / LANES, col = threadIdx.x % LANES * 4;
    if (n == 0 || row >= meta[4]) return;
    auto at = [&](int i) {  // part i
        const long long part = TILES ? (long long)blockIdx.x * a.splits + i
                                     : ((long long)blockIdx.x + i) * 2 + (i == 0);
        return part * block + row;
    };
    float M = -INFINITY;
    for (int i = 0; i < n; ++i) M = fmaxf(M, ws_m[at(i)]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) {
        const float w = __builtin_amdgcn_exp2f(ws_m[at(i)] - ref);
        L = fmaf(w, ws_l[at(i)], L);
        acc += w * *reinterpret_cast<const f32x4*>(ws_o + at(i) * D + col);
    }
    const int rr = meta[3] + row, tok = rr / a.group;
    store_row<D>(a, meta[1] + tok, meta[2] + rr - tok * a.group, col, acc, M, L);
}

template <int D, bool TILES>
hipError_t launch_sum(const PagedArgs& a, int items, int block, hipStream_t stream) {
    constexpr int rows = kNT / (D / 4);
    hipLaunchKernelGGL((paged_sum_kernel<D, TILES>), dim3(items, (block + rows - 1) / rows),
                       dim3(kNT), 0, stream, a, block);
    return hipGetLastError();
}

template <int D, int MT>
hipError_t launch_rows(const PagedArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((paged_rows_kernel<D, MT>), dim3(a.n_wg), dim3(kNT), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_sum<D, false>(a, a.n_wg, 16 * MT, stream);
}

}  // namespace

hipError_t launch_paged_rows(const PagedArgs& a, int d, int block, hipStream_t stream) {
    if (d == 64 && block == 16) return launch_rows<64, 1>(a, stream);
    if (d == 64 && block == 32) return launch_rows<64, 2>(a, stream);
    if (d == 128 && block == 16) return launch_rows<128, 1>(a, stream);
    if (d == 128 && block == 32) return launch_rows<128, 2>(a, stream);
    return hipErrorInvalidValue;
}

hipError_t launch_paged_tiles(const PagedArgs& a, int d, int waves, int form, hipStream_t stream) {
    hipError_t e = hipErrorInvalidValue;
    if (d == 64 && waves == 4) e = launch_paged_tiles_d64_w4(a, form, stream);
    if (d == 64 && waves == 8) e = launch_paged_tiles_d64_w8(a, form, stream);
    if (d == 128 && waves == 4) e = launch_paged_tiles_d128_w4(a, form, stream);
    if (d == 128 && waves == 8) e = launch_paged_tiles_d128_w8(a, form, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    const int items = (int)(a.tile_wgs / a.splits);
    return d == 64 ? launch_sum<64, true>(a, items, 32 * waves, stream)
                   : launch_sum<128, true>(a, items, 32 * waves, stream);
}

}  // namespace attn
