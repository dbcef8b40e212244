// The paged cache's tables and stores.
//
// extend: with s_r tokens of request r in the cache and n_r new ones, pages of p rows,
//     kv_r = s_r + n_r,  cu_r = sum_{r' < r} n_r',  held_r = ceil(s_r / p),
//     need_r = ceil(kv_r / p) - held_r,  first_r = sum_{r' < r} need_r',
// new page i of request r (its page held_r + i) is free[n_free - 1 - first_r - i], and token t of
// request r (cu_r <= t < cu_r + n_r), at position s_r + t - cu_r, lies in row position % p of
// page position / p.  release is the inverse.
//
// Bound by launch and latency: a thousand requests are 8 KB.  So there is one launch, and no
// workgroup waits for another: each sums the requests in front of its own tokens itself, a
// thousand at a time out of L2.  A page's first row is always a new token's, and that token's
// thread writes the table.  extend: 3.9 us for a token, 8.5 for 130k tokens of 1024 requests;
// release: 2.7 us for 64 requests' drafts, 6 for a million pages of 1024.
//
// store: each row of k and v goes to its slot.  Bound: HBM, 16 bytes to a lane, four rows of each
// on their way: 16384 tokens of 8 heads of 128, 134 MB in and out, 26 us or 5.1 TB/s, a large
// copy's rate.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "paged.h"

namespace attn {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kNT = 256;
constexpr int kPer = 4;               // requests to a thread
constexpr int kChunk = kNT * kPer;    // requests summed at a time
constexpr int kTokens = 1024;         // tokens to a workgroup

// Inclusive sums over the workgroup's threads; *total: of all of them.  All threads call it.
__device__ __forceinline__ long long block_scan(long long x, long long* total) {
    __shared__ long long waves[kNT / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const long long y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();  // the last call's reads
    if (lane == 63) waves[wave] = x;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kNT / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return x + before;
}

__device__ __forceinline__ int pages_of(long long tokens, int log2, int most) {
    return (int)min((tokens + (1LL << log2) - 1) >> log2, (long long)most);
}

__global__ __launch_bounds__(kNT) void extend_kernel(const ExtendArgs a) {
    // of the requests at hand: first token, first new page, tokens held, pages held
    __shared__ long long s_cu[kChunk + 1];
    __shared__ long long s_first[kChunk];
    __shared__ int s_seq[kChunk], s_held[kChunk];
    const int tid = threadIdx.x;
    const long long t0 = (long long)blockIdx.x * kTokens, t1 = min(t0 + kTokens, (long long)a.T);
    const bool last = blockIdx.x == gridDim.x - 1;  // writes what is not the tokens'
    const int n_free = min(max(a.n_free[0], 0), a.n_list);
    long long tokens = 0, pages = 0;  // before the requests at hand
    for (int r0 = 0; r0 < a.R && (last || tokens < t1); r0 += kChunk) {
        int seq[kPer], n[kPer], held[kPer], need[kPer];
        long long n_sum = 0, need_sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            seq[i] = r < a.R ? max(a.seq_lens[r], 0) : 0;
            n[i] = r < a.R ? max(a.new_lens[r], 0) : 0;
            held[i] = pages_of(seq[i], a.page_log2, a.max_pages);
            need[i] = pages_of((long long)seq[i] + n[i], a.page_log2, a.max_pages) - held[i];
            n_sum += n[i];
            need_sum += need[i];
        }
        long long n_all, need_all;
        long long cu = tokens + block_scan(n_sum, &n_all) - n_sum;
        long long first = pages + block_scan(need_sum, &need_all) - need_sum;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = tid * kPer + i, r = r0 + j;
            s_cu[j] = cu;
            s_first[j] = first;
            s_seq[j] = seq[i];
            s_held[j] = held[i];
            cu += n[i];
            first += need[i];
            if (last && r < a.R) {
                a.cu[r + 1] = (int)min(cu, (long long)INT_MAX);
                a.kv_lens[r] = (int)min((long long)seq[i] + n[i], (long long)INT_MAX);
            }
        }
        if (tid == kNT - 1) s_cu[kChunk] = cu;
        __syncthreads();
        const long long from = max(t0, tokens), to = min(t1, tokens + n_all);
        for (long long t = from + tid; t < to; t += kNT) {
            int lo = 0, hi = kChunk - 1;  // the last request whose first token is not past t
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_cu[mid] <= t)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            const long long pos = s_seq[lo] + (t - s_cu[lo]);
            const long long page = pos >> a.page_log2;
            long long entry = -1;
            if (page < a.max_pages) {
                int* const at = a.table + (long long)(r0 + lo) * a.table_stride + page;
                if (page < s_held[lo]) {
                    entry = *at;
                } else {
                    const long long i = s_first[lo] + page - s_held[lo];
                    if (i < n_free) entry = a.free_pages[n_free - 1 - i];
                    if ((pos & ((1 << a.page_log2) - 1)) == 0) *at = (int)entry;
                }
            }
            const long long slot = (entry << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
            a.slots[t] = entry < 0 || slot > INT_MAX ? -1 : (int)slot;
            a.positions[t] = (int)min(pos, (long long)INT_MAX);
        }
        tokens += n_all;
        pages += need_all;
        __syncthreads();  // the arrays are written again
    }
    for (long long t = max(t0, tokens) + tid; t < t1; t += kNT) {  // no request's
        a.slots[t] = -1;
        a.positions[t] = 0;
    }
    if (last && tid == 0) {
        a.cu[0] = 0;
        a.n_left[0] = (int)max((long long)n_free - pages, (long long)INT_MIN);
    }
}

// A workgroup returns the pages of `per` requests, behind those of the requests in front.
__global__ __launch_bounds__(kNT) void release_kernel(const ReleaseArgs a, int per) {
    const int tid = threadIdx.x;
    const int r0 = blockIdx.x * per, r1 = min(r0 + per, a.R);
    const int n_free = min(max(a.n_free[0], 0), a.n_list);
    auto kept = [&](int r) { return pages_of(max(a.keep_lens[r], 0), a.page_log2, a.max_pages); };
    auto gone = [&](int r) {
        return max(pages_of(max(a.seq_lens[r], 0), a.page_log2, a.max_pages) - kept(r), 0);
    };
    long long sum = 0, first;
    for (int r = tid; r < r0; r += kNT) sum += gone(r);
    block_scan(sum, &first);
    for (int r = r0; r < r1; ++r) {
        const int k = kept(r), n = gone(r);
        const int* const from = a.table + (long long)r * a.table_stride + k;
        for (int i = tid; i < n; i += kNT) {
            const long long to = n_free + first + i;
            if (to < a.n_list) a.free_pages[to] = from[i];
        }
        first += n;
    }
    if (r1 == a.R && tid == 0) a.n_left[0] = (int)min(n_free + first, (long long)a.n_list);
}

template <int D>
__global__ __launch_bounds__(kNT) void store_kernel(const StoreArgs a) {
    constexpr int LANES = D / 8;         // to a row
    constexpr int ROWS = kNT / LANES;    // to a step
    constexpr int U = 4;
    const int lane = threadIdx.x % LANES;
    const long long rows = (long long)a.T * a.Hkv;
    const long long row0 = (long long)blockIdx.x * (ROWS * U) + threadIdx.x / LANES;
    u32x4 x[U][2];
    int slot[U], head[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long row = min(row0 + u * ROWS, rows - 1);
        const uint32_t t = (uint32_t)row / (uint32_t)a.Hkv;
        head[u] = (int)((uint32_t)row - t * (uint32_t)a.Hkv);
        slot[u] = row0 + u * ROWS < rows ? a.slots[t] : -1;
        const uint16_t* const k = static_cast<const uint16_t*>(a.k.ptr);
        const uint16_t* const v = static_cast<const uint16_t*>(a.v.ptr);
        x[u][0] = *reinterpret_cast<const u32x4*>(k + t * a.k.row_stride +
                                                  head[u] * a.k.head_stride + lane * 8);
        x[u][1] = *reinterpret_cast<const u32x4*>(v + t * a.v.row_stride +
                                                  head[u] * a.v.head_stride + lane * 8);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int page = slot[u] >> a.page_log2, s = slot[u] & ((1 << a.page_log2) - 1);
        if (slot[u] < 0 || page >= a.n_pages) continue;
        auto to = [&](const attn_heads& p) {
            return reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.ptr) +
                                            page * p.batch_stride + s * p.row_stride +
                                            head[u] * p.head_stride + lane * 8);
        };
        *to(a.k_pages) = x[u][0];
        *to(a.v_pages) = x[u][1];
    }
}

template <int D>
hipError_t launch_store(const StoreArgs& a, hipStream_t stream) {
    constexpr int rows = kNT / (D / 8) * 4;
    const long long wgs = ((long long)a.T * a.Hkv + rows - 1) / rows;
    if (wgs > kMaxWorkgroups) return hipErrorInvalidValue;
    hipLaunchKernelGGL(store_kernel<D>, dim3((unsigned)wgs), dim3(kNT), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_extend(const ExtendArgs& a, hipStream_t stream) {
    const int wgs = (a.T + kTokens - 1) / kTokens;
    hipLaunchKernelGGL(extend_kernel, dim3(wgs), dim3(kNT), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged_release(const ReleaseArgs& a, hipStream_t stream) {
    const int per = (a.R + 511) / 512;
    hipLaunchKernelGGL(release_kernel, dim3((a.R + per - 1) / per), dim3(kNT), 0, stream, a, per);
    return hipGetLastError();
}

hipError_t launch_paged_store(const StoreArgs& a, int d, hipStream_t stream) {
    if (d == 64) return launch_store<64>(a, stream);
    if (d == 128) return launch_store<128>(a, stream);
    return hipErrorInvalidValue;
}

}  // namespace attn
