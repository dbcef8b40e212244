// The paged cache's tables and stores.
//
// extend: with s_r tokens of request r in the cache and n_r new ones, pages of p rows,
//     kv_r = s_r + n_r,  cu_r = sum_{r' < r} n_r',  held_r = ceil(s_r / p),
//     need_r = ceil(kv_r / p) - held_r,  first_r = sum_{r' < r} need_r',
// new page i of request r (its page held_r + i) is free[n_free - 1 - first_r - i], and token t of
// request r (cu_r <= t < cu_r + n_r), at position s_r + t - cu_r, lies in row position % p of
// page position / p.  release is the inverse; pages that extend found missing, -1 in the table,
// do not come back: a list that held them would give them out again.
//
// Bound by launch and latency: a thousand requests are 8 KB.  So no workgroup waits for another:
// each sums the requests in front of its own tokens itself, a thousand at a time out of L2.  A
// page's first row is always a new token's, and that token's thread writes the table.  extend:
// one launch, 3.9 us for a token, 8.5 for 130k tokens of 1024 requests.
//
// release: where a page goes depends on the pages in front that are missing, which only the table
// tells.  A small table is counted by every workgroup, in one launch: in a graph 4.5 us for 64
// requests' drafts, 9.7 for 64k pages of 128.  A larger one would be read too often: its pages go
// where the lengths say, and a second launch looks whether any was missing, and only then goes
// through all of them again: 7 us for 256 requests, 10 for 922k pages of 1024, 1100 if some of
// those are missing.  (By lengths alone, one launch: 2.6 and 4.7.)
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

// Inclusive sums over the NT threads of the workgroup; *total: of all of them.  All threads call it.
template <int NT = kNT>
__device__ __forceinline__ long long block_scan(long long x, long long* total) {
    __shared__ long long waves[NT / 64];
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
    for (int w = 0; w < NT / 64; ++w) {
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

// The pages that a request gives back: its table's entries from kept on, `gone` of them.
struct Back {
    int kept, gone;
};
__device__ __forceinline__ Back back_of(const ReleaseArgs& a, int r) {
    const int kept = pages_of(max(a.keep_lens[r], 0), a.page_log2, a.max_pages);
    return {kept, max(pages_of(max(a.seq_lens[r], 0), a.page_log2, a.max_pages) - kept, 0)};
}

constexpr int kBackNT = 1024;
// Up to so many requests and entries in one launch.  128 requests of 512 entries, 1 to 500 pages of
// each given back: 6.0 to 9.7 us in a graph and 6.6 to 9.7 out of it, by two launches 7.2 and 10.2;
// 256 of 512, by two launches, 6.7 and 10.3.
constexpr int kSmallRequests = 256, kSmallTable = 1 << 16;

// A small table, one launch: a workgroup counts the pages that the requests in front give back in
// the table itself, 16 lanes to a request, and puts those of its own `per` requests behind them.
__global__ __launch_bounds__(kBackNT) void release_small_kernel(const ReleaseArgs a, int per) {
    const int tid = threadIdx.x;
    const int r0 = blockIdx.x * per, r1 = min(r0 + per, a.R);
    const int n_free = min(max(a.n_free[0], 0), a.n_list);
    int sum = 0;
    for (int r = tid / 16; r < r0; r += kBackNT / 16) {
        const Back x = back_of(a, r);
        const int* const from = a.table + r * a.table_stride + x.kept;
#pragma unroll 4
        for (int i = tid % 16; i < x.gone; i += 16) sum += from[i] >= 0;
    }
    long long first, all;
    block_scan<kBackNT>(sum, &first);
    first += n_free;
    for (int r = r0; r < r1; ++r) {
        const Back x = back_of(a, r);
        const int* const from = a.table + r * a.table_stride + x.kept;
        for (int i0 = 0; i0 < x.gone; i0 += kBackNT) {
            const int page = i0 + tid < x.gone ? from[i0 + tid] : -1;
            const long long upto = block_scan<kBackNT>(page >= 0, &all);
            if (page >= 0 && first + upto <= a.n_list) a.free_pages[first + upto - 1] = page;
            first += all;
        }
    }
    if (r1 == a.R && tid == 0) a.n_left[0] = (int)min(first, (long long)a.n_list);
}

// A workgroup returns the pages of `per` requests, behind those of the requests in front, as if
// none were missing.  Where one is, the first place of the workgroup's in the list says so: -1.
__global__ __launch_bounds__(kNT) void release_kernel(const ReleaseArgs a, int per) {
    const int tid = threadIdx.x;
    const int r0 = blockIdx.x * per, r1 = min(r0 + per, a.R);
    const int n_free = min(max(a.n_free[0], 0), a.n_list);
    long long sum = 0, first;
    for (int r = tid; r < r0; r += kNT) sum += back_of(a, r).gone;
    block_scan(sum, &first);
    const long long at = n_free + first;
    int missing = 0;
    for (int r = r0; r < r1; ++r) {
        const Back x = back_of(a, r);
        const int* const from = a.table + (long long)r * a.table_stride + x.kept;
        for (int i = tid; i < x.gone; i += kNT) {
            const long long to = n_free + first + i;
            const int entry = from[i];
            missing |= entry < 0;
            if (to < a.n_list) a.free_pages[to] = entry;
        }
        first += x.gone;
    }
    missing = __syncthreads_or(missing);
    if (missing && tid == 0 && at < a.n_list) a.free_pages[at] = -1;
}

// One workgroup, behind release_kernel: n_left, and where pages are missing or the list is too
// short the whole list once more, without those that are not there.
constexpr int kWalkU = 4;  // pages to a thread and step
static_assert(kWalkU * kBackNT == 64 * 64, "a wave sums the counts of a step's 64 waves");
__global__ __launch_bounds__(kBackNT) void release_end_kernel(const ReleaseArgs a) {
    __shared__ long long s_first[kBackNT];
    __shared__ int s_kept[kBackNT], s_count[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n_free = min(max(a.n_free[0], 0), a.n_list);
    long long pages = 0;
    int missing = 0;
    for (int r0 = 0; r0 < a.R; r0 += kBackNT * kPer) {
        int n[kPer];
        long long sum = 0, all;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            n[i] = r < a.R ? back_of(a, r).gone : 0;
            sum += n[i];
        }
        long long at = n_free + pages + block_scan<kBackNT>(sum, &all) - sum;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            // (a workgroup's first place is that of one of its requests)
            if (n[i] > 0 && at < a.n_list) missing |= a.free_pages[at] < 0;
            at += n[i];
        }
        pages += all;
    }
    if (!__syncthreads_or(missing || n_free + pages > a.n_list)) {
        if (tid == 0) a.n_left[0] = (int)(n_free + pages);
        return;
    }
    long long to = n_free;  // the next place in the list
    for (int r0 = 0; r0 < a.R; r0 += kBackNT) {
        Back x = {0, 0};
        if (r0 + tid < a.R) x = back_of(a, r0 + tid);
        long long all;
        const long long upto = block_scan<kBackNT>(x.gone, &all);
        s_first[tid] = upto - x.gone;
        s_kept[tid] = x.kept;
        __syncthreads();
        for (long long p0 = 0; p0 < all; p0 += kWalkU * kBackNT) {
            int entry[kWalkU];
            unsigned long long there[kWalkU];
#pragma unroll
            for (int u = 0; u < kWalkU; ++u) {
                const long long p = p0 + u * kBackNT + tid;
                entry[u] = -1;
                if (p < all) {
                    int lo = 0, hi = kBackNT - 1;  // the last request whose first page is not past p
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) >> 1;
                        if (s_first[mid] <= p)
                            lo = mid;
                        else
                            hi = mid - 1;
                    }
                    entry[u] = a.table[(long long)(r0 + lo) * a.table_stride + s_kept[lo] +
                                       (p - s_first[lo])];
                }
                there[u] = __ballot(entry[u] >= 0);
                if (lane == 0) s_count[u * (kBackNT / 64) + wave] = __popcll(there[u]);
            }
            __syncthreads();
            const int mine = s_count[lane];
            int sum = mine;
#pragma unroll
            for (int off = 1; off < 64; off *= 2) {
                const int y = __shfl_up(sum, off);
                if (lane >= off) sum += y;
            }
#pragma unroll
            for (int u = 0; u < kWalkU; ++u) {
                const int before = __shfl(sum - mine, u * (kBackNT / 64) + wave);
                const long long at = to + before + __popcll(there[u] & ((1ULL << lane) - 1));
                if (entry[u] >= 0 && at < a.n_list) a.free_pages[at] = entry[u];
            }
            to += __shfl(sum, 63);
            __syncthreads();  // the counts are written again
        }
    }
    if (tid == 0) a.n_left[0] = (int)min(to, (long long)a.n_list);
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
    if (a.R <= kSmallRequests && (long long)a.R * a.max_pages <= kSmallTable) {
        const int per = (a.R + 63) / 64;
        hipLaunchKernelGGL(release_small_kernel, dim3((a.R + per - 1) / per), dim3(kBackNT), 0,
                           stream, a, per);
        return hipGetLastError();
    }
    const int per = (a.R + 511) / 512;
    hipLaunchKernelGGL(release_kernel, dim3((a.R + per - 1) / per), dim3(kNT), 0, stream, a, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(release_end_kernel, dim3(1), dim3(kBackNT), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_paged_store(const StoreArgs& a, int d, hipStream_t stream) {
    if (d == 64) return launch_store<64>(a, stream);
    if (d == 128) return launch_store<128>(a, stream);
    return hipErrorInvalidValue;
}

}  // namespace attn
