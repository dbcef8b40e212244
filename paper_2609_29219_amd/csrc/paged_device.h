// Device code that the paged attention kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"
#include "paged_plan.h"

namespace attn {

// Rows of a block, `first` being the first one's number in the request: which token, and which
// head of the group (row = token * group + head).  Inside a block by a product with the inverse,
// 2^32 / group rounded up, which is exact as long as the dividend times the group is under 2^32.
struct GroupDiv {
    int token0, rest, group;
    uint32_t inverse;
    __device__ __forceinline__ GroupDiv(const PagedArgs& a, int first) {
        group = a.group;
        inverse = a.group_inverse;
        token0 = (uint32_t)first / (uint32_t)group;
        rest = first - token0 * group;
    }
    __device__ __forceinline__ int token(int i, int* head) const {
        const int x = rest + i;
        const int t = group == 1 ? x : (int)__umulhi((uint32_t)x, inverse);
        *head = x - t * group;
        return token0 + t;
    }
};

// cap tanh y of u = 2 y log2(e): cap (w - 1) / (w + 1), w = e^2y.  The difference is exact where w
// is near 1, so that what is off is w's last bit, cap 2^-24.  (Past 2^30 it is cap.)  A capped
// prompt of 4096 tokens, 16 query heads to 4, takes 155 us; by cap - 2 cap / (1 + w), which is off
// by about three times as much, 143.
__device__ __forceinline__ float capped(float u, float cap) {
    const float w = __builtin_amdgcn_exp2f(fminf(u, 30.f));
    return fmaf(w, cap, -cap) * __builtin_amdgcn_rcpf(1.f + w);
}

// Inclusive sum over a wave, by moves between lanes inside rows of 16, then of the rows' sums.
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15, into 1, 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31, into 2, 3
    return x;
}

// Inclusive sum over the NT threads of the workgroup; *total: of all.  All threads call it.
template <int NT>
__device__ __forceinline__ int block_scan(int x, int* total) {
    constexpr int NW = NT / 64;
    __shared__ int waves[NW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = wave_scan(x);
    __syncthreads();  // the last call's reads
    if (lane == 63) waves[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return x + before;
}

// The request (r, or -1) that has the nth of something of which request y has count(y), and how
// many there are before it.  found: shared memory.  All threads call it; up to 64 requests each
// wave finds it by itself.
struct PagedFound {
    int r, first;
    PagedRequest x;
};
template <int NT, typename F>
__device__ __forceinline__ PagedFound paged_find(const PagedArgs& a, int nth, int* found,
                                                 F&& count) {
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    if (a.R <= 64) {
        const int lane = threadIdx.x & 63;
        PagedRequest y = {0, 0, 0, 0, 0, 0};
        int mine = 0;
        if (lane < a.R) {
            y = paged_request(a, lane);
            mine = count(y);
        }
        const int upto = wave_scan(mine);
        const unsigned long long here = __ballot(nth >= upto - mine && nth < upto);
        const int r = here ? __ffsll((long long)here) - 1 : 0;
        auto from = [&](int v) { return __builtin_amdgcn_readlane(v, r); };
        return {here ? r : -1,
                from(upto - mine),
                {from(y.q0), from(y.qn), from(y.pos0), from(y.kv), from(y.lo), from(y.bad)}};
    }
    int before = 0;
    for (int r0 = 0; r0 < a.R; r0 += NT) {
        const int r = r0 + threadIdx.x;
        const int mine = r < a.R ? count(paged_request(a, r)) : 0;
        int all;
        const int at = before + block_scan<NT>(mine, &all) - mine;
        // (bounds that overlap: up to 2^31 blocks of these requests, behind fewer than 2^31)
        if ((uint32_t)nth < (uint32_t)before + (uint32_t)all) {
            if (nth >= at && nth < at + mine) {
                found[0] = r;
                found[1] = at;
            }
            __syncthreads();
            const int here = uniform(found[0]);
            return {here, uniform(found[1]), paged_request(a, here)};
        }
        before += all;
    }
    return {-1, 0, {0, 0, 0, 0, 0, 0}};
}

}  // namespace attn
