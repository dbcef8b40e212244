// Per-head RMS norm of queries and keys with the position rotation, forward and
// backward, moving token-major projections [B][S][H][d] (any strides) to and from the
// head-major tensors [B][H][S][d] that attention reads; values are moved along.
//
// Forward, for a row x of d values at position p:
//     r = 1 / sqrt(mean(x^2) + eps),  y = w x r,
//     (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = p inv_freq[i],
// for each of the rot / 2 pairs of y: (i, i + rot/2), or (2i, 2i + 1) interleaved.
// Backward, for the gradient g of the rotated row: g' = g turned by -t, then
//     dw = sum over rows of g' x r,   dx = r (g' w - x r mean(g' w x r)).
//
// Bound: HBM.  A row is read and written once, 16 bytes to a lane; everything else is a
// fraction of that time.  A workgroup takes a tile of tokens and walks all rows of
// some heads of it, so the angles of a token are evaluated once for all of its heads
// (into LDS, as cos and sin): in double precision up to the fraction of a turn, since a
// float product is off by 0.01 rad at position 2^17.  Lane order: the tokens of one head
// are neighbours, so the head-major side is contiguous over the whole tile.
// All arithmetic is fp32 with one rounding at the end.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "common.h"

namespace attn {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kRopeThreads = 256;

__device__ __forceinline__ void widen8(u32x4 u, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(u[e] << 16);
        x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
}

__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    widen8(*reinterpret_cast<const u32x4*>(p), x);
}

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = a[e];
        x[4 + e] = b[e];
    }
}

// NT: past the caches.  Where a call moves more than the 256 MB that the memory-side cache
// holds, keeping the lines only displaces others: B4 S8192 Hq32 Hkv8 d128, 805 MB, 167 us
// through the caches and 151 past them; S4096 alone, 100 MB, 20 and 25 us.
template <bool NT>
__device__ __forceinline__ u32x4 load16(const uint16_t* p) {
    const u32x4* at = reinterpret_cast<const u32x4*>(p);
    return NT ? __builtin_nontemporal_load(at) : *at;
}

template <bool NT>
__device__ __forceinline__ void store16(uint16_t* p, u32x4 y) {
    u32x4* at = reinterpret_cast<u32x4*>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(y, at);
    else
        *at = y;
}

template <bool NT>
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];  // round to nearest even
    store16<NT>(p, __builtin_bit_cast(u32x4, y));
}

// 8 weights of a lane's columns
__device__ __forceinline__ void load_weight(const void* w, int w_f32, int col, float (&x)[8]) {
    if (w_f32)
        load8(static_cast<const float*>(w) + col, x);
    else
        load8(static_cast<const uint16_t*>(w) + col, x);
}

// Sum over the L lanes (8 or 16, aligned) that hold one row; every lane gets it.
template <int L>
__device__ __forceinline__ float row_sum(float x) {
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, false));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, false));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, false));
    if constexpr (L == 16)
        x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xF, 0xF, false));
    return x;
}

// The tokens of a tile, and cos and sin of their angles.
template <int D>
struct RopeLds {
    float cs[2][kRopeMaxTile * (D / 2)];  // [token][pair]
    int b[kRopeMaxTile], s[kRopeMaxTile];
};

template <int D>
__device__ __forceinline__ void load_tile(RopeLds<D>& lds, const RopeArgs& a, long long token0,
                                          int tile) {
    const int half = a.rot / 2;
    for (int t = threadIdx.x; t < tile; t += kRopeThreads) {
        const long long token = token0 + t < a.tokens ? token0 + t : a.tokens - 1;
        const int b = (int)(token / a.S);
        lds.b[t] = b;
        lds.s[t] = (int)(token - (long long)b * a.S);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tile * half; i += kRopeThreads) {
        const int t = i / half, pair = i - t * half;
        double pos = lds.s[t];
        if (a.positions) {
            const long long at = lds.b[t] * a.positions_batch_stride + lds.s[t];
            pos = a.positions_i64 ? (double)static_cast<const long long*>(a.positions)[at]
                                  : (double)static_cast<const int*>(a.positions)[at];
        }
        // in turns, and of those only the fraction
        double turn = pos * (double)a.inv_freq[pair] * 0.15915494309189533577;
        turn -= rint(turn);
        float sn, cn;
        sincospif(2.0f * (float)turn, &sn, &cn);
        lds.cs[0][i] = cn;
        lds.cs[1][i] = sn;
    }
    __syncthreads();
}

// The rotation of a lane's 8 columns of its token's rows, y cos + mate sin with the mate
// of each column: of the next or last column (IL, interleaved pairs), or of the same one
// in the lane half / 8 further or back.  Columns past rot turn by 0.
template <int D, bool IL>
struct Rotation {
    float cn[IL ? 4 : 8], sn[IL ? 4 : 8];
    int mate;    // lane * 4
    bool whole;  // D = 128, all of it rotated: the mate is 8 lanes on, within each 16

    // sign -1: back
    __device__ __forceinline__ void init(const RopeLds<D>& lds, int t, int lane_col, int rot,
                                         float sign) {
        const int half = rot / 2, lane = threadIdx.x & 63;
        const bool in = lane_col * 8 < rot, second = lane_col * 8 >= half;
        const int first = !in ? 0 : IL ? lane_col * 4 : lane_col * 8 - (second ? half : 0);
        whole = D == 128 && rot == D;
        mate = (IL || !in ? lane : second ? lane - half / 8 : lane + half / 8) * 4;
#pragma unroll
        for (int e = 0; e < (IL ? 4 : 8); ++e) {
            cn[e] = in ? lds.cs[0][t * half + first + e] : 1.f;
            sn[e] = in ? lds.cs[1][t * half + first + e] * (IL || second ? sign : -sign) : 0.f;
        }
    }
    // every lane of the wave takes part
    __device__ __forceinline__ void turn(float (&y)[8]) const {
        if constexpr (IL) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = y[2 * e], q = y[2 * e + 1];
                y[2 * e] = p * cn[e] - q * sn[e];
                y[2 * e + 1] = q * cn[e] + p * sn[e];
            }
        } else if (whole) {  // a register exchange (0x128: rows rotated by 8)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y[e] = y[e] * cn[e] + sn[e] * __int_as_float(__builtin_amdgcn_mov_dpp(
                                                  __float_as_int(y[e]), 0x128, 0xF, 0xF, false));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float other =
                    __int_as_float(__builtin_amdgcn_ds_bpermute(mate, __float_as_int(y[e])));
                y[e] = y[e] * cn[e] + other * sn[e];
            }
        }
    }
};

// A group of D / 8 lanes works on the rows of one token t of the tile (a power of two, at
// most the groups of a workgroup), heads first, first + step, ...; the groups that share
// a token, and workgroups along y, share its heads out.
struct GroupRows {
    int lane_col, t, first, step;
    template <int D>
    __device__ __forceinline__ void init(int tile_log2) {
        constexpr int L = D / 8, GROUPS = kRopeThreads / L;
        const int group = threadIdx.x / L;
        lane_col = threadIdx.x % L;
        t = group & ((1 << tile_log2) - 1);
        first = blockIdx.y * (GROUPS >> tile_log2) + (group >> tile_log2);
        step = gridDim.y * (GROUPS >> tile_log2);
    }
    // passes over `heads` heads that the workgroup makes together
    __device__ __forceinline__ int passes(int heads) const { return (heads + step - 1) / step; }
};

__device__ __forceinline__ long long token_offset(const attn_heads& h, int b, int s) {
    return b * h.batch_stride + s * h.row_stride;
}

// Several rows are loaded before the first is worked on, to have enough bytes on their way:
// B4 S8192 Hq32 Hkv8 d128, 805 MB, 152 us (5.3 TB/s, a large copy's rate).  With few heads to a
// token the tile's positions, angles and two barriers ahead of the first row show: B8 S12857 Hq1
// Hkv1 d64, 79 MB, 38 us (2.1 TB/s).
template <int D, bool IL, bool NT>
__global__ __launch_bounds__(kRopeThreads) void rope_fwd_kernel(const RopeArgs a) {
    constexpr int L = D / 8, U = 4;
    __shared__ RopeLds<D> lds;
    const long long token0 = (long long)blockIdx.x << a.tile_log2;
    load_tile<D>(lds, a, token0, 1 << a.tile_log2);
    GroupRows g;
    g.init<D>(a.tile_log2);
    const int b = lds.b[g.t], s = lds.s[g.t];
    const bool token = token0 + g.t < a.tokens;
    Rotation<D, IL> rotation;
    rotation.init(lds, g.t, g.lane_col, a.rot, 1.0f);
    auto rows = [&](auto which_tag, int heads) __attribute__((always_inline)) {
        constexpr int which = decltype(which_tag)::value;
        const attn_heads in = a.in[which], out = a.out[which];
        const uint16_t* src =
            static_cast<const uint16_t*>(in.ptr) + token_offset(in, b, s) + g.lane_col * 8;
        uint16_t* dst = static_cast<uint16_t*>(out.ptr) + token_offset(out, b, s) + g.lane_col * 8;
        float w[8];
        if constexpr (which < 2)
            load_weight(a.weight[which < 2 ? which : 0], a.weight_f32, g.lane_col * 8, w);
        const int n = g.passes(heads);
        for (int i = 0; i < n; i += U) {
            u32x4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int head = min(g.first + (i + u) * g.step, heads - 1);
                raw[u] = load16<NT>(src + head * in.head_stride);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int head = g.first + (i + u) * g.step;
                uint16_t* to = dst + head * out.head_stride;
                if constexpr (which == 2) {
                    if (token && head < heads) store16<NT>(to, raw[u]);
                } else {
                    float x[8];
                    widen8(raw[u], x);
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
                    const float rs = rsqrtf(row_sum<L>(ss) * (1.0f / D) + a.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * rs * w[e];
                    rotation.turn(x);
                    if (token && head < heads) store8<NT>(to, x);
                }
            }
        }
    };
    rows(std::integral_constant<int, 0>{}, a.Hq);
    rows(std::integral_constant<int, 1>{}, a.Hkv);
    if (a.in[2].ptr) rows(std::integral_constant<int, 2>{}, a.Hkv);
}

// in: the gradients of the outputs (bf16, or fp32 with G32); x: the forward pass's
// inputs; out: their gradients.  Workgroups walk the tiles in steps of the grid; each
// leaves the sums of its rows' weight gradients in ws[q, k][D/16][workgroup][16], which
// rope_weight_kernel adds up in a fixed order.  B4 S8192 Hq32 Hkv8 d128, 1.14 GB, 240 us
// (4.8 TB/s); B2 S1777 H16 d64, 58 MB, 14.5 us (4.0 TB/s: one tile to most workgroups, whose
// angles come before its first row).
template <int D, bool IL, bool G32, bool NT>
__global__ __launch_bounds__(kRopeThreads, 3) void rope_bwd_kernel(const RopeArgs a) {
    constexpr int L = D / 8, GROUPS = kRopeThreads / L, U = 2;
    typedef typename std::conditional<G32, float, uint16_t>::type grad_t;
    __shared__ RopeLds<D> lds;
    __shared__ float sums[GROUPS][D];
    GroupRows g;
    g.init<D>(a.tile_log2);
    const int tile = 1 << a.tile_log2;
    const long long tiles = (a.tokens + tile - 1) >> a.tile_log2;
    float dw[2][8] = {};
    for (long long tl = blockIdx.x; tl < tiles; tl += gridDim.x) {
        const long long token0 = tl << a.tile_log2;
        if (tl != blockIdx.x) __syncthreads();  // the last tile's angles are still read
        load_tile<D>(lds, a, token0, tile);
        const int b = lds.b[g.t], s = lds.s[g.t];
        const bool token = token0 + g.t < a.tokens;
        Rotation<D, IL> rotation;
        rotation.init(lds, g.t, g.lane_col, a.rot, -1.0f);
        auto rows = [&](auto which_tag, int heads) __attribute__((always_inline)) {
            constexpr int which = decltype(which_tag)::value, qk = which < 2 ? which : 0;
            const attn_heads in = a.in[which], out = a.out[which], xin = a.x[qk];
            const int c = g.lane_col * 8;
            const grad_t* src = static_cast<const grad_t*>(in.ptr) + token_offset(in, b, s) + c;
            const uint16_t* xs =
                static_cast<const uint16_t*>(xin.ptr) + token_offset(xin, b, s) + c;
            uint16_t* dst = static_cast<uint16_t*>(out.ptr) + token_offset(out, b, s) + c;
            float w[8];
            if constexpr (which < 2) load_weight(a.weight[qk], a.weight_f32, c, w);
            const int n = g.passes(heads);
            for (int i = 0; i < n; i += U) {
                float gr[U][8];
                u32x4 raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int head = min(g.first + (i + u) * g.step, heads - 1);
                    load8(src + head * in.head_stride, gr[u]);
                    if constexpr (which < 2)
                        raw[u] = load16<NT>(xs + head * xin.head_stride);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int head = g.first + (i + u) * g.step;
                    const bool live = token && head < heads;
                    uint16_t* to = dst + head * out.head_stride;
                    if constexpr (which < 2) {
                        float x[8];
                        widen8(raw[u], x);
                        rotation.turn(gr[u]);
                        float ss = 0.f, sg = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            ss = fmaf(x[e], x[e], ss);
                            sg = fmaf(gr[u][e] * w[e], x[e], sg);
                        }
                        ss = row_sum<L>(ss);
                        sg = row_sum<L>(sg);
                        const float rs = rsqrtf(ss * (1.0f / D) + a.eps);
                        const float mean = sg * rs * (1.0f / D);  // mean(g' w x r)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float xn = x[e] * rs;
                            if (live) dw[qk][e] = fmaf(gr[u][e], xn, dw[qk][e]);
                            gr[u][e] = rs * (gr[u][e] * w[e] - xn * mean);
                        }
                    }
                    if (live) store8<NT>(to, gr[u]);
                }
            }
        };
        rows(std::integral_constant<int, 0>{}, a.Hq);
        rows(std::integral_constant<int, 1>{}, a.Hkv);
        if (a.in[2].ptr) rows(std::integral_constant<int, 2>{}, a.Hkv);
    }
    if (!a.ws) return;
    const int n = gridDim.x * gridDim.y, at = (blockIdx.y * gridDim.x + blockIdx.x) * 16;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[threadIdx.x / L][g.lane_col * 8 + e] = dw[which][e];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += kRopeThreads) {
            float sum = 0.f;
            for (int i = 0; i < GROUPS; ++i) sum += sums[i][c];
            a.ws[(which * (D / 16) + c / 16) * (n * 16) + at + c % 16] = sum;
        }
    }
}

// dw[c] = sum over n workgroups, in a fixed order and in double precision (long sums of
// either sign).  A workgroup takes 16 values, whose addends lie together, four to a thread;
// the addends of all of a workgroup's values together instead, and so apart here: 7.2 us
// instead of 4.8 (n = 1024, 2 x 128 values).
__global__ __launch_bounds__(512) void rope_weight_kernel(const float* ws, int n, int D,
                                                          float* dqw, float* dkw) {
    __shared__ double part[8][16];
    const int quad = threadIdx.x % 4;
    const float* p = ws + (long long)blockIdx.x * n * 16 + quad * 4;
    double s[4] = {};
#pragma unroll 8
    for (int i = threadIdx.x / 4; i < n; i += 128) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(p + i * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += (double)x[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int m = 32; m >= 4; m /= 2) s[e] += __shfl_xor(s[e], m, 64);
        if (threadIdx.x % 64 < 4) part[threadIdx.x / 64][quad * 4 + e] = s[e];
    }
    __syncthreads();
    if (threadIdx.x >= 16) return;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += part[i][threadIdx.x];
    const int c = blockIdx.x * 16 + threadIdx.x;
    (c < D ? dqw : dkw - D)[c] = (float)sum;
}

}  // namespace

RopeLaunch rope_launch(long long tokens, int Hq, int Hkv, int d, int num_cus, bool backward) {
    const int rpp = kRopeThreads / (d / 8);
    RopeLaunch l;
    // up to 16 tokens to a tile, fewer where that leaves compute units without a tile
    while (l.tile_log2 < 4 && (tokens >> (l.tile_log2 + 1)) >= 2 * num_cus) ++l.tile_log2;
    const long long tiles = (tokens + (1 << l.tile_log2) - 1) >> l.tile_log2;
    // few tiles: their rows are shared out among workgroups
    const long long passes = (((long long)(Hq > Hkv ? Hq : Hkv) << l.tile_log2) + rpp - 1) / rpp;
    long long y = 1;
    while (y < passes && tiles * y < 2 * num_cus) ++y;
    l.grid_y = (int)y;
    const long long cap = backward ? 4LL * num_cus : 0x7fffffffLL;
    l.grid_x = (int)(tiles < cap ? tiles : cap);
    return l;
}

namespace {
template <int D, bool IL, bool NT>
hipError_t launch_fwd(const RopeArgs& a, const dim3& grid, hipStream_t stream) {
    rope_fwd_kernel<D, IL, NT><<<grid, kRopeThreads, 0, stream>>>(a);
    return hipGetLastError();
}
template <int D, bool IL, bool NT>
hipError_t launch_bwd(const RopeArgs& a, const dim3& grid, int grad_f32, hipStream_t stream) {
    if (grad_f32)
        rope_bwd_kernel<D, IL, true, NT><<<grid, kRopeThreads, 0, stream>>>(a);
    else
        rope_bwd_kernel<D, IL, false, NT><<<grid, kRopeThreads, 0, stream>>>(a);
    return hipGetLastError();
}
// f(D, interleaved, past the caches), as compile-time values
template <typename F>
hipError_t rope_variant(int d, int interleaved, bool nt, F f) {
    using T = std::true_type;
    using N = std::false_type;
    auto with = [&](auto dim) {
        if (interleaved) return nt ? f(dim, T{}, T{}) : f(dim, T{}, N{});
        return nt ? f(dim, N{}, T{}) : f(dim, N{}, N{});
    };
    return d == 64 ? with(std::integral_constant<int, 64>{})
                   : with(std::integral_constant<int, 128>{});
}
bool past_caches(const RopeArgs& a, int d, int bytes_per_value) {
    return a.tokens * (a.Hq + 2LL * a.Hkv) * d * bytes_per_value > 256LL << 20;
}
}  // namespace

hipError_t launch_rope(const RopeArgs& a, const RopeLaunch& l, int d, hipStream_t stream) {
    const dim3 grid(l.grid_x, l.grid_y);
    return rope_variant(d, a.interleaved, past_caches(a, d, 4), [&](auto D, auto IL, auto NT) {
        return launch_fwd<decltype(D)::value, decltype(IL)::value, decltype(NT)::value>(a, grid,
                                                                                      stream);
    });
}

hipError_t launch_rope_bwd(const RopeArgs& a, const RopeLaunch& l, int d, int grad_f32,
                           float* dq_weight, float* dk_weight, hipStream_t stream) {
    const dim3 grid(l.grid_x, l.grid_y);
    const hipError_t e = rope_variant(
        d, a.interleaved, past_caches(a, d, grad_f32 ? 8 : 6), [&](auto D, auto IL, auto NT) {
            return launch_bwd<decltype(D)::value, decltype(IL)::value, decltype(NT)::value>(
                a, grid, grad_f32, stream);
        });
    if (e != hipSuccess || !a.ws) return e;
    rope_weight_kernel<<<2 * d / 16, 512, 0, stream>>>(a.ws, l.grid_x * l.grid_y, d, dq_weight,
                                                  dk_weight);
    return hipGetLastError();
}

}  // namespace attn
