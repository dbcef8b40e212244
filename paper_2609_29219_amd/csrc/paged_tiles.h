// Attention of requests with many new tokens over a paged cache (see paged_rows.hip for the
// definition, and for the requests with few).
//
// A workgroup computes a block of 256 rows (token by token, row = token * group + head of the
// group) of one request and key/value head: S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_32x32x16_bf16, K and V in tiles of 64 keys through LDS, an online softmax.  Each of
// the eight waves has 32 rows, one to a lane and its mate 32 lanes on, so the softmax is in a lane
// but for one exchange.  The products' accumulators give lane half h, in register r, key
// 8 (r / 4) + 4 h + r % 4; the weights of a step of 16 keys are the second product's operand as
// they stand, and V's rows are read from LDS (transposed) in that order: keys 4 h .. 4 h + 3, then
// 8 further.
//
// Bound: the matrix cores with the softmax's exponentials beside them.  Each wave issues the
// products of S of the next tile and of PV of this one one by one, with the softmax of this tile
// between them; while it does, the next tiles come from memory straight into LDS (two slots to
// an operand, one barrier to a tile).  A prompt of 8192 tokens, 32 heads of 128: 490 us, 1120
// TFLOP/s (535 on a slower card); the same over contiguous keys, by attn_fwd, 466.  A chunk of 512 tokens over 16384
// keys, 32 query heads to 8: 129 us.  (Four waves to a block of 128 rows load each tile twice as
// often: 64 requests of 40 rows over 8192 keys 94 us, so 67.  With the weights' sums on the matrix
// cores, as in fwd_kernel.h, the prompt takes the same time, at d = 64 2% less.)
//
// Pages.  A wave brings aligned runs of 16 keys, which lie in one page (or two of eight rows), of
// K or of V: the page number is a scalar, and so is all arithmetic on it; a lane's offset inside
// the run never changes.  Page numbers are read a tile ahead.  Tiles lie in LDS as whole rows,
// 1 KiB to an instruction, their 16-byte pieces exchanged inside a row (by the source address of
// each lane) so that both kinds of reads are free of bank conflicts: K is read 16 rows at a time,
// V four rows of 64 bytes.
//
// Work.  The blocks of all requests are found by each workgroup from the lengths; the last block
// of a request (the longest under a causal mask) comes first, and the heads are dealt to the XCDs.
// Where the host sees too few blocks to fill the device, each block's keys are split; the parts
// (unnormalised, with their maximum) go to the workspace, and a second kernel adds them in order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwd_kernel.h"
#include "paged.h"
#include "paged_device.h"

namespace attn {

constexpr int kTileKeys = 64;

// Tiles in LDS: K's pieces of 1 KiB are 16 bytes apart, V's lie end to end.
template <int D>
struct PagedLds {
    static constexpr int PIECE_ROWS = 512 / D;                    // rows to 1 KiB
    static constexpr int PIECES = kTileKeys / PIECE_ROWS;
    static constexpr int K_PIECE = 1024 + 16, V_PIECE = 1024;     // bytes
    static constexpr int K_TILE = PIECES * K_PIECE, V_TILE = PIECES * V_PIECE;
    static constexpr int BYTES = 2 * (K_TILE + V_TILE);
    // where in its row a 16-byte piece c of row lies (an involution)
    __device__ static constexpr int k_swap(int row) {
        return D == 128 ? 4 * (row & 3) : 2 * ((row >> 1) & 3);
    }
    __device__ static constexpr int v_swap(int row) {
        return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
    }
};

// FORM: 1 capped scores, 2 slopes, 3 both, 4 slopes under a causal mask.  The distance is then
// linear, and slope (j - p) in the products' own units is what their accumulators begin with,
// rounded with them: a prompt of 4096 tokens, 16 query heads to 4, 119 us, in form 2 128.
template <int D, int FORM>
__global__ __launch_bounds__(512, 2) void paged_tiles_kernel(const PagedArgs a) {
    using L = PagedLds<D>;
    constexpr int NW = 8, NT = NW * 64, BM = kPagedTileRows, BN = kTileKeys;
    static_assert(BM == 32 * NW, "");
    constexpr int KD = D / 16, KB = BN / 32, CB = D / 32;
    constexpr int JOB_PIECES = 16 / L::PIECE_ROWS;  // instructions to a wave's part of a tile
    constexpr int STAGE = NW * kFwdStageWaveBytes;
    __shared__ __attribute__((aligned(16))) uint8_t lds[L::BYTES > STAGE ? L::BYTES : STAGE];
    __shared__ int found[2];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, hh = lane >> 5;

    // ---- this workgroup's block: (block of all requests, split), head ---------------
    const int unit = blockIdx.x / a.Hkv, head = blockIdx.x - unit * a.Hkv;
    const int nth = unit / a.splits, split = unit - nth * a.splits;
    int* const meta = a.tile_meta + ((long long)nth * a.Hkv + head) * kPagedMeta;
    auto blocks_of = [&](const PagedRequest& x) __attribute__((always_inline)) -> int {
        const long long rows = (long long)x.qn * a.group;
        return rows > a.few ? (int)((uint32_t)(rows + BM - 1) / BM) : 0;
    };
    const PagedFound here = paged_find<NT>(a, nth, found, blocks_of);
    const int r = here.r;
    if (r < 0) {  // there are fewer blocks
        if (a.splits > 1 && split == 0 && tid == 0) meta[0] = 0;
        return;
    }
    const PagedRequest x = here.x;
    const int n_blocks = (x.qn * a.group + BM - 1) / BM;
    const int blk = n_blocks - 1 - (nth - here.first);
    const int n_rows = min(x.qn * a.group - blk * BM, BM);

    // ---- its rows and keys -------------------------------------------------------
    const int w_row0 = blk * BM + wave * 32;                // first row of this wave
    const int last_row = blk * BM + n_rows - 1;
    const GroupDiv rows(a, blk * BM);
    int qh;
    const int tok = rows.token(min(wave * 32 + l32, n_rows - 1), &qh);  // rows past the end repeat
    qh += head * a.group;                                               // the last
    auto pos_of = [&](int rr) {
        int unused;
        return x.pos0 + rows.token(min(rr, last_row) - blk * BM, &unused);
    };
    const int pos = x.pos0 + tok;
    const int hi = a.causal ? min(pos, x.kv - 1) : x.kv - 1;
    const int lo = a.window ? pos - a.window + 1 : 0;
    // tiles of the block, of this split, and of the wave
    const int b_hi = a.causal ? min(pos_of(last_row), x.kv - 1) : x.kv - 1;
    const int b_lo = a.window ? max(pos_of(blk * BM) - a.window + 1, 0) : 0;
    const int tb = b_lo / BN, te = b_hi >= b_lo ? b_hi / BN + 1 : tb;
    const int n_splits = max(1, min(a.splits, (te - tb) / kPagedMinTiles));
    if (a.splits > 1 && split == 0 && tid == 0) {
        meta[1] = x.q0;
        meta[2] = head * a.group;
        meta[3] = blk * BM;
        meta[4] = n_rows;
        meta[0] = n_splits > 1 ? n_splits : 0;
    }
    if (split >= n_splits) return;
    const int t_begin = tb + (int)((long long)(te - tb) * split / n_splits);
    const int t_end = tb + (int)((long long)(te - tb) * (split + 1) / n_splits);
    const int w_lo_row = min(w_row0, last_row), w_hi_row = min(w_row0 + 31, last_row);
    const int w_hi_min = a.causal ? pos_of(w_lo_row) : x.kv - 1;  // seen by every row ...
    const int w_hi_max = a.causal ? min(pos_of(w_hi_row), x.kv - 1) : x.kv - 1;  // ... by any
    const int w_lo_max = a.window ? pos_of(w_hi_row) - a.window + 1 : 0;
    // the wave's last tile (before t_begin: it has none)
    const int t_last = w_row0 > last_row || w_hi_max < 0 ? t_begin - 1
                                                         : min(t_end - 1, w_hi_max / BN);

    // ---- queries: B operand, 16 dims x 32 rows ------------------------------------
    bf16x8 qf[KD];
    {
        const uint16_t* const qp = a.q + (x.q0 + tok) * a.q_row + qh * a.q_head + hh * 8;
#pragma unroll
        for (int ks = 0; ks < KD; ++ks)
            qf[ks] = __builtin_bit_cast(
                bf16x8, *reinterpret_cast<const u32x4*>(qp + ks * 16) ^ a.q_sign);
    }
    float slope = 0.f;
    if constexpr (FORM & 2) slope = a.slopes[qh] * 1.4426950408889634f;
    if constexpr (FORM == 4)  // (finite: 0 times it has to be 0)
        slope = fmaxf(fminf(a.slopes[qh] * 1.4426950408889634f / a.scale_log2, 3.4e38f), -3.4e38f);

    // ---- tile loads ------------------------------------------------------------
    // A tile's 64 rows of K are four waves' job, 16 rows to each, and V's the others', so that a
    // wave has one page to find for a tile (two of eight rows).
    const int* const table = a.table + (long long)r * a.table_stride;
    const int page_mask = (1 << a.page_log2) - 1;
    const bool small_pages = a.page_log2 == 3;
    const uint32_t lds_base = lds_address(lds);
    constexpr int KS0 = 0, KS1 = L::K_TILE, VS0 = 2 * L::K_TILE, VS1 = VS0 + L::V_TILE;
    bool bad = x.bad != 0;
    const int p_row = lane / (D / 8), p_chunk = lane % (D / 8);  // this lane's place in 1 KiB
    const int last_key = x.kv - 1;
    const bool is_k = wave < 4;
    const PagedSide& side = is_k ? a.k : a.v;
    const uint16_t* const base = side.ptr + head * side.head;
    const uint32_t page16 = side.page16, row16 = side.row16;
    const int ahead = is_k ? 2 : 1;  // tiles from the one at work to the one that is loaded
    const int job_row = 16 * (wave & 3);
    const int piece = is_k ? L::K_PIECE : L::V_PIECE;
    const int slot0 = (is_k ? KS0 : VS0) + job_row / L::PIECE_ROWS * piece;
    const int slot1 = slot0 + (is_k ? L::K_TILE : L::V_TILE);
    // this lane's source in the job's first piece
    const int swap = p_chunk ^ (is_k ? L::k_swap(p_row) : L::v_swap(p_row));
    const int off = p_row * (int)row16 * 16 + swap * 16;
    int next0 = 0, next1 = 0;  // page numbers of the next tile that is loaded
    // first key of `n` (8 or 16) aligned ones, clamped to those that hold a key that some row sees
    auto run_of = [&](int t, int at, int n) __attribute__((always_inline)) {
        return max(min(t * BN + job_row + at, last_key & ~(n - 1)), x.lo & ~(n - 1));
    };
    // (as vector loads, which land with the tiles' before the barrier: scalar ones would hold up
    // the tile's first reads from LDS, which are waited for by the same count)
    int zero;
    asm volatile("v_mov_b32 %0, 0" : "=v"(zero));
    auto entry0_of = [&](int t) __attribute__((always_inline)) -> int {
        const int at = small_pages ? run_of(t, 0, 8) >> 3 : run_of(t, 0, 16) >> a.page_log2;
        return table[at + zero];
    };
    auto entry1_of = [&](int t) __attribute__((always_inline)) -> int {  // with small_pages
        return table[(run_of(t, 8, 8) >> 3) + zero];
    };
    // Rows of tile t from piece p0 to p1 of the job, which lie in page `entry` from key0 on.
    auto bring_run = [&](int t, int key0, int entry, auto p0c, auto p1c, int slot)
        __attribute__((always_inline)) {
        constexpr int p0 = decltype(p0c)::value, p1 = decltype(p1c)::value;
        const bool out = (uint32_t)entry >= (uint32_t)a.n_pages;
        bad |= out;
        const uint64_t at = (uint64_t)(uint32_t)(out ? 0 : entry) * page16 +
                            (uint64_t)(uint32_t)(key0 & page_mask) * row16;
        const dma_rsrc_t rsrc = make_dma_rsrc(base + at * 8, 0x7fffffffu);
        if (t * BN < x.lo || t * BN + BN > x.kv) {
            // keys that no row sees are copies of the nearest that one does
#pragma unroll 1
            for (int p = 0; p < p1 - p0; ++p) {
                const int rr = p * L::PIECE_ROWS + p_row;
                const int from = max(min(key0 + rr, last_key), x.lo) - key0;
                lds_dma16(rsrc, lds_base + slot + (p0 + p) * piece,
                          from * (int)row16 * 16 + swap * 16, 0);
            }
        } else {
#pragma unroll
            for (int p = p0; p < p1; ++p)
                lds_dma16(rsrc, lds_base + slot + p * piece, off,
                          (p - p0) * L::PIECE_ROWS * (int)row16 * 16);
        }
    };
    auto bring_job = [&](int t, int slot, int entry0, int entry1) __attribute__((always_inline)) {
        using std::integral_constant;
        auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
        integral_constant<int, 0> none;
        integral_constant<int, JOB_PIECES / 2> half;
        integral_constant<int, JOB_PIECES> all;
        if (small_pages) {
            bring_run(t, run_of(t, 0, 8), uniform(entry0), none, half, slot);
            bring_run(t, run_of(t, 8, 8), uniform(entry1), half, all, slot);
        } else {
            bring_run(t, run_of(t, 0, 16), uniform(entry0), none, all, slot);
        }
    };

    // ---- online softmax, one row to a lane ------------------------------------
    float m_i = -INFINITY;  // reference of the row's weights, log2 units
    float l_i = 0.f;        // their sum (this lane's half of the keys), unrounded: the
                            // log-sum-exp is fp32's
    f32x16 oacc[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[cb][e] = 0.f;
    const float scale_log2 = a.scale_log2;
    constexpr bool LOG2 = FORM >= 1 && FORM <= 3;

    // K operands: lane reads row l32 of a 32-row block, 16-byte piece 2 ks + hh
    const uint8_t* k_at[KD];
#pragma unroll
    for (int ks = 0; ks < KD; ++ks)
        k_at[ks] = lds + (l32 / L::PIECE_ROWS) * L::K_PIECE + (l32 % L::PIECE_ROWS) * (D * 2) +
                   (((2 * ks + hh) ^ L::k_swap(l32)) * 16);
    constexpr int K_BLOCK = 32 / L::PIECE_ROWS * L::K_PIECE;  // bytes of 32 rows
    // V operands: lane i of 16 reads row i / 4 of four, at column 16 ((lane / 16) % 2) + 4 (i % 4)
    // of 32 (the rows' numbers are i / 4 more than multiples of 4)
    const int tr_row = (lane & 15) >> 2;
    const uint8_t* v_at[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
        v_at[cb] = lds + (4 * hh + tr_row) * (D * 2) + ((cb * 64) ^ (L::v_swap(tr_row) * 16)) +
                   ((lane >> 4) & 1) * 32 + 8 * (lane & 3);
    auto fetch_k = [&](int kslot, int kb, int ks) __attribute__((always_inline)) -> bf16x8 {
        return *reinterpret_cast<const bf16x8*>(k_at[ks] + kslot + kb * K_BLOCK);
    };
    auto fetch_v = [&](int vslot, int kb, int h2, int cb) __attribute__((always_inline)) -> bf16x8 {
        const uint16_t* const p = reinterpret_cast<const uint16_t*>(
            v_at[cb] + vslot + (kb * 32 + 16 * h2) * (D * 2));
        const s16x4 w0 = lds_read_tr(p), w1 = lds_read_tr(p + 8 * D);
        const s16x8 w = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
        return __builtin_bit_cast(bf16x8, w);
    };
    // A score of tile t, capped, moved and masked.  With form 1 to 3: in log2 units from here on.
    // c: its key less t * BN + 4 hh; room, below: the last and the first such that is seen
    auto finish = [&](float s, int c, float away, int room, int below, auto mask_tag)
        __attribute__((always_inline)) -> float {
        if constexpr (FORM & 1) {
            s = capped(s * a.cap_in, a.cap_out);
        } else if constexpr (FORM == 2) {
            s *= scale_log2;
        }
        if constexpr (FORM & 2) s = fmaf(-slope, fabsf(away - (float)c), s);
        if (decltype(mask_tag)::value && (c > room || c < below)) s = -INFINITY;
        return s;
    };
    auto key_const = [](int kb, int e) { return kb * 32 + 8 * (e >> 2) + (e & 3); };

    // The reference moves only when a tile's maximum exceeds it by more than kRescaleSlack:
    // weights are then at most 2^8.  Returns what to subtract (0 before the first key).
    auto update_ref = [&](float mx) __attribute__((always_inline)) -> float {
        const float tmax = LOG2 || mx == -INFINITY ? mx : mx * scale_log2;
        const bool move = tmax > m_i + kRescaleSlack;  // also the first finite one
        if (__any(move)) {
            const float m_new = move ? tmax : m_i;
            const float alpha = move ? __builtin_amdgcn_exp2f(m_i - m_new) : 1.f;
            l_i *= alpha;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[cb][e] *= alpha;
            m_i = m_new;
        }
        return m_i == -INFINITY ? 0.f : m_i;
    };
    auto weight = [&](float s, float m_ref) __attribute__((always_inline)) {
        return __builtin_amdgcn_exp2f(LOG2 ? s - m_ref : fmaf(s, scale_log2, -m_ref));
    };

    // One tile t: the products of S(t + 1) into s_nxt (HAS_S) and of PV(t), one by one; between
    // them the weights of tile t (scores s_cur) and, once S(t + 1) is there, its finished scores
    // and their maximum, which is returned.
    auto fused_tile = [&](auto odd_tag, const f32x16 (&s_cur)[KB], f32x16 (&s_nxt)[KB],
                          int t, float m_ref, auto has_s_tag, auto mask_tag)
        __attribute__((always_inline)) -> float {
        constexpr bool HAS_S = decltype(has_s_tag)::value, ODD = decltype(odd_tag)::value;
        constexpr int kslot = ODD ? KS0 : KS1, vslot = ODD ? VS1 : VS0;  // of tiles t + 1 and t
        constexpr int NS = HAS_S ? KB * KD : 0, NPV = KB * 2 * CB, NM = NS + NPV;
        constexpr int PF = 3;                                // operands on their way, and in use
        constexpr int NPAIR = KB * 8;
        constexpr int EXP_SLOTS = HAS_S ? NS + NPV / 2 : 0;  // slots with exponentials
        constexpr int MAX0 = EXP_SLOTS + 1;                  // first slot with the next maximum
        constexpr int NMAXV = HAS_S ? KB * 16 : 0;
        constexpr int LAG = HAS_S ? fwd_pair_lag(NPAIR, EXP_SLOTS, NS, CB) : 0;
        static_assert(!HAS_S || (LAG >= 0 && MAX0 < NM), "");
        bf16x8 pb[KB][2];
        float mx = -INFINITY, rs0 = 0.f, rs1 = 0.f;
        float xe[NPAIR][2];
        auto exps = [&](int pp) __attribute__((always_inline)) {
            const int kb = pp / 8, e = 2 * (pp % 8);
            xe[pp][0] = weight(s_cur[kb][e], m_ref);
            xe[pp][1] = weight(s_cur[kb][e + 1], m_ref);
        };
        // P is rounded to bf16 (at most 2^-8 of each weight) as the operand it has to be
        auto round_sum = [&](int pp) __attribute__((always_inline)) {
            const int kb = pp / 8, h2 = (pp / 4) % 2, e = 2 * (pp % 4);
            const bf16x2 pk = {(__bf16)xe[pp][0], (__bf16)xe[pp][1]};
            pb[kb][h2][e] = pk[0];
            pb[kb][h2][e + 1] = pk[1];
            rs0 += xe[pp][0];
            rs1 += xe[pp][1];
        };
        if (!HAS_S) {
#pragma unroll
            for (int pp = 0; pp < NPAIR; ++pp) {
                exps(pp);
                round_sum(pp);
            }
        }
        const int key1 = (t + 1) * BN + 4 * hh;
        const int room = hi - key1, below = lo - key1;
        const float away = (float)(pos - key1);
        auto fetch = [&](auto ic) __attribute__((always_inline)) -> bf16x8 {
            constexpr int i = decltype(ic)::value;
            if constexpr (i < NS) {
                return fetch_k(kslot, i % KB, i / KB);
            } else {
                constexpr int j = i - NS;
                return fetch_v(vslot, j / (2 * CB), (j / CB) % 2, j % CB);
            }
        };
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 fr[PF];
        static_for<0, PF - 1>([&](auto ic) __attribute__((always_inline)) {
            fr[decltype(ic)::value] = fetch(ic);
        });
        static_for<0, NM>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            const bf16x8 op = fr[i % PF];
            if constexpr (i + PF - 1 < NM)
                fr[(i + PF - 1) % PF] = fetch(std::integral_constant<int, i + PF - 1>{});
            if constexpr (i < NS) {
                constexpr int ks = i / KB, kb = i % KB;
                f32x16 c = {};
                if constexpr (ks > 0) {
                    c = s_nxt[kb];
                } else if constexpr (FORM == 4) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) c[e] = slope * ((float)key_const(kb, e) - away);
                }
                s_nxt[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, qf[ks], c, 0, 0, 0);
            } else {
                constexpr int j = i - NS, kb = j / (2 * CB), h2 = (j / CB) % 2, cb = j % CB;
                oacc[cb] =
                    __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, pb[kb][h2], oacc[cb], 0, 0, 0);
            }
            if constexpr (HAS_S) {
                static_for<0, NPAIR>([&](auto pc) __attribute__((always_inline)) {
                    constexpr int pp = decltype(pc)::value;
                    if constexpr (pp * EXP_SLOTS / NPAIR == i) exps(pp);
                    if constexpr (pp * EXP_SLOTS / NPAIR + LAG == i) round_sum(pp);
                });
                static_for<0, NMAXV>([&](auto vc) __attribute__((always_inline)) {
                    constexpr int v = decltype(vc)::value;
                    if constexpr (MAX0 + v * (NM - MAX0) / NMAXV == i) {
                        constexpr int kb = v / 16, e = v % 16;
                        if constexpr (LOG2 || decltype(mask_tag)::value)
                            s_nxt[kb][e] = finish(s_nxt[kb][e], key_const(kb, e), away, room,
                                                  below, mask_tag);
                        mx = __builtin_elementwise_maximum(mx, s_nxt[kb][e]);
                    }
                });
                asm volatile("" : "+v"(rs0), "+v"(rs1), "+v"(mx));
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        l_i += rs0 + rs1;
        return HAS_S ? half_swap_max(mx) : -INFINITY;
    };

    // ---- the loop ------------------------------------------------------------------
    // While iteration t runs, LDS holds K(t + 1) and V(t), and K(t + 2) and V(t + 1) come in:
    // tile j in slot (j - t_begin) % 2.  Page numbers are read an iteration ahead.
    f32x16 sA[KB], sB[KB];
    float mx_next = -INFINITY;
    const bool has_keys = t_end > t_begin;
    if (has_keys) {
        // (all page numbers first: a wait for one is a wait for every load before it)
        const int second = min(t_begin + 1, t_end - 1), third = min(t_begin + ahead, t_end - 1);
        const int a0 = entry0_of(t_begin), b0 = entry0_of(second);
        next0 = entry0_of(third);
        int a1 = 0, b1 = 0;
        if (small_pages) {
            a1 = entry1_of(t_begin);
            b1 = entry1_of(second);
            next1 = entry1_of(third);
        }
        bring_job(t_begin, slot0, a0, a1);
        if (is_k && t_begin + 1 < t_end) bring_job(t_begin + 1, slot1, b0, b1);
        publish_barrier<0>();
        if (t_last >= t_begin) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    // (the distance as a difference of integers: fp32 holds positions to 2^24)
                    sA[kb][e] = FORM == 4
                                    ? slope * (float)(t_begin * BN + 4 * hh + key_const(kb, e) - pos)
                                    : 0.f;
#pragma unroll
                for (int ks = 0; ks < KD; ++ks)
                    sA[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fetch_k(KS0, kb, ks), qf[ks],
                                                                     sA[kb], 0, 0, 0);
            }
            const int key0 = t_begin * BN + 4 * hh;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    sA[kb][e] = finish(sA[kb][e], key_const(kb, e), (float)(pos - key0), hi - key0,
                                       lo - key0, std::true_type{});
                    mx_next = __builtin_elementwise_maximum(mx_next, sA[kb][e]);
                }
            mx_next = half_swap_max(mx_next);
        }
        publish_barrier<0>();  // slot 0 takes K(t_begin + 2)
    }
    // loads of iteration t
    auto bring = [&](int t, bool odd) __attribute__((always_inline)) {
        const int to = t + ahead;
        if (to < t_end) bring_job(to, is_k == odd ? slot1 : slot0, next0, next1);
        const int then = min(to + 1, t_end - 1);
        next0 = entry0_of(then);
        if (small_pages) next1 = entry1_of(then);
    };
    // Iteration t of a wave: scores of an even tile (from t_begin) are in set A, of an odd one in
    // set B, so that slots and sets are known at compile time.
    auto iter = [&](auto odd_tag, int t, const f32x16 (&s_cur)[KB], f32x16 (&s_nxt)[KB],
                    auto mask_tag) __attribute__((always_inline)) {
        bring(t, decltype(odd_tag)::value);
        const float m_ref = update_ref(mx_next);
        mx_next = fused_tile(odd_tag, s_cur, s_nxt, t, m_ref, std::true_type{}, mask_tag);
        publish_barrier<0>();
    };
    // Iterations [t0, t1), t0 being even (from t_begin).
    auto run = [&](int t0, int t1, auto mask_tag) __attribute__((always_inline)) {
#pragma unroll 1
        for (int t = t0; t < t1; t += 2) {
            iter(std::false_type{}, t, sA, sB, mask_tag);
            if (t + 1 < t1) iter(std::true_type{}, t + 1, sB, sA, mask_tag);
        }
    };
    auto last_iter = [&](auto odd_tag, const f32x16 (&s_cur)[KB], f32x16 (&s_nxt)[KB])
        __attribute__((always_inline)) {
        bring(t_last, decltype(odd_tag)::value);
        const float m_ref = update_ref(mx_next);
        fused_tile(odd_tag, s_cur, s_nxt, t_last, m_ref, std::false_type{}, std::true_type{});
        publish_barrier<0>();
    };
    if (t_last >= t_begin) {
        // iteration t finishes tile t + 1: masked where the window begins, not in between (an
        // even number of tiles from an even one), masked at the diagonal and at the end
        const int first_free = max(w_lo_max + BN - 1, 0) / BN;
        const int first_masked = max(w_hi_min + 1, 0) / BN;
        int s1 = max(first_free - 1, t_begin);
        s1 = min(s1 + ((s1 - t_begin) & 1), t_last);
        int s2 = min(max(first_masked - 1, s1), t_last);
        s2 = max(s2 - ((s2 - t_begin) & 1), s1);
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            run(pass ? s2 : t_begin, pass ? t_last : s1, std::true_type{});
            if (pass == 0) run(s1, s2, std::false_type{});
        }
        if ((t_last - t_begin) & 1)
            last_iter(std::true_type{}, sB, sA);
        else
            last_iter(std::false_type{}, sA, sB);
    }
    for (int t = max(t_last + 1, t_begin); t < t_end; ++t) {
        bring(t, (t - t_begin) & 1);
        publish_barrier<0>();
    }

    // ---- epilogue: O = O^T / l, through LDS so that stores are whole lines ---------------
    bad = __syncthreads_or(bad);
    const float l_row = bad ? NAN : half_swap_sum(l_i);
    const bool partial = n_splits > 1;
    const float inv = partial ? 1.f : l_row == 0.f ? 0.f : 1.f / l_row;
    const bool out16 = a.out_bf16 && !partial;
    uint8_t* const stage = lds + wave * kFwdStageWaveBytes;
    constexpr int SROW = kFwdStageRowBytes;
    const long long part0 = (((long long)nth * a.Hkv + head) * a.splits + split) * BM;
    char* const obase = partial ? reinterpret_cast<char*>(a.tile_o) : static_cast<char*>(a.o);
    const int row_bytes = out16 ? 2 * D : 4 * D;
    long long orow[4];  // of the rows that this lane stores
    bool there[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = wave * 32 + (lane >> 3) + 8 * j;
        there[j] = i < n_rows;
        int h;
        const int tk = rows.token(i, &h);
        orow[j] = partial ? part0 + i : (long long)(x.q0 + tk) * a.Hq + head * a.group + h;
    }
    auto emit = [&](int piece) __attribute__((always_inline)) {
        u32x4 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = *reinterpret_cast<const u32x4*>(stage + ((lane >> 3) + 8 * j) * SROW +
                                                   (lane & 7) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (there[j])
                *reinterpret_cast<u32x4*>(obase + orow[j] * row_bytes + piece * 128 +
                                          (lane & 7) * 16) = w[j];
    };
    if (out16) {
        static_for<0, CB / 2>([&](auto pc) __attribute__((always_inline)) {
            constexpr int piece = decltype(pc)::value;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16& o = oacc[2 * piece + half];
                    const bf16x2 y0 = {(__bf16)(o[4 * g] * inv), (__bf16)(o[4 * g + 1] * inv)};
                    const bf16x2 y1 = {(__bf16)(o[4 * g + 2] * inv), (__bf16)(o[4 * g + 3] * inv)};
                    uint32_t* const to = reinterpret_cast<uint32_t*>(
                        stage + l32 * SROW + (half * 32 + 8 * g + 4 * hh) * 2);
                    to[0] = __builtin_bit_cast(uint32_t, y0);
                    to[1] = __builtin_bit_cast(uint32_t, y1);
                }
            asm volatile("" ::: "memory");  // staging writes before the reads
            emit(piece);
            asm volatile("" ::: "memory");  // and the reads before the next piece's writes
        });
    } else {
        static_for<0, CB>([&](auto pc) __attribute__((always_inline)) {
            constexpr int cb = decltype(pc)::value;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 y = {oacc[cb][4 * g] * inv, oacc[cb][4 * g + 1] * inv,
                                 oacc[cb][4 * g + 2] * inv, oacc[cb][4 * g + 3] * inv};
                *reinterpret_cast<f32x4*>(stage + l32 * SROW + (8 * g + 4 * hh) * 4) = y;
            }
            asm volatile("" ::: "memory");
            emit(cb);
            asm volatile("" ::: "memory");
        });
    }
    if (hh == 0 && w_row0 + l32 <= last_row) {
        if (partial) {
            a.tile_m[part0 + wave * 32 + l32] = m_i;
            a.tile_l[part0 + wave * 32 + l32] = l_row;
        } else if (a.lse) {
            a.lse[(long long)(x.q0 + tok) * a.Hq + qh] =
                l_row == 0.f ? -INFINITY : (m_i + __builtin_log2f(l_row)) * kLn2;
        }
    }
}

template <int D, int FORM>
hipError_t launch_paged_tiles_form(const PagedArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((paged_tiles_kernel<D, FORM>), dim3((unsigned)a.tile_wgs), dim3(512), 0,
                       stream, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_paged_tiles_d(const PagedArgs& a, int form, hipStream_t stream) {
    if (form == 0) return launch_paged_tiles_form<D, 0>(a, stream);
    if (form == 1) return launch_paged_tiles_form<D, 1>(a, stream);
    if (form == 2) return launch_paged_tiles_form<D, 2>(a, stream);
    if (form == 3) return launch_paged_tiles_form<D, 3>(a, stream);
    if (form == 4) return launch_paged_tiles_form<D, 4>(a, stream);
    return hipErrorInvalidValue;
}

}  // namespace attn
