// Declarations of the paged cache's operators: attention of new tokens over a cache whose rows
// lie in pages, and the tables, slots and stores that go with it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace attn {

// ------------------------------------------------------------------ tables --
struct ExtendArgs {
    int* table;
    long long table_stride;
    const int *seq_lens, *new_lens, *free_pages, *n_free;
    int *slots, *positions, *cu, *kv_lens, *n_left;
    int R, T, max_pages, n_list, page_log2;
};
struct ReleaseArgs {
    const int* table;
    long long table_stride;
    const int *seq_lens, *keep_lens, *n_free;
    int *free_pages, *n_left;
    int R, max_pages, n_list, page_log2;
};
struct StoreArgs {
    attn_heads k, v, k_pages, v_pages;  // (batch strides of k and v unused)
    const int* slots;
    int T, Hkv, n_pages, page_log2;
};
hipError_t launch_paged_extend(const ExtendArgs& a, hipStream_t stream);
hipError_t launch_paged_release(const ReleaseArgs& a, hipStream_t stream);
hipError_t launch_paged_store(const StoreArgs& a, int d, hipStream_t stream);

// --------------------------------------------------------------- attention --
constexpr int kPagedMinPageLog2 = 3;   // 8 rows of a tile lie in one page
constexpr int kPagedMaxPageLog2 = 16;

// A buffer of pages; head h of row s of page p starts at (p * page16 + s * row16) * 8 + h * head
// values
struct PagedSide {
    const uint16_t* ptr;
    uint32_t page16, row16;  // 16 bytes each
    long long head;
};

struct PagedArgs {
    const uint16_t* q;
    long long q_row, q_head;
    PagedSide k, v;
    void* o;          // [T][Hq][D], fp32 or bf16 (out_bf16)
    float* lse;       // [T][Hq] natural log, or null
    const int* table; // [R], table_stride apart
    long long table_stride;
    const int *kv_lens, *cu;  // cu null: token r is request r's
    const float* slopes;      // [Hq] or null
    int T, R, Hq, Hkv, group;
    uint32_t group_inverse;   // 2^32 / group, rounded up (group at most kPagedMaxGroup)
    int n_pages, page_log2, max_pages;
    int causal, window;       // window 0: none
    int out_bf16;
    int few;                  // requests of up to this many rows (of all heads of a group) are
                              // the row kernel's
    float scale_log2;         // |scale| * log2(e), > 0
    float cap_in, cap_out;    // capped scores in log2 units: cap_out tanh(s cap_in / (2 log2 e));
                              // cap_out 0: not capped
    uint32_t q_sign;          // sign bits xor-ed into Q (negative scale)
    // Partial results of the row kernel, two to a workgroup: [workgroup][2][rows] of ws_m (log2
    // units), ws_l and ws_o (D values each), and what the second one belongs to; meta null: no
    // item is shared by workgroups
    float *ws_m, *ws_l, *ws_o;
    int* meta;
    int n_wg;
    int unit_log2;  // its work is shared out in units of 2^unit_log2 steps
    // The tile kernel's blocks of rows: their keys split `splits` ways at most, whose partial
    // results lie at [block][head][split][row]
    int splits;
    long long tile_wgs;
    float *tile_m, *tile_l, *tile_o;
    int* tile_meta;
};

// A request as the kernels see it.
struct PagedRequest {
    int q0, qn;    // its tokens in q: first, how many
    int pos0;      // position of the first
    int kv, lo;    // its keys that any token sees: [lo, kv)
    int bad;       // more keys than its table holds
};

// Keys to a step of the row kernel (with four waves), and its workgroups that a compute unit holds
// at once: as many as share the work of a call, since one more would have its part alone at the
// end.  (By LDS at d = 64 with 16 rows and at d = 128, by registers at d = 64 with 32 rows, of
// which 32 times 8 over 4096 keys take 61 us by three, by four 70.)
constexpr int kPagedRowKeys = 128;
constexpr int paged_row_wgs_per_cu(int d, int block) { return d == 128 ? 2 : block == 16 ? 4 : 3; }
constexpr int kPagedMeta = 8;  // ints to a workgroup
constexpr int kPagedMaxGroup = 1 << 15;
// Requests of up to this many rows are the row kernel's (by 16 or 32 rows), which streams
// a little faster and shares its work evenly among workgroups whatever the lengths are; beyond,
// its block's state no longer fits in registers.  32 requests of 32 rows over 4096 keys of 8
// heads: 100 us, by the tile kernel 102.
constexpr int kPagedFewRows = 32;
hipError_t launch_paged_rows(const PagedArgs& a, int d, int block, int waves, hipStream_t stream);
// Adds both kernels' partial results.
hipError_t launch_paged_sums(const PagedArgs& a, int d, int row_block, hipStream_t stream);
// Fewest tiles of keys to a split of the tile kernel (a start costs as much as three), and most
// splits of a block.
constexpr int kPagedMinTiles = 4;
constexpr int kPagedMaxSplits = 64;
constexpr int kPagedTileRows = 256;  // to a block of the tile kernel
// form: 1 capped scores, 2 slopes, 3 both, 4 slopes under a causal mask
hipError_t launch_paged_tiles(const PagedArgs& a, int d, int form, hipStream_t stream);
hipError_t launch_paged_tiles_d64(const PagedArgs& a, int form, hipStream_t stream);
hipError_t launch_paged_tiles_d128(const PagedArgs& a, int form, hipStream_t stream);

}  // namespace attn
