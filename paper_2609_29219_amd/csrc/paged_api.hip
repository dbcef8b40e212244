// C entry points of the paged cache's operators: argument checks, launch sizes, workspace.
#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "host.h"
#include "paged.h"
#include "paged_plan.h"

using namespace attn;

namespace {

constexpr int kPagedMost = 1 << 30;  // tokens of a call or of a request, requests

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// log2 of the page size, or an error
int page_log2(int page_size, int* out) {
    int log2 = kPagedMinPageLog2;
    while (log2 < kPagedMaxPageLog2 && (1 << log2) != page_size) ++log2;
    if ((1 << log2) != page_size)
        return host::fail(ATTN_EUNSUPPORTED, "page size %d is no power of two from %d to %d",
                          page_size, 1 << kPagedMinPageLog2, 1 << kPagedMaxPageLog2);
    *out = log2;
    return ATTN_OK;
}

int validate_table(const int* table, long long stride, int R, int max_pages, int page_size) {
    if (!table || !aligned(table, 4))
        return host::fail(ATTN_EINVAL, "block table: null or misaligned pointer");
    if (R <= 0 || max_pages <= 0)
        return host::fail(ATTN_EINVAL, "dimensions must be positive (R=%d max_pages=%d)", R,
                          max_pages);
    if (R > 1 && (stride < max_pages || stride > (1LL << 56) / R))
        return host::fail(ATTN_EINVAL, "block table: stride %lld of rows of %d", stride, max_pages);
    if ((long long)max_pages * page_size > kPagedMost)
        return host::fail(ATTN_EUNSUPPORTED, "a table row of %d pages holds more than 2^30 tokens",
                          max_pages);
    if (R > kPagedMost) return host::fail(ATTN_EUNSUPPORTED, "more than 2^30 requests");
    return ATTN_OK;
}

int validate_ints(const void* p, const char* name) {
    if (!p || !aligned(p, 4))
        return host::fail(ATTN_EINVAL, "%s: null or misaligned pointer", name);
    return ATTN_OK;
}

// The pages of one side of the cache.
int validate_pages(const attn_heads* p, const char* name, int n_pages, int page_size, int Hkv,
                   int d, bool written) {
    int rc = host::check_heads(p, name, n_pages, page_size, Hkv, d, written);
    if (rc) return rc;
    // (offsets inside eight rows, and strides in steps of 16 bytes, are 32-bit)
    if (p->row_stride > (1LL << 26) || (n_pages > 1 && p->batch_stride / 8 > UINT32_MAX))
        return host::fail(ATTN_EUNSUPPORTED, "%s: rows %lld or pages %lld values apart", name,
                          p->row_stride, p->batch_stride);
    return ATTN_OK;
}

int validate_cache_dims(int T, int Hkv, int d, int n_pages, int page_size) {
    if (T <= 0 || Hkv <= 0 || d <= 0 || n_pages <= 0)
        return host::fail(ATTN_EINVAL,
                          "dimensions must be positive (T=%d Hkv=%d d=%d n_pages=%d)", T, Hkv, d,
                          n_pages);
    if (d != 64 && d != 128)
        return host::fail(ATTN_EUNSUPPORTED, "head dim %d not in {64, 128}", d);
    if ((long long)n_pages * page_size > INT_MAX)
        return host::fail(ATTN_EUNSUPPORTED, "a cache of more than 2^31 - 1 rows");
    return ATTN_OK;
}

int validate_paged_dims(int T, int R, int Hq, int Hkv, int d, int max_q) {
    if (T <= 0 || R <= 0 || Hq <= 0 || d <= 0)
        return host::fail(ATTN_EINVAL, "dimensions must be positive (T=%d R=%d Hq=%d d=%d)", T, R,
                          Hq, d);
    if (Hkv <= 0 || Hq % Hkv != 0)
        return host::fail(ATTN_EINVAL, "Hkv (%d) must be positive and divide Hq (%d)", Hkv, Hq);
    if (d != 64 && d != 128)
        return host::fail(ATTN_EUNSUPPORTED, "head dim %d not in {64, 128}", d);
    if (max_q < 0) return host::fail(ATTN_EINVAL, "max_q (%d) must not be negative", max_q);
    // (the tile kernel numbers rows, those that fill up a request's last block too, in 32 bits)
    if ((long long)T * Hq > INT_MAX - kPagedTileRows)
        return host::fail(ATTN_EUNSUPPORTED, "more than 2^31 - 257 query rows");
    if (T > kPagedMost) return host::fail(ATTN_EUNSUPPORTED, "more than 2^30 tokens");
    if (Hq / Hkv > kPagedMaxGroup)
        return host::fail(ATTN_EUNSUPPORTED, "more than %d query heads to a key/value head",
                          kPagedMaxGroup);
    return ATTN_OK;
}

}  // namespace

extern "C" {

int attn_paged_extend(int* block_table, long long table_stride, const int* seq_lens,
                      const int* new_lens, const int* free_pages, int list_len, const int* n_free,
                      int* slots, int* positions, int* cu_seqlens, int* kv_lens, int* n_left,
                      int R, int max_pages, int page_size, int T) {
    return host::guarded([&]() -> int {
        ExtendArgs a{};
        int rc = page_log2(page_size, &a.page_log2);
        if (!rc) rc = validate_table(block_table, table_stride, R, max_pages, page_size);
        const std::pair<const void*, const char*> ints[] = {
            {seq_lens, "seq_lens"}, {new_lens, "new_lens"}, {free_pages, "free_pages"},
            {n_free, "n_free"}, {slots, "slots"}, {positions, "positions"},
            {cu_seqlens, "cu_seqlens"}, {kv_lens, "kv_lens"}, {n_left, "n_left"}};
        for (const auto& x : ints)
            if (!rc) rc = validate_ints(x.first, x.second);
        if (!rc && (T <= 0 || list_len <= 0))
            rc = host::fail(ATTN_EINVAL, "dimensions must be positive (T=%d list_len=%d)", T,
                            list_len);
        if (!rc && T > kPagedMost) rc = host::fail(ATTN_EUNSUPPORTED, "more than 2^30 tokens");
        if (rc) return rc;
        const Rows results[] = {
            host::plain_rows("block_table", block_table, 4, max_pages, table_stride, R),
            host::plain_rows("slots", slots, 4, T), host::plain_rows("positions", positions, 4, T),
            host::plain_rows("cu_seqlens", cu_seqlens, 4, R + 1LL),
            host::plain_rows("kv_lens", kv_lens, 4, R), host::plain_rows("n_left", n_left, 4, 1)};
        const Rows operands[] = {
            host::plain_rows("seq_lens", seq_lens, 4, R),
            host::plain_rows("new_lens", new_lens, 4, R),
            host::plain_rows("free_pages", free_pages, 4, list_len),
            host::plain_rows("n_free", n_free, 4, 1)};
        rc = host::check_apart(results, 6, operands, 4);
        if (rc) return rc;
        host::DeviceRef dev;
        rc = host::device(&dev);
        if (rc) return rc;
        a.table = block_table;
        a.table_stride = table_stride;
        a.seq_lens = seq_lens;
        a.new_lens = new_lens;
        a.free_pages = free_pages;
        a.n_free = n_free;
        a.slots = slots;
        a.positions = positions;
        a.cu = cu_seqlens;
        a.kv_lens = kv_lens;
        a.n_left = n_left;
        a.R = R;
        a.T = T;
        a.max_pages = max_pages;
        a.n_list = list_len;
        const hipError_t e = launch_paged_extend(a, host::stream());
        return e == hipSuccess ? ATTN_OK : host::fail_hip(e, "paged extend launch");
    });
}

int attn_paged_release(const int* block_table, long long table_stride, const int* seq_lens,
                       const int* keep_lens, int* free_pages, int list_len, const int* n_free,
                       int* n_left, int R, int max_pages, int page_size) {
    return host::guarded([&]() -> int {
        ReleaseArgs a{};
        int rc = page_log2(page_size, &a.page_log2);
        if (!rc) rc = validate_table(block_table, table_stride, R, max_pages, page_size);
        const std::pair<const void*, const char*> ints[] = {
            {seq_lens, "seq_lens"}, {keep_lens, "keep_lens"}, {free_pages, "free_pages"},
            {n_free, "n_free"}, {n_left, "n_left"}};
        for (const auto& x : ints)
            if (!rc) rc = validate_ints(x.first, x.second);
        if (!rc && list_len <= 0)
            rc = host::fail(ATTN_EINVAL, "dimensions must be positive (list_len=%d)", list_len);
        if (rc) return rc;
        const Rows results[] = {host::plain_rows("free_pages", free_pages, 4, list_len),
                                host::plain_rows("n_left", n_left, 4, 1)};
        const Rows operands[] = {
            host::plain_rows("block_table", block_table, 4, max_pages, table_stride, R),
            host::plain_rows("seq_lens", seq_lens, 4, R),
            host::plain_rows("keep_lens", keep_lens, 4, R),
            host::plain_rows("n_free", n_free, 4, 1)};
        rc = host::check_apart(results, 2, operands, 4);
        if (rc) return rc;
        host::DeviceRef dev;
        rc = host::device(&dev);
        if (rc) return rc;
        a.table = block_table;
        a.table_stride = table_stride;
        a.seq_lens = seq_lens;
        a.keep_lens = keep_lens;
        a.n_free = n_free;
        a.free_pages = free_pages;
        a.n_left = n_left;
        a.R = R;
        a.max_pages = max_pages;
        a.n_list = list_len;
        const hipError_t e = launch_paged_release(a, host::stream());
        return e == hipSuccess ? ATTN_OK : host::fail_hip(e, "paged release launch");
    });
}

int attn_paged_store(const attn_heads* k, const attn_heads* v, const int* slots,
                     const attn_heads* k_pages, const attn_heads* v_pages, int T, int Hkv, int d,
                     int n_pages, int page_size) {
    return host::guarded([&]() -> int {
        StoreArgs a{};
        int rc = page_log2(page_size, &a.page_log2);
        if (!rc) rc = validate_cache_dims(T, Hkv, d, n_pages, page_size);
        if (!rc) rc = host::check_heads(k, "k", 1, T, Hkv, d, false);
        if (!rc) rc = host::check_heads(v, "v", 1, T, Hkv, d, false);
        if (!rc) rc = validate_pages(k_pages, "k_pages", n_pages, page_size, Hkv, d, true);
        if (!rc) rc = validate_pages(v_pages, "v_pages", n_pages, page_size, Hkv, d, true);
        if (!rc) rc = validate_ints(slots, "slots");
        if (!rc && (long long)T * Hkv > INT_MAX)
            rc = host::fail(ATTN_EUNSUPPORTED, "more than 2^31 - 1 rows");
        if (rc) return rc;
        const Rows results[] = {
            host::heads_rows("k_pages", *k_pages, n_pages, page_size, Hkv, d, 2),
            host::heads_rows("v_pages", *v_pages, n_pages, page_size, Hkv, d, 2)};
        const Rows operands[] = {host::heads_rows("k", *k, 1, T, Hkv, d, 2),
                                 host::heads_rows("v", *v, 1, T, Hkv, d, 2),
                                 host::plain_rows("slots", slots, 4, T)};
        rc = host::check_apart(results, 2, operands, 3);
        if (rc) return rc;
        host::DeviceRef dev;
        rc = host::device(&dev);
        if (rc) return rc;
        a.k = *k;
        a.v = *v;
        a.k_pages = *k_pages;
        a.v_pages = *v_pages;
        a.slots = slots;
        a.T = T;
        a.Hkv = Hkv;
        a.n_pages = n_pages;
        const hipError_t e = launch_paged_store(a, d, host::stream());
        return e == hipSuccess ? ATTN_OK : host::fail_hip(e, "paged store launch");
    });
}

long long attn_paged_workspace_bytes(int T, int R, int max_q, int Hq, int Hkv, int d,
                                     int page_size, int max_pages, int window) {
    return host::guarded([&]() -> long long {
        int log2 = 0;
        int rc = page_log2(page_size, &log2);
        if (!rc) rc = validate_paged_dims(T, R, Hq, Hkv, d, max_q);
        if (!rc && (max_pages <= 0 || window < 0))
            rc = host::fail(ATTN_EINVAL, "max_pages (%d) must be positive, window (%d) not negative",
                            max_pages, window);
        if (rc) return rc;
        host::DeviceRef dev;
        rc = host::device(&dev);
        if (rc) return rc;
        const long long max_keys = (long long)max_pages << log2;
        return (long long)paged_launch(T, R, Hq, Hkv, d, max_q, max_keys,
                                       window >= max_keys ? 0 : window, dev.desc->num_cus)
            .bytes(d);
    });
}

int attn_paged(const attn_heads* q, const attn_heads* k_pages, const attn_heads* v_pages, void* o,
               float* lse, const int* block_table, long long table_stride, const int* kv_lens,
               const int* cu_seqlens, const float* slopes, int T, int R, int max_q, int Hq,
               int Hkv, int d, int n_pages, int page_size, int max_pages, float scale,
               float softcap, int window, int causal, int flags, void* workspace,
               size_t workspace_bytes) {
    return host::guarded([&]() -> int {
        PagedArgs a{};
        int rc = page_log2(page_size, &a.page_log2);
        if (!rc) rc = validate_paged_dims(T, R, Hq, Hkv, d, max_q);
        if (!rc) rc = validate_cache_dims(T, Hkv, d, n_pages, page_size);
        if (!rc) rc = validate_table(block_table, table_stride, R, max_pages, page_size);
        if (!rc) rc = host::check_heads(q, "q", 1, T, Hq, d, false);
        if (!rc) rc = validate_pages(k_pages, "k_pages", n_pages, page_size, Hkv, d, false);
        if (!rc) rc = validate_pages(v_pages, "v_pages", n_pages, page_size, Hkv, d, false);
        if (!rc) rc = validate_ints(kv_lens, "kv_lens");
        if (rc) return rc;
        if (!o || !aligned(o, 16)) return host::fail(ATTN_EINVAL, "o: null or misaligned pointer");
        if (!aligned(lse, 4) || !aligned(cu_seqlens, 4) || !aligned(slopes, 4))
            return host::fail(ATTN_EINVAL, "lse, cu_seqlens or slopes misaligned");
        if (!cu_seqlens && T != R)
            return host::fail(ATTN_EINVAL, "%d tokens of %d requests without cu_seqlens", T, R);
        if (flags & ~ATTN_OUT_BF16) return host::fail(ATTN_EINVAL, "unknown flags 0x%x", flags);
        if (!isfinite(scale)) return host::fail(ATTN_EINVAL, "scale must be finite");
        if (!(softcap >= 0.f) || !isfinite(softcap))
            return host::fail(ATTN_EINVAL, "softcap must be finite and not negative");
        if (window < 0) return host::fail(ATTN_EINVAL, "window must not be negative");
        if (window && !causal)
            return host::fail(ATTN_EUNSUPPORTED, "a window needs the causal mask");
        // (a window of all that a table's row holds hides nothing)
        const long long max_keys = (long long)max_pages * page_size;
        if (window >= max_keys) window = 0;
        Rows results[3], operands[7];
        results[0] = host::plain_rows("o", o, (flags & ATTN_OUT_BF16) ? 2 : 4, (long long)T * Hq * d);
        int n_results = 1, n_operands = 0;
        if (lse) results[n_results++] = host::plain_rows("lse", lse, 4, (long long)T * Hq);
        operands[n_operands++] = host::heads_rows("q", *q, 1, T, Hq, d, 2);
        operands[n_operands++] = host::heads_rows("k_pages", *k_pages, n_pages, page_size, Hkv, d, 2);
        operands[n_operands++] = host::heads_rows("v_pages", *v_pages, n_pages, page_size, Hkv, d, 2);
        operands[n_operands++] =
            host::plain_rows("block_table", block_table, 4, max_pages, table_stride, R);
        operands[n_operands++] = host::plain_rows("kv_lens", kv_lens, 4, R);
        if (cu_seqlens) operands[n_operands++] = host::plain_rows("cu_seqlens", cu_seqlens, 4, R + 1LL);
        if (slopes) operands[n_operands++] = host::plain_rows("slopes", slopes, 4, Hq);
        host::DeviceRef dev;
        rc = host::check_apart(results, n_results, operands, n_operands);
        if (!rc) rc = host::device(&dev);
        if (rc) return rc;
        PagedLaunch l = paged_launch(T, R, Hq, Hkv, d, max_q, max_keys, window,
                                     dev.desc->num_cus);
        const size_t need = l.bytes(d);
        if (l.items * l.splits * 2 > kMaxWorkgroups)
            return host::fail(ATTN_EUNSUPPORTED, "more workgroups than one launch holds");
        if (workspace) {
            results[n_results] = host::plain_rows("workspace", workspace, 1, (long long)need);
            rc = host::check_apart(results, n_results + 1, operands, n_operands);
            if (rc) return rc;
        }
        void* ws = nullptr;
        std::unique_lock<std::mutex> ws_lock;  // held until the kernels are enqueued
        rc = host::workspace(dev, need, workspace, workspace_bytes, &ws_lock, &ws);
        if (rc == ATTN_ENOMEM)
            l.unsplit();  // without memory for the parts
        else if (rc)
            return rc;
        a.q = static_cast<const uint16_t*>(q->ptr);
        a.q_row = q->row_stride;
        a.q_head = q->head_stride;
        auto side = [](const attn_heads& p, int n_pages) {
            // (a single page's stride is any number)
            return PagedSide{static_cast<const uint16_t*>(p.ptr),
                             n_pages > 1 ? (uint32_t)(p.batch_stride / 8) : 0,
                             (uint32_t)(p.row_stride / 8), p.head_stride};
        };
        a.k = side(*k_pages, n_pages);
        a.v = side(*v_pages, n_pages);
        a.o = o;
        a.lse = lse;
        a.table = block_table;
        a.table_stride = table_stride;
        a.kv_lens = kv_lens;
        a.cu = cu_seqlens;
        a.slopes = slopes;
        a.T = T;
        a.R = R;
        a.Hq = Hq;
        a.Hkv = Hkv;
        a.group = Hq / Hkv;
        a.group_inverse = (uint32_t)(((1ULL << 32) + a.group - 1) / a.group);
        a.n_pages = n_pages;
        a.max_pages = max_pages;
        a.causal = causal ? 1 : 0;
        a.window = window;
        a.out_bf16 = (flags & ATTN_OUT_BF16) ? 1 : 0;
        a.few = l.few;
        // softmax in base 2; a negative scale flips Q's signs (exact), and a zero one becomes the
        // smallest normal float, with which all weights are equal
        const double log2e = 1.4426950408889634;
        const double s = std::max(fabs((double)scale) * log2e, (double)FLT_MIN);
        a.scale_log2 = (float)s;
        a.q_sign = scale < 0.f ? 0x80008000u : 0u;
        if (softcap > 0.f) {
            a.cap_in = (float)std::min(2.0 * s / softcap, (double)FLT_MAX);
            a.cap_out = (float)std::min(softcap * log2e, (double)FLT_MAX);
        }
        float* f = static_cast<float*>(ws);
        a.ws_o = f;
        a.tile_o = f += l.row_parts() * d;
        a.ws_m = f += l.tile_parts() * d;
        a.ws_l = f += l.row_parts();
        a.tile_m = f += l.row_parts();
        a.tile_l = f += l.tile_parts();
        int* const meta = reinterpret_cast<int*>(f += l.tile_parts());
        a.meta = l.shared ? meta : nullptr;
        a.tile_meta = meta + l.n_wg * kPagedMeta;
        a.n_wg = l.n_wg;
        a.unit_log2 = l.unit_log2;
        a.splits = l.splits;
        a.tile_wgs = l.items * l.splits;
        hipError_t e = hipSuccess;
        if (l.n_wg) e = launch_paged_rows(a, d, l.block, l.waves, host::stream());
        if (e == hipSuccess && l.items)
            e = launch_paged_tiles(a, d,
                                   softcap > 0.f                  ? (slopes ? 3 : 1)
                                   : !slopes                      ? 0
                                   : causal && a.scale_log2 > 1e-6f ? 4  // (slopes over it)
                                                                  : 2,
                                   host::stream());
        if (e == hipSuccess)
            e = launch_paged_sums(a, d, l.block, host::stream());
        return e == hipSuccess ? ATTN_OK : host::fail_hip(e, "paged attention launch");
    });
}

// The calls as the Python binding makes them: one pointer to all operands, and the stream
// (the thread's from then on), since a foreign-function call costs its caller time for
// every argument.
struct PackedExtend {
    int* block_table;
    long long table_stride;
    const int *seq_lens, *new_lens, *free_pages, *n_free;
    int *slots, *positions, *cu_seqlens, *kv_lens, *n_left;
    hipStream_t stream;
    int list_len, R, max_pages, page_size, T;
};
static_assert(offsetof(PackedExtend, T) == 12 * 8 + 4 * 4, "QqQQQQQQQQQQ5i");
int attn__paged_extend_packed(const PackedExtend* c) {
    attn_set_stream(c->stream);
    return attn_paged_extend(c->block_table, c->table_stride, c->seq_lens, c->new_lens,
                             c->free_pages, c->list_len, c->n_free, c->slots, c->positions,
                             c->cu_seqlens, c->kv_lens, c->n_left, c->R, c->max_pages,
                             c->page_size, c->T);
}

struct PackedRelease {
    const int* block_table;
    long long table_stride;
    const int *seq_lens, *keep_lens;
    int* free_pages;
    const int* n_free;
    int* n_left;
    hipStream_t stream;
    int list_len, R, max_pages, page_size;
};
static_assert(offsetof(PackedRelease, page_size) == 8 * 8 + 3 * 4, "QqQQQQQQ4i");
int attn__paged_release_packed(const PackedRelease* c) {
    attn_set_stream(c->stream);
    return attn_paged_release(c->block_table, c->table_stride, c->seq_lens, c->keep_lens,
                              c->free_pages, c->list_len, c->n_free, c->n_left, c->R,
                              c->max_pages, c->page_size);
}

struct PackedStore {
    attn_heads k, v, k_pages, v_pages;
    const int* slots;
    hipStream_t stream;
    int T, Hkv, d, n_pages, page_size;
};
static_assert(offsetof(PackedStore, page_size) == 18 * 8 + 4 * 4, "16qQQ5i");
int attn__paged_store_packed(const PackedStore* c) {
    attn_set_stream(c->stream);
    return attn_paged_store(&c->k, &c->v, c->slots, &c->k_pages, &c->v_pages, c->T, c->Hkv, c->d,
                            c->n_pages, c->page_size);
}

struct PackedPaged {
    attn_heads q, k_pages, v_pages;
    void* o;
    float* lse;
    const int* block_table;
    long long table_stride;
    const int *kv_lens, *cu_seqlens;
    const float* slopes;
    void* workspace;
    size_t workspace_bytes;
    hipStream_t stream;
    int T, R, max_q, Hq, Hkv, d, n_pages, page_size, max_pages, window, causal, flags;
    float scale, softcap;
};
static_assert(offsetof(PackedPaged, softcap) == 22 * 8 + 13 * 4, "12q3Qq6Q12i2f");
int attn__paged_packed(const PackedPaged* c) {
    attn_set_stream(c->stream);
    return attn_paged(&c->q, &c->k_pages, &c->v_pages, c->o, c->lse, c->block_table,
                      c->table_stride, c->kv_lens, c->cu_seqlens, c->slopes, c->T, c->R, c->max_q,
                      c->Hq, c->Hkv, c->d, c->n_pages, c->page_size, c->max_pages, c->scale,
                      c->softcap, c->window, c->causal, c->flags, c->workspace,
                      c->workspace_bytes);
}

}  // extern "C"
