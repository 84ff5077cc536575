// C entry points of the 4-bit paged cache and of the page operations: argument
// validation, then launch.  Nothing is enqueued unless every check passes.
#include <algorithm>
#include <cstdlib>
#include <string>

#include "kv4.hpp"

namespace oc {

// pages of K and of V in every layer, whose byte offsets are 64-bit
static int check_pool_bytes(const oc_layout &l, int64_t page_bytes) {
    if (l.num_pages > INT64_MAX / 2 / l.num_layers / page_bytes) return fail(OC_ERANGE, "a pool of more than 2^63 bytes");
    return OC_OK;
}

int check_kv4_layout(const oc_layout &l) {
    const int rc = check_layout(l);
    if (rc) return rc;
    if (l.head_dim % 32) return fail(OC_ESHAPE, "a 4-bit pool needs a head_dim that is a multiple of 32");
    if ((int64_t)l.page_size * l.head_dim > INT32_MAX || kv4_page_bytes(l) > INT32_MAX)
        return fail(OC_ERANGE, "a 4-bit page of 2^31 bytes or more");
    return check_pool_bytes(l, kv4_page_bytes(l));
}

static Kv4Args kv4_args(const oc_kv_pool *pool, const oc_block_table *bt, int32_t layer, int64_t first, int64_t tokens) {
    const oc_layout &l = pool->layout;
    Kv4Args a{};
    a.page_bytes = kv4_page_bytes(l);
    a.code_bytes = (int32_t)kv4_code_bytes(l);
    a.pool_k = static_cast<unsigned char *>(pool->base) + (int64_t)layer * 2 * l.num_pages * a.page_bytes;
    a.pool_v = a.pool_k + l.num_pages * a.page_bytes;
    a.pages = bt->pages;
    a.first = (int32_t)first;
    a.end = (int32_t)(first + tokens);
    a.G = l.chunk_tokens;
    a.n_kv = l.num_kv_heads;
    a.d = l.head_dim;
    a.Ps = l.page_size;
    a.num_pages = pages_of(l);
    return a;
}

// the kernels' positions are 32-bit, and so is their grid (64 work-items for
// each page, half and head)
static int check_kv4_tokens(const oc_layout &l, int64_t tokens) {
    if (tokens > INT32_MAX - l.page_size) return fail(OC_ERANGE, "more than 2^31 tokens");
    if ((tokens / l.page_size + 2) * 2 > OC_MAX_GRID_ITEMS / 64 / l.num_kv_heads)
        return fail(OC_ERANGE, "more than 2^32 work-items in one launch");
    return OC_OK;
}

static int layer_ingest(const oc_staging *staging, const oc_block_table *bt, oc_kv_pool *pool, int32_t layer, void *stream) {
    clear_error();
    if (!staging || !pool) return fail(OC_EINVAL, "staging and kv_pool must not be NULL");
    const oc_layout &l = pool->layout;
    int rc = check_kv4_layout(l);
    if (rc) return rc;
    if ((rc = check_table(bt, l))) return rc;
    if (layer < 0 || layer >= l.num_layers) return fail(OC_ERANGE, "layer out of range");
    if ((rc = check_staging_shape(l, bt, staging->num_chunks, staging->per_layer_chunk_bytes))) return rc;
    if ((rc = check_kv4_tokens(l, bt->num_tokens))) return rc;
    if (bt->num_tokens == 0) return OC_OK;
    if (!staging->data || !pool->base) return fail(OC_EINVAL, "NULL data or pool base");
    if (!aligned(staging->data, 16) || !aligned(pool->base, 16))
        return fail(OC_EALIGN, "staging data and pool base must be 16-byte aligned");
    Kv4Args a = kv4_args(pool, bt, layer, 0, bt->num_tokens);
    a.k = static_cast<const uint16_t *>(staging->data);
    OC_HIP(launch_kv4_ingest(a, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

static int suffix_append(const void *k_new, const void *v_new, int64_t tokens, const oc_block_table *bt, oc_kv_pool *pool,
                         int32_t layer, void *stream) {
    clear_error();
    if (!pool) return fail(OC_EINVAL, "kv_pool must not be NULL");
    const oc_layout &l = pool->layout;
    int rc = check_kv4_layout(l);
    if (rc) return rc;
    if ((rc = check_table(bt, l))) return rc;
    if (layer < 0 || layer >= l.num_layers) return fail(OC_ERANGE, "layer out of range");
    if (tokens < 0) return fail(OC_EINVAL, "negative suffix_tokens");
    if (tokens > INT32_MAX) return fail(OC_ERANGE, "more than 2^31 tokens");
    if ((rc = check_append_table(bt, l, tokens))) return rc;
    if ((rc = check_kv4_tokens(l, bt->num_tokens + tokens))) return rc;
    if (tokens == 0) return OC_OK;
    if (!k_new || !v_new || !pool->base) return fail(OC_EINVAL, "NULL k_new, v_new or pool base");
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(pool->base, 16))
        return fail(OC_EALIGN, "k_new, v_new and pool base must be 16-byte aligned");
    Kv4Args a = kv4_args(pool, bt, layer, bt->num_tokens, tokens);
    a.k = static_cast<const uint16_t *>(k_new);
    a.v = static_cast<const uint16_t *>(v_new);
    OC_HIP(launch_kv4_append(a, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

static int layer_gather(const oc_block_table *bt, const oc_kv_pool *pool, int32_t layer, void *staging_out,
                        int64_t num_chunks, int64_t per_layer_chunk_bytes, void *stream) {
    clear_error();
    if (!pool) return fail(OC_EINVAL, "kv_pool must not be NULL");
    const oc_layout &l = pool->layout;
    int rc = check_kv4_layout(l);
    if (rc) return rc;
    if ((rc = check_table(bt, l))) return rc;
    if (layer < 0 || layer >= l.num_layers) return fail(OC_ERANGE, "layer out of range");
    if ((rc = check_staging_shape(l, bt, num_chunks, per_layer_chunk_bytes))) return rc;
    if ((rc = check_kv4_tokens(l, bt->num_tokens))) return rc;
    if (bt->num_tokens == 0) return OC_OK;
    if (!staging_out || !pool->base) return fail(OC_EINVAL, "NULL staging_out or pool base");
    if (!aligned(staging_out, 16) || !aligned(pool->base, 16))
        return fail(OC_EALIGN, "staging and pool base must be 16-byte aligned");
    Kv4Args a = kv4_args(pool, bt, layer, 0, bt->num_tokens);
    a.out = static_cast<uint16_t *>(staging_out);
    OC_HIP(launch_kv4_gather(a, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

static int check_workspace(void *workspace, size_t have, size_t need, uintptr_t alignment) {
    if (!workspace) return fail(OC_EINVAL, "NULL workspace");
    if (!aligned(workspace, alignment))
        return fail(OC_EALIGN, "workspace must be " + std::to_string(alignment) + "-byte aligned");
    if (have < need) return fail(OC_EINVAL, "workspace too small: need " + std::to_string(need) + " bytes");
    return OC_OK;
}

static Kv4AttnArgs attention_args(const void *q, const void *k_new, const void *v_new, const oc_kv_pool *pool, int32_t layer,
                                  void *out, void *workspace) {
    const oc_layout &l = pool->layout;
    Kv4AttnArgs a{};
    a.q = static_cast<const uint16_t *>(q);
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.page_bytes = kv4_page_bytes(l);
    a.code_bytes = (int32_t)kv4_code_bytes(l);
    a.pool_k = static_cast<unsigned char *>(pool->base) + (int64_t)layer * 2 * l.num_pages * a.page_bytes;
    a.pool_v = a.pool_k + l.num_pages * a.page_bytes;
    a.out = static_cast<uint16_t *>(out);
    a.ws = static_cast<unsigned char *>(workspace);
    a.num_pages = pages_of(l);
    return a;
}

static int check_rows(const void *q, const void *k_new, const void *v_new, const void *out, const oc_kv_pool *pool) {
    if (!q || !k_new || !v_new || !out) return fail(OC_EINVAL, "NULL tensor");
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(pool->base, 16))
        return fail(OC_EALIGN, "q, k_new, v_new, out and pool base must be 16-byte aligned");
    return OC_OK;
}

static int suffix_prefill(const void *q, const void *k_new, const void *v_new, int64_t tokens, const oc_kv_pool *pool,
                          const oc_block_table *bt, int32_t layer, void *out, void *workspace, size_t workspace_bytes,
                          void *stream) {
    clear_error();
    if (!pool) return fail(OC_EINVAL, "kv_pool must not be NULL");
    const oc_layout &l = pool->layout;
    int rc = check_kv4_layout(l);
    if (rc) return rc;
    if ((rc = check_table(bt, l))) return rc;
    if (layer < 0 || layer >= l.num_layers) return fail(OC_ERANGE, "layer out of range");
    if (tokens < 1) return fail(OC_EINVAL, "suffix_tokens must be >= 1");
    Kv4Plan p;
    if ((rc = plan_kv4_attention(l, bt->num_tokens, tokens, &p))) return rc;
    if (bt->num_tokens > 0 && !pool->base) return fail(OC_EINVAL, "NULL pool base");
    if ((rc = check_rows(q, k_new, v_new, out, pool))) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, p.total, 256))) return rc;
    Kv4AttnArgs a = attention_args(q, k_new, v_new, pool, layer, out, workspace);
    a.pages = bt->pages;
    OC_HIP(launch_kv4_attention(p, a, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

// tables of which `need` entries of each of `n` rows are used
static int check_tables(const oc_page_tables *t, int64_t n, int64_t need) {
    if (!t) return fail(OC_EINVAL, "tables are NULL");
    if (t->num_tables < 0 || t->num_entries < 0) return fail(OC_EINVAL, "negative table size");
    if (t->num_tables < n) return fail(OC_ERANGE, "fewer tables than requests");
    if (n > 1 && t->stride < t->num_entries) return fail(OC_EINVAL, "tables overlap: stride below num_entries");
    if (n > 0 && t->num_entries < need)
        return fail(OC_ERANGE, "each table needs " + std::to_string(need) + " entries");
    if (n > 0 && need > 0 && !t->pages) return fail(OC_EINVAL, "tables' pages pointer is NULL");
    return OC_OK;
}

static int decode(const void *q, const void *k_new, const void *v_new, int64_t batch, oc_kv_pool *pool,
                  const oc_page_tables *tables, const int32_t *num_tokens, int64_t max_tokens, int32_t layer, void *out,
                  void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    if (!pool) return fail(OC_EINVAL, "kv_pool must not be NULL");
    const oc_layout &l = pool->layout;
    int rc = check_kv4_layout(l);
    if (rc) return rc;
    if (layer < 0 || layer >= l.num_layers) return fail(OC_ERANGE, "layer out of range");
    if (batch < 0) return fail(OC_EINVAL, "negative batch");
    if (batch == 0) return OC_OK;
    Kv4Plan p;
    if ((rc = plan_kv4_decode(l, batch, max_tokens, &p))) return rc;
    // the tokens before, and the one that is appended
    if ((rc = check_tables(tables, batch, max_tokens / l.page_size + 1))) return rc;
    if (max_tokens / l.page_size + 1 > l.num_pages) return fail(OC_ERANGE, "max_tokens needs more pages than the pool has");
    if (!num_tokens || !pool->base) return fail(OC_EINVAL, "NULL num_tokens or pool base");
    if ((rc = check_rows(q, k_new, v_new, out, pool))) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, p.total, 256))) return rc;
    Kv4AttnArgs a = attention_args(q, k_new, v_new, pool, layer, out, workspace);
    a.pages = tables->pages;
    a.table_stride = tables->stride;
    a.num_tokens = num_tokens;
    a.max_tokens = (int32_t)max_tokens;
    OC_HIP(launch_kv4_attention(p, a, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

// ---- pages --------------------------------------------------------------------

static int check_pages_layout(const oc_layout &l) {
    const int rc = check_layout(l);
    if (rc) return rc;
    if (l.num_pages > INT32_MAX) return fail(OC_ERANGE, "more than 2^31 pages");
    if (l.num_layers > INT32_MAX / 2) return fail(OC_ERANGE, "more than 2^30 layers");
    return OC_OK;
}

// a pool of `bits` per value as the page kernels see it
static int pages_args(const oc_kv_pool *pool, int32_t bits, PagesArgs *a) {
    if (!pool) return fail(OC_EINVAL, "kv_pool must not be NULL");
    const oc_layout &l = pool->layout;
    int rc = check_pages_layout(l);
    if (rc) return rc;
    if (bits != 16 && bits != 4) return fail(OC_EINVAL, "bits must be 16 or 4");
    if (bits == 4 && (rc = check_kv4_layout(l))) return rc;
    if (bits == 16 && (int64_t)l.num_kv_heads * l.page_size > INT64_MAX / 2 / l.head_dim)
        return fail(OC_ERANGE, "a page of more than 2^63 bytes");
    *a = PagesArgs{};
    a->page_bytes = bits == 4 ? kv4_page_bytes(l) : (int64_t)l.num_kv_heads * l.page_size * l.head_dim * 2;
    if ((rc = check_pool_bytes(l, a->page_bytes))) return rc;
    a->pool = static_cast<unsigned char *>(pool->base);
    a->regions = 2 * l.num_layers;
    a->num_pages = (int32_t)l.num_pages;
    return OC_OK;
}

static int check_pool_base(const oc_kv_pool *pool) {
    if (!pool->base) return fail(OC_EINVAL, "NULL pool base");
    return aligned(pool->base, 16) ? OC_OK : fail(OC_EALIGN, "pool base must be 16-byte aligned");
}

static int pages_take(const oc_layout *layout, int32_t *counts, int64_t n, int32_t *out, int32_t *status, void *stream) {
    clear_error();
    if (!layout) return fail(OC_EINVAL, "layout is NULL");
    const int rc = check_pages_layout(*layout);
    if (rc) return rc;
    if (n < 0) return fail(OC_EINVAL, "negative number of pages");
    if (n > layout->num_pages) return fail(OC_ERANGE, "more pages than the pool has");
    if (!counts || !status || (n > 0 && !out)) return fail(OC_EINVAL, "NULL page_counts, pages_out or status");
    PagesArgs a{};
    a.num_pages = (int32_t)layout->num_pages;
    a.counts = counts;
    a.status = status;
    OC_HIP(launch_pages_take(a, (int32_t)n, out, 1, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

static int pages_copy(oc_kv_pool *pool, int32_t bits, const int32_t *src, const int32_t *dst, int64_t n, void *stream) {
    clear_error();
    PagesArgs a;
    int rc = pages_args(pool, bits, &a);
    if (rc) return rc;
    if (n < 0) return fail(OC_EINVAL, "negative number of pages");
    if (n > pool->layout.num_pages) return fail(OC_ERANGE, "more pages than the pool has");
    if (n == 0) return OC_OK;
    if (!src || !dst) return fail(OC_EINVAL, "NULL src_pages or dst_pages");
    if ((rc = check_pool_base(pool))) return rc;
    OC_HIP(launch_pages_copy(a, src, dst, (int32_t)n, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

// Do the first `need` entries of `pages` meet those of one of the n tables?  (n, need > 0)
static bool overlaps(const int32_t *pages, const oc_page_tables &t, int64_t n, int64_t need) {
    const int64_t off = (int64_t)((intptr_t)pages - (intptr_t)t.pages) / 4;
    if (off <= -need) return false;
    // the table that begins at or before `pages`, and the next
    const int64_t c = n > 1 ? std::max<int64_t>(0, std::min(off / t.stride, n - 1)) : 0;
    return std::abs(off - c * t.stride) < need || (c + 1 < n && (c + 1) * t.stride - off < need);
}

static int pages_fork(oc_kv_pool *pool, int32_t bits, const oc_block_table *parent, const oc_page_tables *children,
                      int64_t n, int32_t *counts, int32_t *status, void *stream) {
    clear_error();
    PagesArgs a;
    int rc = pages_args(pool, bits, &a);
    if (rc) return rc;
    const oc_layout &l = pool->layout;
    if ((rc = check_table(parent, l))) return rc;
    if (n < 0) return fail(OC_EINVAL, "negative number of children");
    if (n > INT32_MAX) return fail(OC_ERANGE, "more than 2^31 children");
    const int64_t need = (parent->num_tokens + l.page_size - 1) / l.page_size;
    if ((rc = check_tables(children, n, need))) return rc;
    if (!counts || !status) return fail(OC_EINVAL, "NULL page_counts or status");
    if (need > 0 && n > 0 && (rc = check_pool_base(pool))) return rc;
    if (need > 0 && n > 0 && overlaps(parent->pages, *children, n, need))
        return fail(OC_EINVAL, "the parent's table is among the children's");
    a.counts = counts;
    a.status = status;
    const bool part = n > 0 && parent->num_tokens % l.page_size != 0;
    const int64_t full = n > 0 ? parent->num_tokens / l.page_size : 0;
    OC_HIP(launch_pages_fork(a, parent->pages, (int32_t)full, part, (int32_t)n, children->pages, children->stride,
                             static_cast<hipStream_t>(stream)));
    return OC_OK;
}

static int pages_release(const oc_block_table *bt, const oc_layout *layout, int32_t *counts, void *stream) {
    clear_error();
    if (!layout) return fail(OC_EINVAL, "layout is NULL");
    int rc = check_pages_layout(*layout);
    if (rc) return rc;
    if ((rc = check_table(bt, *layout))) return rc;
    if (bt->num_tokens == 0) return OC_OK;
    if (!counts) return fail(OC_EINVAL, "NULL page_counts");
    PagesArgs a{};
    a.num_pages = (int32_t)layout->num_pages;
    a.counts = counts;
    const int64_t n = (bt->num_tokens + layout->page_size - 1) / layout->page_size;
    OC_HIP(launch_pages_release(a, bt->pages, (int32_t)n, static_cast<hipStream_t>(stream)));
    return OC_OK;
}

static int pages_compact(oc_kv_pool *pool, int32_t bits, int32_t *counts, const oc_page_tables *tables, int32_t *num_live,
                         void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    PagesArgs a;
    int rc = pages_args(pool, bits, &a);
    if (rc) return rc;
    if (!tables) return fail(OC_EINVAL, "tables are NULL");
    if ((rc = check_tables(tables, tables->num_tables, 0))) return rc;
    const bool any = tables->num_tables > 0 && tables->num_entries > 0;
    if (any && !tables->pages) return fail(OC_EINVAL, "tables' pages pointer is NULL");
    if (tables->num_tables > INT32_MAX || tables->num_entries > INT32_MAX) return fail(OC_ERANGE, "tables of 2^31 entries");
    if (!counts || !num_live) return fail(OC_EINVAL, "NULL page_counts or num_live");
    if ((rc = check_pool_base(pool))) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(pool->layout.num_pages), 16))) return rc;
    a.counts = counts;
    OC_HIP(launch_pages_compact(a, tables->pages, any ? (int32_t)tables->num_tables : 0, (int32_t)tables->num_entries,
                                tables->stride, num_live, static_cast<int32_t *>(workspace), static_cast<hipStream_t>(stream)));
    return OC_OK;
}

// What a size function returns: 0 where the layout or sizes are refused.
template <class F>
static size_t bytes_of(const oc_layout *layout, F &&body) noexcept {
    size_t n = 0;
    const int rc = guarded([&]() -> int {
        clear_error();
        return layout ? body(&n) : fail(OC_EINVAL, "layout is NULL");
    });
    return rc ? 0 : n;
}

}  // namespace oc

using namespace oc;

extern "C" {

size_t oc_kv4_pool_bytes(const oc_layout *layout) {
    return bytes_of(layout, [&](size_t *n) {
        const int rc = check_kv4_layout(*layout);
        *n = rc ? 0 : (size_t)(2 * layout->num_layers * layout->num_pages * kv4_page_bytes(*layout));
        return rc;
    });
}

int oc_kv4_layer_ingest(const oc_staging *staging, const oc_block_table *block_table, oc_kv_pool *kv_pool, int32_t layer,
                        void *stream) {
    return guarded([&] { return layer_ingest(staging, block_table, kv_pool, layer, stream); });
}

int oc_kv4_suffix_append(const void *k_new, const void *v_new, int64_t suffix_tokens, const oc_block_table *block_table,
                         oc_kv_pool *kv_pool, int32_t layer, void *stream) {
    return guarded([&] { return suffix_append(k_new, v_new, suffix_tokens, block_table, kv_pool, layer, stream); });
}

int oc_kv4_layer_gather(const oc_block_table *block_table, const oc_kv_pool *kv_pool, int32_t layer, void *staging_out,
                        int64_t num_chunks, int64_t per_layer_chunk_bytes, void *stream) {
    return guarded([&] {
        return layer_gather(block_table, kv_pool, layer, staging_out, num_chunks, per_layer_chunk_bytes, stream);
    });
}

size_t oc_kv4_attention_workspace_bytes(const oc_layout *layout, int64_t prefix_tokens, int64_t suffix_tokens) {
    return bytes_of(layout, [&](size_t *n) {
        Kv4Plan p;
        const int rc = plan_kv4_attention(*layout, prefix_tokens, suffix_tokens, &p);
        *n = rc ? 0 : p.total;
        return rc;
    });
}

int oc_kv4_suffix_prefill_layer(const void *q, const void *k_new, const void *v_new, int64_t suffix_tokens,
                                const oc_kv_pool *kv_pool, const oc_block_table *block_table, int32_t layer, void *out,
                                void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&] {
        return suffix_prefill(q, k_new, v_new, suffix_tokens, kv_pool, block_table, layer, out, workspace, workspace_bytes,
                              stream);
    });
}

size_t oc_kv4_decode_workspace_bytes(const oc_layout *layout, int64_t batch, int64_t max_tokens) {
    return bytes_of(layout, [&](size_t *n) {
        Kv4Plan p;
        const int rc = plan_kv4_decode(*layout, batch, max_tokens, &p);
        *n = rc ? 0 : p.total;
        return rc;
    });
}

int oc_kv4_decode_layer(const void *q, const void *k_new, const void *v_new, int64_t batch, oc_kv_pool *kv_pool,
                        const oc_page_tables *tables, const int32_t *num_tokens, int64_t max_tokens, int32_t layer,
                        void *out, void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&] {
        return decode(q, k_new, v_new, batch, kv_pool, tables, num_tokens, max_tokens, layer, out, workspace,
                      workspace_bytes, stream);
    });
}

int oc_kv_pages_take(const oc_layout *layout, int32_t *page_counts, int64_t n, int32_t *pages_out, int32_t *status,
                     void *stream) {
    return guarded([&] { return pages_take(layout, page_counts, n, pages_out, status, stream); });
}

int oc_kv_pages_copy(oc_kv_pool *kv_pool, int32_t bits, const int32_t *src_pages, const int32_t *dst_pages, int64_t n,
                     void *stream) {
    return guarded([&] { return pages_copy(kv_pool, bits, src_pages, dst_pages, n, stream); });
}

int oc_kv_pages_fork(oc_kv_pool *kv_pool, int32_t bits, const oc_block_table *parent, const oc_page_tables *children,
                     int64_t num_children, int32_t *page_counts, int32_t *status, void *stream) {
    return guarded([&] { return pages_fork(kv_pool, bits, parent, children, num_children, page_counts, status, stream); });
}

int oc_kv_pages_release(const oc_block_table *block_table, const oc_layout *layout, int32_t *page_counts, void *stream) {
    return guarded([&] { return pages_release(block_table, layout, page_counts, stream); });
}

size_t oc_kv_pages_workspace_bytes(const oc_layout *layout) {
    return bytes_of(layout, [&](size_t *n) {
        const int rc = check_pages_layout(*layout);
        *n = rc ? 0 : pages_workspace_bytes(layout->num_pages);
        return rc;
    });
}

int oc_kv_pages_compact(oc_kv_pool *kv_pool, int32_t bits, int32_t *page_counts, const oc_page_tables *tables,
                        int32_t *num_live, void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&] {
        return pages_compact(kv_pool, bits, page_counts, tables, num_live, workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
