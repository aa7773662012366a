// C ABI of the cache in pages: argument checks and launches.  All checks run before the first launch; nothing here allocates,
// frees or synchronises.
#include "psa_internal.h"

namespace psa {

static bool off_by(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
constexpr int64_t kMostGroups = (1 << 24) - 1;         // work-groups of 256 threads: a launch has fewer than 2^32 threads
constexpr int kMostKeys = 1 << 28, kMostSequences = 1 << 20;

static bool good_pages(int32_t n_pages, int32_t page_rows, int32_t max_pages)
{
    return n_pages >= 1 && n_pages <= (1 << 28) && page_rows >= 1 && page_rows <= (1 << 16) && (page_rows & (page_rows - 1)) == 0 && max_pages >= 1 &&
           (int64_t)max_pages * page_rows <= kMostKeys;
}
static int check_shape(const psa_paged_shape_t& s, bool attention)
{
    if (s.dtype != PSA_F32 && s.dtype != PSA_BF16) return PSA_ERR_DTYPE;
    if (s.B < 1 || s.B > kMostSequences || s.H_kv < 1 || s.H_kv > 65535 || s.T < 1 || s.T > (1 << 28) || s.D != kD) return PSA_ERR_SHAPE;
    if (!attention) return append_groups(s) > kMostGroups ? PSA_ERR_SHAPE : PSA_OK;
    if (s.H < 1 || s.H > 65535 || s.H % s.H_kv != 0 || (int64_t)s.T * (s.H / s.H_kv) > INT32_MAX - 65536) return PSA_ERR_SHAPE;
    // (the kernels hold scale * log2(e) in float32: 0 there would make NaN of a masked score)
    if ((s.causal != 0 && s.causal != 1) || !(s.scale >= 1e-30) || !(s.scale <= 1e30)) return PSA_ERR_ARG;
    return PSA_OK;
}
// What can be said of a cache without its tensors
static int check_cache_shape(const psa_cache_t& c, const psa_paged_shape_t& s)
{
    if (!good_pages(c.n_pages, c.page_rows, c.max_pages)) return PSA_ERR_SHAPE;
    if (c.format != PSA_CACHE_PLAIN && c.format != PSA_CACHE_MX) return PSA_ERR_ARG;
    if ((int64_t)s.B * c.max_pages > (1 << 30)) return PSA_ERR_SHAPE;
    return PSA_OK;
}
static int check_cache(const psa_cache_t& c, const psa_paged_shape_t& s, bool written)
{
    const bool mx = c.format == PSA_CACHE_MX;
    for (const psa_heads_t* t : {&c.K, &c.V}) {
        const int rc = check_heads(*t, mx ? 16 : s.dtype == PSA_F32 ? 4 : 8, 64, 16, c.n_pages, s.H_kv, c.page_rows, written);
        if (rc != PSA_OK) return rc;
    }
    if (mx) {
        for (const psa_heads_t* t : {&c.K_scales, &c.V_scales}) {
            const int rc = check_heads(*t, 2, 2, 2, c.n_pages, s.H_kv, c.page_rows, written);
            if (rc != PSA_OK) return rc;
        }
    }
    if (off_by(c.table, 4) || off_by(c.lengths, 4)) return PSA_ERR_ALIGN;
    return PSA_OK;
}
static bool has_data(const psa_heads_t* t) { return t && t->data; }
static bool has_tensors(const psa_cache_t* c)
{
    return c && c->K.data && c->V.data && c->table && c->lengths && (c->format != PSA_CACHE_MX || (c->K_scales.data && c->V_scales.data));
}
static int check_rows(const psa_paged_shape_t& s, const int32_t* offsets)
{
    if (!offsets && s.T % s.B != 0) return PSA_ERR_SHAPE;
    return off_by(offsets, 4) ? PSA_ERR_ALIGN : PSA_OK;
}
static int check_attention(const psa_cache_t& c, const psa_paged_shape_t& s, PagedPlan* p)
{
    int rc = check_shape(s, true);
    if (rc == PSA_OK) rc = check_cache_shape(c, s);
    if (rc != PSA_OK) return rc;
    *p = make_paged_plan(c, s);
    return p->n_part * s.H_kv > kMostGroups || p->n_join * s.H_kv > kMostGroups ? PSA_ERR_SHAPE : PSA_OK;
}
static bool good_holders(int32_t B, int32_t B_out, int32_t n_pages, int32_t page_rows, int32_t max_pages)
{
    return B >= 1 && B <= kMostSequences && B_out >= 1 && B_out <= kMostSequences && good_pages(n_pages, page_rows, max_pages) &&
           (int64_t)B * max_pages <= (1 << 30) && (int64_t)B_out * max_pages <= (1 << 30);
}
static int status(hipError_t e) { return e == hipSuccess ? PSA_OK : PSA_ERR_HIP; }

}  // namespace psa

extern "C" {

int probsparse_cache_append(const psa_heads_t* K, const psa_heads_t* V, const int32_t* offsets, const psa_cache_t* cache, const psa_paged_shape_t* shape,
                            void* stream)
{
    using namespace psa;
    if (!has_data(K) || !has_data(V) || !shape || !has_tensors(cache)) return PSA_ERR_NULL;
    const psa_paged_shape_t& s = *shape;
    int rc;
    if ((rc = check_shape(s, false)) != PSA_OK || (rc = check_cache_shape(*cache, s)) != PSA_OK || (rc = check_rows(s, offsets)) != PSA_OK) return rc;
    for (const psa_heads_t* t : {K, V})
        if ((rc = check_heads(*t, s.dtype == PSA_F32 ? 4 : 8, 64, 16, 1, s.H_kv, s.T, false)) != PSA_OK) return rc;
    if ((rc = check_cache(*cache, s, true)) != PSA_OK) return rc;
    return status(launch_cache_append(*K, *V, offsets, *cache, s, static_cast<hipStream_t>(stream)));
}

size_t dense_attn_paged_workspace_bytes(const psa_cache_t* cache, const psa_paged_shape_t* shape)
{
    psa::PagedPlan p;
    return cache && shape && psa::check_attention(*cache, *shape, &p) == PSA_OK ? p.total : 0;
}

int dense_attn_paged_fwd(const psa_heads_t* Q, const int32_t* offsets, const psa_cache_t* cache, const psa_heads_t* out, float* lse,
                         const psa_paged_shape_t* shape, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace psa;
    if (!has_data(Q) || !has_data(out) || !shape || !has_tensors(cache) || !workspace) return PSA_ERR_NULL;
    const psa_paged_shape_t& s = *shape;
    PagedPlan p;
    int rc;
    if ((rc = check_attention(*cache, s, &p)) != PSA_OK || (rc = check_rows(s, offsets)) != PSA_OK) return rc;
    const int64_t unit = s.dtype == PSA_F32 ? 4 : 8;
    if ((rc = check_heads(*Q, unit, 64, 16, 1, s.H, s.T, false)) != PSA_OK || (rc = check_heads(*out, unit, 64, 16, 1, s.H, s.T, true)) != PSA_OK ||
        (rc = check_cache(*cache, s, false)) != PSA_OK) return rc;
    if (off_by(lse, 4) || off_by(workspace, 256)) return PSA_ERR_ALIGN;
    if (workspace_bytes < p.total) return PSA_ERR_WORKSPACE;
    return status(launch_paged(p, s, *Q, offsets, *cache, *out, lse, workspace, static_cast<hipStream_t>(stream)));
}

size_t probsparse_cache_update_workspace_bytes(int32_t B, int32_t B_out, int32_t n_pages)
{
    return psa::good_holders(B, B_out, n_pages, 1, 1) ? psa::cache_update_bytes(B, B_out, n_pages) : 0;
}

int probsparse_cache_update(const int32_t* table, const int32_t* lengths, const int32_t* refs, int32_t B, const int32_t* parents, const int32_t* grow,
                            int32_t B_out, int32_t n_pages, int32_t page_rows, int32_t max_pages, int32_t* table_out, int32_t* lengths_out,
                            int32_t* refs_out, int32_t* pairs, int32_t* counts, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace psa;
    if (!table || !lengths || !refs || !table_out || !lengths_out || !refs_out || !pairs || !counts || !workspace) return PSA_ERR_NULL;
    if (!good_holders(B, B_out, n_pages, page_rows, max_pages) || (!parents && B != B_out)) return PSA_ERR_SHAPE;
    for (const void* p : {(const void*)table, (const void*)lengths, (const void*)refs, (const void*)parents, (const void*)grow, (const void*)table_out,
                          (const void*)lengths_out, (const void*)refs_out, (const void*)pairs, (const void*)counts})
        if (off_by(p, 4)) return PSA_ERR_ALIGN;
    if (off_by(workspace, 256)) return PSA_ERR_ALIGN;
    // (parts of the two that overlap otherwise are the caller's to avoid)
    if (table_out == table || lengths_out == lengths || refs_out == refs) return PSA_ERR_ARG;
    if (workspace_bytes < cache_update_bytes(B, B_out, n_pages)) return PSA_ERR_WORKSPACE;
    const CacheUpdate u{table, lengths, refs, parents, grow, B, B_out, n_pages, page_rows, max_pages, table_out, lengths_out, refs_out, pairs, counts};
    return status(launch_cache_update(u, workspace, static_cast<hipStream_t>(stream)));
}

size_t probsparse_cache_compact_workspace_bytes(int32_t n_pages) { return n_pages >= 1 && n_pages <= (1 << 28) ? psa::cache_compact_bytes(n_pages) : 0; }

int probsparse_cache_compact(const int32_t* table, const int32_t* refs, int32_t B, int32_t n_pages, int32_t max_pages, int32_t* table_out, int32_t* refs_out,
                             int32_t* pairs, int32_t* counts, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace psa;
    if (!table || !refs || !table_out || !refs_out || !counts || !workspace || (!pairs && n_pages > 1)) return PSA_ERR_NULL;
    if (!good_holders(B, 1, n_pages, 1, max_pages)) return PSA_ERR_SHAPE;
    for (const void* p : {(const void*)table, (const void*)refs, (const void*)table_out, (const void*)refs_out, (const void*)pairs, (const void*)counts})
        if (off_by(p, 4)) return PSA_ERR_ALIGN;
    if (off_by(workspace, 256)) return PSA_ERR_ALIGN;
    if (refs_out == refs) return PSA_ERR_ARG;
    if (workspace_bytes < cache_compact_bytes(n_pages)) return PSA_ERR_WORKSPACE;
    return status(launch_cache_compact(table, refs, B, n_pages, max_pages, table_out, refs_out, pairs, counts, workspace, static_cast<hipStream_t>(stream)));
}

int probsparse_cache_copy(const psa_pool_t* pools, int32_t n_pools, int32_t n_pages, const int32_t* pairs, const int32_t* counts, int32_t n_pairs,
                          void* stream)
{
    using namespace psa;
    if (!pools || (!pairs && n_pairs > 0)) return PSA_ERR_NULL;
    if (n_pools < 1 || n_pages < 1 || n_pages > (1 << 28) || n_pairs < 0 || n_pairs > (1 << 28)) return PSA_ERR_SHAPE;
    for (int32_t i = 0; i < n_pools; ++i) {
        if (!pools[i].data) return PSA_ERR_NULL;
        if (pools[i].page_bytes < 1 || pools[i].page_bytes > ((int64_t)1 << 40) || pools[i].page_stride > (INT64_MAX >> 2) / n_pages) return PSA_ERR_SHAPE;
        if (n_pages > 1 && pools[i].page_stride < pools[i].page_bytes) return PSA_ERR_ARG;
    }
    if (off_by(pairs, 4) || off_by(counts, 4)) return PSA_ERR_ALIGN;
    if (n_pairs == 0) return PSA_OK;
    return status(launch_cache_copy(pools, n_pools, n_pages, pairs, counts, n_pairs, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
