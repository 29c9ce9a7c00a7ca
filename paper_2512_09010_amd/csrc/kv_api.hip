// C ABI of the paged key-value cache (declared in include/luvc.h): argument checks, the counting of pages, dispatch.
// Every check happens before the first launch, so a failing call enqueues nothing.
#include <cmath>
#include <cstdlib>

#include "common.hpp"
#include "kv.hpp"

using namespace luvc;

namespace {

bool cache_shape_ok(const luvc_kv_cache* c, luvc_status* rc)
{
    *rc = LUVC_ERR_INVALID_ARG;
    if (!c) { set_error("the cache must not be NULL"); return false; }
    if (c->dtype != LUVC_F32 && c->dtype != LUVC_BF16) { set_error("unknown dtype %d", (int)c->dtype); return false; }
    if (c->n_heads < 1 || c->D < 1) { set_error("n_heads and D must be positive (got %d, %d)", c->n_heads, c->D); return false; }
    *rc = LUVC_ERR_UNSUPPORTED;
    if (c->n_heads > kKvMaxHeads) { set_error("n_heads=%d exceeds %d", c->n_heads, kKvMaxHeads); return false; }
    if (c->D > kKvMaxD) { set_error("D=%d exceeds %d channels per head", c->D, kKvMaxD); return false; }
    *rc = LUVC_OK;
    return true;
}

bool cache_ok(const luvc_kv_cache* c, luvc_status* rc)
{
    if (!cache_shape_ok(c, rc)) return false;
    *rc = LUVC_ERR_INVALID_ARG;
    if (!c->k || !c->v) { set_error("k and v of the cache must not be NULL"); return false; }
    if (c->n_layers < 1 || c->n_pages < 1 || c->page_tokens < 1) {
        set_error("n_layers, n_pages and page_tokens must be positive (got %d, %d, %d)", c->n_layers, c->n_pages, c->page_tokens);
        return false;
    }
    if (((uintptr_t)c->k | (uintptr_t)c->v) % kv_esize(*c) || (uintptr_t)c->sizes % 4) { set_error("k, v and sizes must be aligned to their elements"); return false; }
    *rc = LUVC_ERR_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1))) {
        set_error("page_tokens=%d must be a power of two from 16 to 1024", c->page_tokens);
        return false;
    }
    *rc = LUVC_ERR_INVALID_ARG;
    if (c->layer_stride < c->n_pages * kv_page_elems(*c)) {
        set_error("layer_stride %lld is smaller than the %d pages of a layer", (long long)c->layer_stride, c->n_pages);
        return false;
    }
    *rc = LUVC_OK;
    return true;
}

bool layer_ok(const luvc_kv_cache* c, int layer, luvc_status* rc)
{
    if (!cache_ok(c, rc)) return false;
    if (layer < 0 || layer >= c->n_layers) { set_error("layer %d is not in 0..%d", layer, c->n_layers - 1); *rc = LUVC_ERR_INVALID_ARG; return false; }
    return true;
}

// The n free pages with the lowest numbers go to pages[0], pages[step], ...; false if there are fewer
bool take(int32_t* refs, int n_pages, int n, int32_t* pages, int64_t step)
{
    constexpr int AT_ONCE = 16;                      // pages in use are passed over in groups: a full pool is a long list
    int got = 0;
    for (int p = 0; p < n_pages && got < n; ++p) {
        if (p % AT_ONCE == 0 && p + AT_ONCE <= n_pages) {
            int free_ones = 0;
            for (int i = 0; i < AT_ONCE; ++i) free_ones += refs[p + i] == 0;
            if (!free_ones) { p += AT_ONCE - 1; continue; }
        }
        if (refs[p] == 0) pages[got++ * step] = p;
    }
    if (got < n) { set_error("%d pages are needed, %d of %d are free", n, got, n_pages); return false; }
    for (int i = 0; i < n; ++i) refs[pages[i * step]] = 1;
    return true;
}

}  // namespace

extern "C" {

luvc_status luvc_kv_write(const luvc_kv_cache* cache, int layer, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                          const int32_t* sizes, int64_t tokens, const int32_t* seq, const int32_t* pos, const int32_t* table,
                          int n_seqs, int max_pages, void* hip_stream)
{
    luvc_status rc;
    if (!layer_ok(cache, layer, &rc)) return rc;
    if (tokens < 0 || n_seqs < 1 || max_pages < 1) { set_error("tokens must not be negative, n_seqs and max_pages must be positive"); return LUVC_ERR_INVALID_ARG; }
    if (sizes && !cache->sizes) { set_error("sizes given for a cache without sizes"); return LUVC_ERR_INVALID_ARG; }
    const int64_t row = (int64_t)cache->n_heads * cache->D;
    if (k_stride < row || v_stride < row) { set_error("token strides must be at least n_heads * D = %lld", (long long)row); return LUVC_ERR_INVALID_ARG; }
    if (tokens == 0) return LUVC_OK;
    if (!k || !v || !pos || !table) { set_error("k, v, pos and table must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    if (((uintptr_t)k | (uintptr_t)v) % kv_esize(*cache)) { set_error("k and v must be aligned to their elements"); return LUVC_ERR_INVALID_ARG; }
    if (tokens >= ((int64_t)1 << 25)) { set_error("tokens must stay below 2^25 per call"); return LUVC_ERR_UNSUPPORTED; }
    return kv_write_run(*cache, layer, k, k_stride, v, v_stride, sizes, tokens, seq, pos, table, n_seqs, max_pages, (hipStream_t)hip_stream);
}

static bool attend_sizes_ok(const luvc_kv_cache* cache, int n_seqs, int n_q_heads, int max_tokens, luvc_status* rc)
{
    *rc = LUVC_ERR_INVALID_ARG;
    if (n_seqs < 1 || n_q_heads < 1 || max_tokens < 1) { set_error("n_seqs, n_q_heads and max_tokens must be positive (got %d, %d, %d)", n_seqs, n_q_heads, max_tokens); return false; }
    if (n_q_heads % cache->n_heads) { set_error("n_q_heads=%d is no multiple of the cache's %d heads", n_q_heads, cache->n_heads); return false; }
    *rc = LUVC_ERR_UNSUPPORTED;
    if (max_tokens >= (1 << 30)) { set_error("max_tokens must stay below 2^30"); return false; }
    if ((int64_t)n_seqs * n_q_heads >= ((int64_t)1 << 22)) { set_error("n_seqs * n_q_heads must stay below 2^22"); return false; }
    *rc = LUVC_OK;
    return true;
}

size_t luvc_kv_attend_workspace_bytes(const luvc_kv_cache* cache, int n_seqs, int n_q_heads, int max_tokens)
{
    luvc_status rc;
    if (!cache_shape_ok(cache, &rc) || !attend_sizes_ok(cache, n_seqs, n_q_heads, max_tokens, &rc)) return 0;
    return kv_attend_workspace(n_seqs, n_q_heads, cache->n_heads, cache->D, cache->dtype, max_tokens);
}

luvc_status luvc_kv_attend(const luvc_kv_cache* cache, int layer, const void* q, int64_t q_stride, int n_q_heads, int n_seqs,
                           const int32_t* table, int max_pages, const int32_t* lengths, int max_tokens, const double* scale, int enhance,
                           void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    luvc_status rc;
    if (!layer_ok(cache, layer, &rc)) return rc;
    if (!q || !table || !lengths || !out) { set_error("q, table, lengths and out must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    if (!attend_sizes_ok(cache, n_seqs, n_q_heads, max_tokens, &rc)) return rc;
    if (max_pages < 1) { set_error("max_pages must be positive"); return LUVC_ERR_INVALID_ARG; }
    const int64_t row = (int64_t)n_q_heads * cache->D;
    if (q_stride < row || out_stride < row) { set_error("sequence strides must be at least n_q_heads * D = %lld", (long long)row); return LUVC_ERR_INVALID_ARG; }
    if (((uintptr_t)q | (uintptr_t)out) % kv_esize(*cache)) { set_error("q and out must be aligned to their elements"); return LUVC_ERR_INVALID_ARG; }
    if (enhance && !cache->sizes) { set_error("the term log s needs a cache with sizes"); return LUVC_ERR_INVALID_ARG; }
    const double sc = scale ? *scale : 1.0 / std::sqrt((double)cache->D);
    if (!std::isfinite((float)(2.0 * sc))) { set_error("scale must be finite in fp32"); return LUVC_ERR_INVALID_ARG; }
    const size_t need = kv_attend_workspace(n_seqs, n_q_heads, cache->n_heads, cache->D, cache->dtype, max_tokens);
    if (!workspace_ok(workspace, workspace_bytes, need)) return LUVC_ERR_WORKSPACE;
    const KvAttend a{q, out, q_stride, out_stride, table, lengths, n_seqs, n_q_heads, max_pages, max_tokens, sc, enhance != 0};
    return kv_attend_run(*cache, layer, a, workspace, (hipStream_t)hip_stream);
}

luvc_status luvc_kv_compact(const luvc_kv_cache* cache, int n_seqs, const int32_t* lengths, const int32_t* first, const int32_t* span,
                            const int32_t* n_keep, const int32_t* kept_idx, const int32_t* table_in, int max_pages_in,
                            const int32_t* table_out, int max_pages_out, void* hip_stream)
{
    luvc_status rc;
    if (!cache_ok(cache, &rc)) return rc;
    if (n_seqs < 1 || max_pages_in < 1 || max_pages_out < 1) { set_error("n_seqs and the tables' widths must be positive"); return LUVC_ERR_INVALID_ARG; }
    if (!lengths || !first || !span || !n_keep || !table_in || !table_out) {
        set_error("lengths, first, span, n_keep, table_in and table_out must not be NULL");
        return LUVC_ERR_INVALID_ARG;
    }
    const int64_t P = cache->page_tokens;
    int64_t kept = 0;
    for (int i = 0; i < n_seqs; ++i) {
        if (first[i] < 0 || span[i] < 0 || n_keep[i] < 0 || n_keep[i] > span[i] || (int64_t)first[i] + span[i] > lengths[i]) {
            set_error("sequence %d: %d of %d tokens from position %d on do not fit a length of %d", i, n_keep[i], span[i], first[i], lengths[i]);
            return LUVC_ERR_INVALID_ARG;
        }
        const int64_t after = (int64_t)lengths[i] - span[i] + n_keep[i];
        if (lengths[i] > max_pages_in * P || after > max_pages_out * P) {
            set_error("sequence %d: %d tokens before and %lld after do not fit the tables' %d and %d pages", i, lengths[i], (long long)after, max_pages_in, max_pages_out);
            return LUVC_ERR_INVALID_ARG;
        }
        if (lengths[i] >= (1 << 25)) { set_error("sequence %d: lengths must stay below 2^25", i); return LUVC_ERR_UNSUPPORTED; }
        kept += n_keep[i];
    }
    if (kept && !kept_idx) { set_error("kept_idx must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    kept = 0;
    for (int i0 = 0; i0 < n_seqs; i0 += kKvMaxSeqs) {
        KvSpan spans[kKvMaxSeqs];
        const int n = n_seqs - i0 < kKvMaxSeqs ? n_seqs - i0 : kKvMaxSeqs;
        for (int j = 0; j < n; ++j) {
            const int i = i0 + j;
            spans[j] = KvSpan{first[i], span[i], n_keep[i], lengths[i] - span[i] + n_keep[i], kept};
            kept += n_keep[i];
        }
        rc = kv_compact_run(*cache, spans, n, i0, kept_idx, table_in, max_pages_in, table_out, max_pages_out, (hipStream_t)hip_stream);
        if (rc != LUVC_OK) return rc;
    }
    return LUVC_OK;
}

luvc_status luvc_kv_copy_pages(const luvc_kv_cache* cache, const int32_t* src, const int32_t* dst, int n, void* hip_stream)
{
    luvc_status rc;
    if (!cache_ok(cache, &rc)) return rc;
    if (n < 0) { set_error("n must not be negative"); return LUVC_ERR_INVALID_ARG; }
    if (n == 0) return LUVC_OK;
    if (!src || !dst) { set_error("src and dst must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    for (int i = 0; i < n; ++i)
        if (src[i] < 0 || src[i] >= cache->n_pages || dst[i] < 0 || dst[i] >= cache->n_pages) {
            set_error("pair %d: pages %d and %d are not in 0..%d", i, src[i], dst[i], cache->n_pages - 1);
            return LUVC_ERR_INVALID_ARG;
        }
    // a page is written once and never read: few pairs are compared with each other, for more there is a mark per page
    int bad = -1;
    if (n <= 16) {
        for (int i = 0; i < n && bad < 0; ++i)
            for (int j = 0; j < n; ++j)
                if (dst[i] == src[j] || (j < i && dst[i] == dst[j])) bad = i;
    } else {
        unsigned char* seen = (unsigned char*)calloc((size_t)cache->n_pages, 1);
        if (!seen) { set_error("no host memory for the check of %d pages", cache->n_pages); return LUVC_ERR_WORKSPACE; }
        for (int i = 0; i < n; ++i) seen[src[i]] = 1;
        for (int i = 0; i < n && bad < 0; ++i) {
            if (seen[dst[i]]) bad = i;
            seen[dst[i]] = 2;
        }
        free(seen);
    }
    if (bad >= 0) { set_error("pair %d: page %d is written to and in use by another pair", bad, dst[bad]); return LUVC_ERR_INVALID_ARG; }
    return kv_copy_run(*cache, src, 1, dst, 1, n, cache->page_tokens, (hipStream_t)hip_stream);
}

luvc_status luvc_kv_take(int32_t* refs, int n_pages, int n, int32_t* pages)
{
    if (n_pages < 1 || n < 0) { set_error("n_pages must be positive, n not negative"); return LUVC_ERR_INVALID_ARG; }
    if (n == 0) return LUVC_OK;
    if (!refs || !pages) { set_error("refs and pages must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    return take(refs, n_pages, n, pages, 1) ? LUVC_OK : LUVC_ERR_WORKSPACE;
}

luvc_status luvc_kv_fork(const luvc_kv_cache* cache, int32_t* refs, const int32_t* pages, int64_t length, int n_children,
                         int32_t* child_pages, void* hip_stream)
{
    luvc_status rc;
    if (!cache_ok(cache, &rc)) return rc;
    if (length < 1 || n_children < 1) { set_error("length and n_children must be positive"); return LUVC_ERR_INVALID_ARG; }
    if (!refs || !pages || !child_pages) { set_error("refs, pages and child_pages must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    const int64_t P = cache->page_tokens;
    if (length > cache->n_pages * P) { set_error("%lld tokens do not fit %d pages", (long long)length, cache->n_pages); return LUVC_ERR_INVALID_ARG; }
    const int64_t full = length / P, all = (length + P - 1) / P;
    const int rows = (int)(length % P);
    for (int64_t j = 0; j < all; ++j)
        if (pages[j] < 0 || pages[j] >= cache->n_pages || refs[pages[j]] < 1) {
            set_error("page %d at %lld of the sequence is not in use", pages[j], (long long)j);
            return LUVC_ERR_INVALID_ARG;
        }
    // counted one by one: a sequence may hold a page at several places
    auto uncount = [&](int64_t n) { while (n-- > 0) refs[pages[n]] -= n_children; };
    for (int64_t j = 0; j < full; ++j) {
        if (refs[pages[j]] > INT32_MAX - n_children) {
            set_error("page %d would count too many sequences", pages[j]);
            uncount(j);
            return LUVC_ERR_INVALID_ARG;
        }
        refs[pages[j]] += n_children;
    }
    if (rows) {
        if (!take(refs, cache->n_pages, n_children, child_pages + full, all)) { uncount(full); return LUVC_ERR_WORKSPACE; }
        rc = kv_copy_run(*cache, pages + full, 0, child_pages + full, (int)all, n_children, rows, (hipStream_t)hip_stream);
        if (rc != LUVC_OK) {
            for (int i = 0; i < n_children; ++i) refs[child_pages[i * all + full]] = 0;
            uncount(full);
            return rc;
        }
    }
    for (int i = 0; i < n_children; ++i)
        for (int64_t j = 0; j < full; ++j) child_pages[i * all + j] = pages[j];
    return LUVC_OK;
}

luvc_status luvc_kv_release(int32_t* refs, int n_pages, const int32_t* pages, int n)
{
    if (n_pages < 1 || n < 0) { set_error("n_pages must be positive, n not negative"); return LUVC_ERR_INVALID_ARG; }
    if (n == 0) return LUVC_OK;
    if (!refs || !pages) { set_error("refs and pages must not be NULL"); return LUVC_ERR_INVALID_ARG; }
    for (int i = 0; i < n; ++i) {
        if (pages[i] >= 0 && pages[i] < n_pages && refs[pages[i]] > 0) { --refs[pages[i]]; continue; }
        set_error("page %d at %d of the list is not in use", pages[i], i);
        while (i-- > 0) ++refs[pages[i]];
        return LUVC_ERR_INVALID_ARG;
    }
    return LUVC_OK;
}

}  // extern "C"
