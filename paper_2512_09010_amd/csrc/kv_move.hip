// Moving rows of the paged key-value cache: new tokens into their pages (kv_write), whole pages and the rows of a partial
// one to other pages (kv_copy), the survivors of a stage of SPU (paper Section 3.3) to the front (kv_compact).
//
// Nothing is computed, so what bounds all three is HBM: every byte read once and written once.  Rows move in the
// largest pieces that addresses and lengths allow, 16 bytes where D fills them; the loads of a trip are all in flight before
// the first store waits for one.
#include "common.hpp"
#include "kv.hpp"

namespace luvc {

namespace {

// What a thread moves at a time
template <int BYTES> struct piece_of;
template <> struct piece_of<16> { using type = uint4; };
template <> struct piece_of<8> { using type = uint2; };
template <> struct piece_of<4> { using type = uint32_t; };
template <> struct piece_of<2> { using type = uint16_t; };

#define LUVC_KV_PIECES(BYTES, CALL)                                                                       \
    switch (BYTES) {                                                                                      \
    case 16: CALL(16); break;                                                                             \
    case 8: CALL(8); break;                                                                               \
    case 4: CALL(4); break;                                                                               \
    default: CALL(2); break;                                                                              \
    }

// ------------------------------------------------------------------ new tokens
// A wavefront per token.  All lengths and strides in pieces.
constexpr int kWritePieces = 2;                    // of K and of V each, in flight per lane
template <typename P>
__global__ void __launch_bounds__(256)
kv_write(const P* __restrict__ k, const P* __restrict__ v, int64_t k_stride, int64_t v_stride, const int32_t* __restrict__ sizes,
         int tokens, const int32_t* __restrict__ seq, const int32_t* __restrict__ pos, const int32_t* __restrict__ table,
         int n_seqs, int max_pages, P* __restrict__ kp, P* __restrict__ vp, int32_t* __restrict__ page_sizes,
         int n_pages, int n_heads, int log2_page, KvDiv row)
{
    const int lane = threadIdx.x & 63;
    const int t = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6)));
    if (t >= tokens) return;
    const int s = seq ? seq[t] : t, at = pos[t];
    const int n = n_heads * (int)row.d;
    if (s < 0 || s >= n_seqs || at < 0 || (at >> log2_page) >= max_pages) return;
    const int page = table[(int64_t)s * max_pages + (at >> log2_page)];
    if (page < 0 || page >= n_pages) return;
    const int P0 = 1 << log2_page, r = at & (P0 - 1);
    const P *ks = k + (int64_t)t * k_stride, *vs = v + (int64_t)t * v_stride;
    const int64_t to = (int64_t)page * n << log2_page;
    if (page_sizes && lane == 0) page_sizes[((int64_t)page << log2_page) + r] = sizes ? sizes[t] : 1;
    for (int i0 = lane; i0 < n; i0 += 64 * kWritePieces) {
        P a[kWritePieces], b[kWritePieces];
#pragma unroll
        for (int u = 0; u < kWritePieces; ++u) {
            const int i = i0 + 64 * u;
            if (i < n) { a[u] = ks[i]; b[u] = vs[i]; }
        }
#pragma unroll
        for (int u = 0; u < kWritePieces; ++u) {
            const int i = i0 + 64 * u;
            if (i >= n) continue;
            const int h = (int)((uint32_t)i / row);
            const int64_t o = to + ((int64_t)(h << log2_page) + r) * row.d + (i - h * (int)row.d);
            kp[o] = a[u];
            vp[o] = b[u];
        }
    }
}

// ------------------------------------------------------------------ pages
constexpr int kCopyPairs = 256, kCopyPieces = 4;
struct KvPairs { int32_t src[kCopyPairs], dst[kCopyPairs]; };

// Block x of pair y; z: layer, keys or values, segment.  A page is `segs` segments of `count` pieces, `step` apart.
template <typename P>
__global__ void __launch_bounds__(256)
kv_copy(KvPairs pairs, P* __restrict__ k, P* __restrict__ v, int64_t layer_stride, int64_t page_stride, int count, int segs, int step,
        int32_t* __restrict__ page_sizes, int rows, int log2_page)
{
    const int src = pairs.src[blockIdx.y], dst = pairs.dst[blockIdx.y];
    const int seg = blockIdx.z % segs, which = blockIdx.z / segs;
    P* pool = (which & 1 ? v : k) + (int64_t)(which >> 1) * layer_stride + (int64_t)seg * step;
    const P* a = pool + (int64_t)src * page_stride;
    P* b = pool + (int64_t)dst * page_stride;
    const int i0 = blockIdx.x * 256 * kCopyPieces + threadIdx.x;
    P p[kCopyPieces];
#pragma unroll
    for (int u = 0; u < kCopyPieces; ++u)
        if (i0 + 256 * u < count) p[u] = a[i0 + 256 * u];
#pragma unroll
    for (int u = 0; u < kCopyPieces; ++u)
        if (i0 + 256 * u < count) b[i0 + 256 * u] = p[u];
    if (page_sizes && blockIdx.x == 0 && blockIdx.z == 0)
        for (int r = threadIdx.x; r < rows; r += 256) page_sizes[((int64_t)dst << log2_page) + r] = page_sizes[((int64_t)src << log2_page) + r];
}

// ------------------------------------------------------------------ survivors
constexpr int kCompactTokens = 64, kCompactPieces = 4;

// Block x: 64 places of sequence y; z: layer, keys or values, group of heads.
template <typename P>
__global__ void __launch_bounds__(256)
kv_compact(KvSpans spans, const int32_t* __restrict__ kept_idx, const int32_t* __restrict__ table_in, int max_in,
           const int32_t* __restrict__ table_out, int max_out, P* __restrict__ k, P* __restrict__ v, int64_t layer_stride,
           int32_t* __restrict__ page_sizes, int n_pages, int n_heads, int heads_each, int log2_page, KvDiv row)
{
    __shared__ int64_t from[kCompactTokens], to[kCompactTokens];         // rows of the pool, head 0; -1: nothing to move
    const KvSpan& s = spans.s[blockIdx.y];
    const int j0 = blockIdx.x * kCompactTokens;
    if (j0 >= s.after) return;
    const int groups = (n_heads + heads_each - 1) / heads_each;
    const int h0 = (int)(blockIdx.z % groups) * heads_each, which = blockIdx.z / groups;
    const int h1 = h0 + heads_each < n_heads ? h0 + heads_each : n_heads;
    const int mask = (1 << log2_page) - 1;
    if (threadIdx.x < kCompactTokens) {
        const int j = j0 + threadIdx.x;
        int64_t a = -1, b = -1;
        if (j < s.after) {
            int p = j;
            bool ok = true;
            if (j >= s.first && j < s.first + s.keep) {
                const int i = kept_idx[s.kept + j - s.first];
                ok = i >= 0 && i < s.span;
                p = s.first + i;
            } else if (j >= s.first) {
                p = j - s.keep + s.span;
            }
            if (ok) {
                const int64_t line = spans.row0 + blockIdx.y;
                const int pi = table_in[line * max_in + (p >> log2_page)], po = table_out[line * max_out + (j >> log2_page)];
                if (pi >= 0 && pi < n_pages && po >= 0 && po < n_pages && !(pi == po && p == j)) {
                    a = ((int64_t)pi * n_heads << log2_page) + (p & mask);
                    b = ((int64_t)po * n_heads << log2_page) + (j & mask);
                    if (page_sizes && blockIdx.z == 0) page_sizes[((int64_t)po << log2_page) + (j & mask)] = page_sizes[((int64_t)pi << log2_page) + (p & mask)];
                }
            }
        }
        from[threadIdx.x] = a;
        to[threadIdx.x] = b;
    }
    __syncthreads();
    P* pool = (which & 1 ? v : k) + (int64_t)(which >> 1) * layer_stride;
    const int n = kCompactTokens * (int)row.d;
    for (int h = h0; h < h1; ++h) {
        const int64_t head = (int64_t)h << log2_page;
        for (int i0 = threadIdx.x; i0 < n; i0 += 256 * kCompactPieces) {
            P p[kCompactPieces];
            int64_t o[kCompactPieces];
#pragma unroll
            for (int u = 0; u < kCompactPieces; ++u) {
                const int i = i0 + 256 * u;
                o[u] = -1;
                if (i >= n) continue;
                const int t = (int)((uint32_t)i / row), c = i - t * (int)row.d;
                if (from[t] < 0) continue;
                p[u] = pool[(from[t] + head) * row.d + c];
                o[u] = (to[t] + head) * row.d + c;
            }
#pragma unroll
            for (int u = 0; u < kCompactPieces; ++u)
                if (o[u] >= 0) pool[o[u]] = p[u];
        }
    }
}

}  // namespace

luvc_status kv_write_run(const luvc_kv_cache& c, int layer, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* sizes,
                         int64_t tokens, const int32_t* seq, const int32_t* pos, const int32_t* table, int n_seqs, int max_pages, hipStream_t st)
{
    const int es = (int)kv_esize(c);
    const int64_t skip = layer * c.layer_stride * es;
    char *kp = (char*)c.k + skip, *vp = (char*)c.v + skip;
    const int bytes = kv_piece((uintptr_t)k | (uintptr_t)v | (uintptr_t)kp | (uintptr_t)vp | (uint64_t)(k_stride * es) | (uint64_t)(v_stride * es) | (uint64_t)(c.D * es));
    const unsigned grid = (unsigned)((tokens + 3) / 4);
#define LUVC_KV_WRITE(B)                                                                                                                   \
    {                                                                                                                                      \
        using P = typename piece_of<B>::type;                                                                                              \
        LUVC_LAUNCH("kv_write", (kv_write<P>), dim3(grid), dim3(256), 0, st, (const P*)k, (const P*)v, k_stride * es / B, v_stride * es / B, \
                    sizes, (int)tokens, seq, pos, table, n_seqs, max_pages, (P*)kp, (P*)vp, c.sizes, c.n_pages, c.n_heads,                 \
                    kv_log2_page(c), kv_div((uint32_t)(c.D * es / B)));                                                                    \
    }
    LUVC_KV_PIECES(bytes, LUVC_KV_WRITE)
#undef LUVC_KV_WRITE
    return check_launch("write to the cache");
}

luvc_status kv_copy_run(const luvc_kv_cache& c, const int32_t* src, int src_step, const int32_t* dst, int dst_step, int n, int rows, hipStream_t st)
{
    const int es = (int)kv_esize(c);
    const bool whole = rows == c.page_tokens;
    const int64_t seg = (int64_t)rows * c.D * es, step = (int64_t)c.page_tokens * c.D * es;
    const int64_t len = whole ? step * c.n_heads : seg;
    const int bytes = kv_piece((uintptr_t)c.k | (uintptr_t)c.v | (uint64_t)(c.layer_stride * es) | (uint64_t)len | (uint64_t)step);
    const int segs = whole ? 1 : c.n_heads, count = (int)(len / bytes);
    // layers x 2 x segments may exceed what a grid takes in z
    const int most = 65535 / (2 * segs);
    for (int i0 = 0; i0 < n; i0 += kCopyPairs) {
        KvPairs pairs;
        const int m = n - i0 < kCopyPairs ? n - i0 : kCopyPairs;
        for (int i = 0; i < m; ++i) {
            pairs.src[i] = src[(int64_t)(i0 + i) * src_step];
            pairs.dst[i] = dst[(int64_t)(i0 + i) * dst_step];
        }
        for (int l0 = 0; l0 < c.n_layers; l0 += most) {
            const int layers = c.n_layers - l0 < most ? c.n_layers - l0 : most;
            char *k = (char*)c.k + l0 * c.layer_stride * es, *v = (char*)c.v + l0 * c.layer_stride * es;
            const unsigned gx = (unsigned)((count + 256 * kCopyPieces - 1) / (256 * kCopyPieces));
            const dim3 grid(gx, m, (unsigned)(layers * 2 * segs));
#define LUVC_KV_COPY(B)                                                                                                               \
    {                                                                                                                                 \
        using P = typename piece_of<B>::type;                                                                                         \
        LUVC_LAUNCH("kv_copy", (kv_copy<P>), grid, dim3(256), 0, st, pairs, (P*)k, (P*)v, c.layer_stride * es / B,                    \
                    step * c.n_heads / B, count, segs, (int)(step / B), l0 == 0 ? c.sizes : nullptr, rows, kv_log2_page(c));          \
    }
            LUVC_KV_PIECES(bytes, LUVC_KV_COPY)
#undef LUVC_KV_COPY
            const luvc_status rc = check_launch("copy of pages");
            if (rc != LUVC_OK) return rc;
        }
    }
    return LUVC_OK;
}

luvc_status kv_compact_run(const luvc_kv_cache& c, const KvSpans& spans, const int32_t* kept_idx, const int32_t* table_in, int max_in,
                           const int32_t* table_out, int max_out, hipStream_t st)
{
    const int es = (int)kv_esize(c);
    const int bytes = kv_piece((uintptr_t)c.k | (uintptr_t)c.v | (uint64_t)(c.layer_stride * es) | (uint64_t)(c.D * es));
    int most = 0;
    for (int i = 0; i < spans.n; ++i) most = spans.s[i].after > most ? spans.s[i].after : most;
    if (most == 0) return LUVC_OK;
    const unsigned gx = (unsigned)((most + kCompactTokens - 1) / kCompactTokens);
    // all heads of 64 tokens to a block, fewer where that leaves compute units without work
    int heads_each = c.n_heads;
    while (heads_each > 1 && (int64_t)gx * spans.n * c.n_layers * 2 * ((c.n_heads + heads_each - 1) / heads_each) < 1024) heads_each = (heads_each + 1) / 2;
    const int groups = (c.n_heads + heads_each - 1) / heads_each, max_layers = 65535 / (2 * groups);
    for (int l0 = 0; l0 < c.n_layers; l0 += max_layers) {
        const int layers = c.n_layers - l0 < max_layers ? c.n_layers - l0 : max_layers;
        char *k = (char*)c.k + l0 * c.layer_stride * es, *v = (char*)c.v + l0 * c.layer_stride * es;
#define LUVC_KV_COMPACT(B)                                                                                                            \
    {                                                                                                                                 \
        using P = typename piece_of<B>::type;                                                                                         \
        LUVC_LAUNCH("kv_compact", (kv_compact<P>), dim3(gx, spans.n, layers * 2 * groups), dim3(256), 0, st, spans, kept_idx,         \
                    table_in, max_in, table_out, max_out, (P*)k, (P*)v, c.layer_stride * es / B, l0 == 0 ? c.sizes : nullptr,         \
                    c.n_pages, c.n_heads, heads_each, kv_log2_page(c), kv_div((uint32_t)(c.D * es / B)));                             \
    }
        LUVC_KV_PIECES(bytes, LUVC_KV_COMPACT)
#undef LUVC_KV_COMPACT
        const luvc_status rc = check_launch("compaction of the cache");
        if (rc != LUVC_OK) return rc;
    }
    return LUVC_OK;
}

}  // namespace luvc
