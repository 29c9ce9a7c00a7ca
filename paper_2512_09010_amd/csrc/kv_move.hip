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
template <> struct piece_of<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct piece_of<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct piece_of<4> { using type = uint32_t; };
template <> struct piece_of<2> { using type = uint16_t; };

// Stored past the L2: a kernel is over only when what it left there has been written back, which these would leave to the end (1024 pages of
// 8 layers, 537 MB: 242 -> 207 us; 32 copies of a partial page: 19.4 -> 4.8; compacting 729 tokens: 14.8 -> 4.1)
template <typename P> __device__ __forceinline__ void put(P* p, P v) { __builtin_nontemporal_store(v, p); }

#define LUVC_KV_PIECES(BYTES, CALL)                                                                       \
    switch (BYTES) {                                                                                      \
    case 16: CALL(16); break;                                                                             \
    case 8: CALL(8); break;                                                                               \
    case 4: CALL(4); break;                                                                               \
    default: CALL(2); break;                                                                              \
    }
// 16-byte pieces with as many lanes to a row as it has of them, up to 64; smaller ones a wavefront to a row
#define LUVC_KV_ROWS(BYTES, LANES, CALL)                                                                  \
    switch (BYTES) {                                                                                      \
    case 16:                                                                                              \
        if (LANES == 64) CALL(16, 64) else if (LANES == 32) CALL(16, 32) else if (LANES == 16) CALL(16, 16) else CALL(16, 8) \
        break;                                                                                            \
    case 8: CALL(8, 64) break;                                                                            \
    case 4: CALL(4, 64) break;                                                                            \
    default: CALL(2, 64) break;                                                                           \
    }

// Rows of tokens: LPT lanes to a row (the power of two that holds its pieces, 64 at most), so 64 / LPT tokens to a wavefront, and
// kRowUnits rows of each in flight (33100 tokens of 4 heads written: 29.2 us with one, 28.0 with two, 26.3 with four, 26.8 with eight; 4
// videos compacted: 22.1, 20.9, 21.3, 22.1).  A token has 2 * n_heads rows in a layer, keys and then values.
constexpr int kRowUnits = 4;

// ------------------------------------------------------------------ new tokens
// What is read does not wait for where it goes.  Strides in pieces; block y: kRowUnits of the rows.
template <typename P, int LPT>
__global__ void __launch_bounds__(256)
kv_write(const P* __restrict__ k, const P* __restrict__ v, int64_t k_stride, int64_t v_stride, const int32_t* __restrict__ sizes,
         int tokens, const int32_t* __restrict__ seq, const int32_t* __restrict__ pos, const int32_t* __restrict__ table,
         int n_seqs, int max_pages, P* __restrict__ kp, P* __restrict__ vp, int32_t* __restrict__ page_sizes,
         int n_pages, int n_heads, int log2_page, int pieces)
{
    const int lane = threadIdx.x & 63, c0 = lane % LPT;
    const int t = (int)(blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / LPT) + lane / LPT;
    if (t >= tokens) return;
    const int u0 = blockIdx.y * kRowUnits;
    P a[kRowUnits];
    auto fetch = [&](int c) {
#pragma unroll
        for (int u = 0; u < kRowUnits; ++u) {
            const int unit = u0 + u, h = unit < n_heads ? unit : unit - n_heads;
            if (unit < 2 * n_heads && c < pieces) a[u] = (unit < n_heads ? k + t * k_stride : v + t * v_stride)[(int64_t)h * pieces + c];
        }
    };
    fetch(c0);
    const int s = seq ? seq[t] : t, at = pos[t];
    if (s < 0 || s >= n_seqs || at < 0 || (at >> log2_page) >= max_pages) return;
    const int page = table[(int64_t)s * max_pages + (at >> log2_page)];
    if (page < 0 || page >= n_pages) return;
    const int r = at & ((1 << log2_page) - 1);
    if (page_sizes && blockIdx.y == 0 && c0 == 0) page_sizes[((int64_t)page << log2_page) + r] = sizes ? sizes[t] : 1;
    for (int c = c0; c < pieces; c += LPT) {
        if (c != c0) fetch(c);
#pragma unroll
        for (int u = 0; u < kRowUnits; ++u) {
            const int unit = u0 + u, h = unit < n_heads ? unit : unit - n_heads;
            if (unit < 2 * n_heads) put((unit < n_heads ? kp : vp) + ((((int64_t)page * n_heads + h) << log2_page) + r) * pieces + c, a[u]);
        }
    }
}

// ------------------------------------------------------------------ pages
// As many as 4 KB of arguments hold, and a short list, which the host passes 0.1 to 0.5 us sooner (calls
// of 8 pages one after the other: 4.8 and 4.4 us, on another host 4.3 and 4.2)
constexpr int kCopyPairs = 480, kFewPairs = 16;
template <int N> struct KvPairs { int32_t src[N], dst[N]; };

// Block x of pair y; z: layer, keys or values, segment.  A page is `segs` segments of `count` pieces, `step` apart.  A piece to a thread: with
// eight the launch of 1024 pages takes 282 us for 207.
template <typename P, int N>
__global__ void __launch_bounds__(256)
kv_copy(KvPairs<N> pairs, P* __restrict__ k, P* __restrict__ v, int64_t layer_stride, int64_t page_stride, int count, int segs, int step,
        int32_t* __restrict__ page_sizes, int rows, int log2_page)
{
    const int src = pairs.src[blockIdx.y], dst = pairs.dst[blockIdx.y];
    const int seg = blockIdx.z % segs, which = blockIdx.z / segs, i = blockIdx.x * 256 + threadIdx.x;
    P* pool = (which & 1 ? v : k) + (int64_t)(which >> 1) * layer_stride + (int64_t)seg * step;
    if (i < count) put(pool + (int64_t)dst * page_stride + i, pool[(int64_t)src * page_stride + i]);
    if (page_sizes && blockIdx.x == 0 && blockIdx.z == 0)
        for (int r = threadIdx.x; r < rows; r += 256) page_sizes[((int64_t)dst << log2_page) + r] = page_sizes[((int64_t)src << log2_page) + r];
}

// ------------------------------------------------------------------ survivors
template <int N> struct KvSpans { KvSpan s[N]; };
constexpr int kFewSpans = 8;                       // a short argument list, as above

// A place j of sequence blockIdx.y and the token that goes there; block z: kRowUnits rows of it among those of all layers.
template <typename P, int LPT, int N>
__global__ void __launch_bounds__(256)
kv_compact(KvSpans<N> spans, int row0, const int32_t* __restrict__ kept_idx, const int32_t* __restrict__ table_in, int max_in,
           const int32_t* __restrict__ table_out, int max_out, P* __restrict__ k, P* __restrict__ v, int64_t layer_stride,
           int32_t* __restrict__ page_sizes, int n_pages, int n_heads, int n_layers, int log2_page, int pieces)
{
    const KvSpan& s = spans.s[blockIdx.y];
    const int lane = threadIdx.x & 63, c0 = lane % LPT, mask = (1 << log2_page) - 1;
    const int j = (int)(blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / LPT) + lane / LPT;
    if (j >= s.after) return;
    const int64_t line = row0 + blockIdx.y;
    const int po = table_out[line * max_out + (j >> log2_page)];
    int p = j;
    if (j >= s.first && j < s.first + s.keep) {
        const int i = kept_idx[s.kept + j - s.first];
        if (i < 0 || i >= s.span) return;
        p = s.first + i;
    } else if (j >= s.first) {
        p = j - s.keep + s.span;
    }
    const int pi = table_in[line * max_in + (p >> log2_page)];
    if (pi < 0 || pi >= n_pages || po < 0 || po >= n_pages || (pi == po && p == j)) return;
    const int64_t from = (((int64_t)pi * n_heads << log2_page) + (p & mask)) * pieces, to = (((int64_t)po * n_heads << log2_page) + (j & mask)) * pieces;
    if (page_sizes && blockIdx.z == 0 && c0 == 0) page_sizes[((int64_t)po << log2_page) + (j & mask)] = page_sizes[((int64_t)pi << log2_page) + (p & mask)];
    const int u0 = blockIdx.z * kRowUnits, units = 2 * n_heads * n_layers, head = pieces << log2_page;
    for (int c = c0; c < pieces; c += LPT) {
        P a[kRowUnits];
        P* to_row[kRowUnits];
#pragma unroll
        for (int u = 0; u < kRowUnits; ++u) {
            const int unit = u0 + u < units ? u0 + u : units - 1, layer = unit / (2 * n_heads), i = unit - layer * 2 * n_heads;
            P* rows = (i < n_heads ? k : v) + layer * layer_stride + (int64_t)(i < n_heads ? i : i - n_heads) * head + c;
            a[u] = rows[from];
            to_row[u] = rows + to;
        }
#pragma unroll
        for (int u = 0; u < kRowUnits; ++u)
            if (u0 + u < units) put(to_row[u], a[u]);
    }
}

}  // namespace

static int row_lanes(int bytes, int pieces) { return bytes < 16 || pieces > 32 ? 64 : pieces > 16 ? 32 : pieces > 8 ? 16 : 8; }

luvc_status kv_write_run(const luvc_kv_cache& c, int layer, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* sizes,
                         int64_t tokens, const int32_t* seq, const int32_t* pos, const int32_t* table, int n_seqs, int max_pages, hipStream_t st)
{
    const int es = (int)kv_esize(c);
    const int64_t skip = layer * c.layer_stride * es;
    char *kp = (char*)c.k + skip, *vp = (char*)c.v + skip;
    const int bytes = kv_piece((uintptr_t)k | (uintptr_t)v | (uintptr_t)kp | (uintptr_t)vp | (uint64_t)(k_stride * es) | (uint64_t)(v_stride * es) | (uint64_t)(c.D * es));
    const int pieces = c.D * es / bytes, lpt = row_lanes(bytes, pieces), each = 4 * (64 / lpt);
    const dim3 grid((unsigned)((tokens + each - 1) / each), (unsigned)((2 * c.n_heads + kRowUnits - 1) / kRowUnits));
#define LUVC_KV_WRITE(B, LPT)                                                                                                              \
    {                                                                                                                                      \
        using P = typename piece_of<B>::type;                                                                                              \
        LUVC_LAUNCH("kv_write", (kv_write<P, LPT>), grid, dim3(256), 0, st, (const P*)k, (const P*)v, k_stride * es / B, v_stride * es / B, \
                    sizes, (int)tokens, seq, pos, table, n_seqs, max_pages, (P*)kp, (P*)vp, c.sizes, c.n_pages, c.n_heads,                 \
                    kv_log2_page(c), pieces);                                                                                              \
    }
    LUVC_KV_ROWS(bytes, lpt, LUVC_KV_WRITE)
#undef LUVC_KV_WRITE
    return check_launch("write to the cache");
}

template <int N>
static luvc_status copy_launches(const luvc_kv_cache& c, const int32_t* src, int src_step, const int32_t* dst, int dst_step, int n, int rows, hipStream_t st)
{
    const int es = (int)kv_esize(c);
    const bool whole = rows == c.page_tokens;
    const int64_t seg = (int64_t)rows * c.D * es, step = (int64_t)c.page_tokens * c.D * es;
    const int64_t len = whole ? step * c.n_heads : seg;
    const int bytes = kv_piece((uintptr_t)c.k | (uintptr_t)c.v | (uint64_t)(c.layer_stride * es) | (uint64_t)len | (uint64_t)step);
    const int segs = whole ? 1 : c.n_heads, count = (int)(len / bytes);
    // layers x 2 x segments may exceed what a grid takes in z
    const int most = 65535 / (2 * segs);
    for (int i0 = 0; i0 < n; i0 += N) {
        KvPairs<N> pairs;
        const int m = n - i0 < N ? n - i0 : N;
        for (int i = 0; i < m; ++i) {
            pairs.src[i] = src[(int64_t)(i0 + i) * src_step];
            pairs.dst[i] = dst[(int64_t)(i0 + i) * dst_step];
        }
        for (int l0 = 0; l0 < c.n_layers; l0 += most) {
            const int layers = c.n_layers - l0 < most ? c.n_layers - l0 : most;
            char *k = (char*)c.k + l0 * c.layer_stride * es, *v = (char*)c.v + l0 * c.layer_stride * es;
            const unsigned gx = (unsigned)((count + 255) / 256);
            const dim3 grid(gx, m, (unsigned)(layers * 2 * segs));
#define LUVC_KV_COPY(B)                                                                                                               \
    {                                                                                                                                 \
        using P = typename piece_of<B>::type;                                                                                         \
        LUVC_LAUNCH("kv_copy", (kv_copy<P, N>), grid, dim3(256), 0, st, pairs, (P*)k, (P*)v, c.layer_stride * es / B,                 \
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

luvc_status kv_copy_run(const luvc_kv_cache& c, const int32_t* src, int src_step, const int32_t* dst, int dst_step, int n, int rows, hipStream_t st)
{
    return n <= kFewPairs ? copy_launches<kFewPairs>(c, src, src_step, dst, dst_step, n, rows, st)
                          : copy_launches<kCopyPairs>(c, src, src_step, dst, dst_step, n, rows, st);
}

template <int N>
static luvc_status compact_launches(const luvc_kv_cache& c, const KvSpan* list, int n, int row0, const int32_t* kept_idx, const int32_t* table_in, int max_in,
                                    const int32_t* table_out, int max_out, hipStream_t st)
{
    KvSpans<N> spans;
    int most = 0;
    for (int i = 0; i < n; ++i) {
        spans.s[i] = list[i];
        most = list[i].after > most ? list[i].after : most;
    }
    if (most == 0) return LUVC_OK;
    const int es = (int)kv_esize(c);
    const int bytes = kv_piece((uintptr_t)c.k | (uintptr_t)c.v | (uint64_t)(c.layer_stride * es) | (uint64_t)(c.D * es));
    const int pieces = c.D * es / bytes, lpt = row_lanes(bytes, pieces), each = 4 * (64 / lpt);
    const unsigned gx = (unsigned)((most + each - 1) / each);
    const int max_layers = 65535 * kRowUnits / (2 * c.n_heads);
    for (int l0 = 0; l0 < c.n_layers; l0 += max_layers) {
        const int layers = c.n_layers - l0 < max_layers ? c.n_layers - l0 : max_layers;
        char *k = (char*)c.k + l0 * c.layer_stride * es, *v = (char*)c.v + l0 * c.layer_stride * es;
        const dim3 grid(gx, n, (unsigned)((2 * c.n_heads * layers + kRowUnits - 1) / kRowUnits));
#define LUVC_KV_COMPACT(B, LPT)                                                                                                       \
    {                                                                                                                                 \
        using P = typename piece_of<B>::type;                                                                                         \
        LUVC_LAUNCH("kv_compact", (kv_compact<P, LPT, N>), grid, dim3(256), 0, st, spans, row0, kept_idx, table_in, max_in, table_out,         \
                    max_out, (P*)k, (P*)v, c.layer_stride * es / B, l0 == 0 ? c.sizes : nullptr, c.n_pages, c.n_heads, layers,        \
                    kv_log2_page(c), pieces);                                                                                         \
    }
        LUVC_KV_ROWS(bytes, lpt, LUVC_KV_COMPACT)
#undef LUVC_KV_COMPACT
        const luvc_status rc = check_launch("compaction of the cache");
        if (rc != LUVC_OK) return rc;
    }
    return LUVC_OK;
}

luvc_status kv_compact_run(const luvc_kv_cache& c, const KvSpan* spans, int n, int row0, const int32_t* kept_idx,
                           const int32_t* table_in, int max_in, const int32_t* table_out, int max_out, hipStream_t st)
{
    return n <= kFewSpans ? compact_launches<kFewSpans>(c, spans, n, row0, kept_idx, table_in, max_in, table_out, max_out, st)
                          : compact_launches<kKvMaxSeqs>(c, spans, n, row0, kept_idx, table_in, max_in, table_out, max_out, st);
}

}  // namespace luvc
