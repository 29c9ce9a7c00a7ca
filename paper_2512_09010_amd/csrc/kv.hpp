// Internal interface between the C-ABI layer and the kernels of the paged key-value cache.
#pragma once
#include "common.hpp"

namespace luvc {

constexpr int kKvMaxD = 256, kKvMaxHeads = 1024;

inline size_t kv_esize(const luvc_kv_cache& c) { return c.dtype == LUVC_F32 ? 4 : 2; }
inline int64_t kv_page_elems(const luvc_kv_cache& c) { return (int64_t)c.n_heads * c.page_tokens * c.D; }
inline int kv_log2_page(const luvc_kv_cache& c) { return 31 - __builtin_clz((unsigned)c.page_tokens); }

// Bytes that rows may be moved in at a time: the largest power of two up to 16 that divides everything in `bits` (offsets, lengths and
// addresses in bytes, or'ed)
inline int kv_piece(uint64_t bits)
{
    int p = 16;
    while (p > 2 && bits % p) p >>= 1;
    return p;
}

luvc_status kv_write_run(const luvc_kv_cache& c, int layer, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* sizes,
                         int64_t tokens, const int32_t* seq, const int32_t* pos, const int32_t* table, int n_seqs, int max_pages, hipStream_t st);

// rows [0, rows) of page src[i * src_step] to page dst[i * dst_step], all layers, i < n
luvc_status kv_copy_run(const luvc_kv_cache& c, const int32_t* src, int src_step, const int32_t* dst, int dst_step, int n, int rows, hipStream_t st);

struct KvSpan { int32_t first, span, keep, after; int64_t kept; };       // kept: where its entries of kept_idx start
constexpr int kKvMaxSeqs = 64;                   // sequences of a call
// spans[i] is table row row0 + i, i < n
luvc_status kv_compact_run(const luvc_kv_cache& c, const KvSpan* spans, int n, int row0, const int32_t* kept_idx, const int32_t* table_in, int max_in,
                           const int32_t* table_out, int max_out, hipStream_t st);

struct KvAttend {
    const void* q;
    void* out;
    int64_t q_stride, out_stride;
    const int32_t *table, *lengths;
    int n_seqs, n_q_heads, max_pages, max_tokens;
    double scale;
    bool enhance;
};
size_t kv_attend_workspace(int n_seqs, int n_q_heads, int n_heads, int D, luvc_dtype dt, int max_tokens);
luvc_status kv_attend_run(const luvc_kv_cache& c, int layer, const KvAttend& a, void* ws, hipStream_t st);

}  // namespace luvc
