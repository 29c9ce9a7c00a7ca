// Attention of one new token per sequence over the paged key-value cache (paper Section 3.2, Eq. 3: O = A (V + log s)).
//
// A wavefront per query head goes through the tokens one after the other with the running maximum and sum of the softmax.
#include "common.hpp"
#include "kv.hpp"

namespace luvc {

template <typename T>
__global__ void __launch_bounds__(64)
kv_attend(const T* __restrict__ k, const T* __restrict__ v, const int32_t* __restrict__ sizes, int n_pages, int n_heads, int log2_page, int D, KvAttend a)
{
    using tr = io_traits<T>;
    const int lane = threadIdx.x, s = blockIdx.x / a.n_q_heads, h = blockIdx.x % a.n_q_heads;
    const int kv = h / (a.n_q_heads / n_heads), P = 1 << log2_page;
    const T* q = (const T*)a.q + s * a.q_stride + (int64_t)h * D;
    float qr[4], acc[4] = {}, m = -3.0e38f, l = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) qr[u] = lane + 64 * u < D ? tr::load(q + lane + 64 * u) * a.scale : 0.f;
    int64_t n = (int64_t)a.max_pages << log2_page;
    n = n < a.max_tokens ? n : a.max_tokens;
    n = n < a.lengths[s] ? n : a.lengths[s];
    for (int j = 0; j < n; ++j) {
        const int page = a.table[(int64_t)s * a.max_pages + (j >> log2_page)];
        if (page < 0 || page >= n_pages) continue;
        const int size = sizes ? sizes[((int64_t)page << log2_page) + (j & (P - 1))] : 1;
        if (size < 1) continue;
        const int64_t at = ((((int64_t)page * n_heads + kv) << log2_page) + (j & (P - 1))) * D;
        float dot = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (lane + 64 * u < D) dot += qr[u] * tr::load(k + at + lane + 64 * u);
        dot = wave_sum(dot);
        const float mn = fmaxf(m, dot), f = expf(m - mn), p = expf(dot - mn), ls = a.enhance ? logf((float)size) : 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (lane + 64 * u < D) acc[u] = acc[u] * f + p * (tr::load(v + at + lane + 64 * u) + ls);
        l = l * f + p;
        m = mn;
    }
    T* out = (T*)a.out + s * a.out_stride + (int64_t)h * D;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (lane + 64 * u < D) tr::store(out + lane + 64 * u, l > 0.f ? (double)(acc[u] / l) : 0.0);
}

size_t kv_attend_workspace(int n_seqs, int n_q_heads, int n_heads, int D, luvc_dtype dt, int max_tokens)
{
    (void)n_seqs, (void)n_q_heads, (void)n_heads, (void)D, (void)dt, (void)max_tokens;
    return 256;
}

luvc_status kv_attend_run(const luvc_kv_cache& c, int layer, const KvAttend& a, void* ws, hipStream_t st)
{
    (void)ws;
    const unsigned g = (unsigned)(a.n_seqs * a.n_q_heads);
#define LUVC_KV_ATTEND(T) LUVC_LAUNCH("kv_attend", (kv_attend<T>), dim3(g), dim3(64), 0, st, (const T*)c.k + layer * c.layer_stride, \
                                      (const T*)c.v + layer * c.layer_stride, c.sizes, c.n_pages, c.n_heads, kv_log2_page(c), c.D, a)
    if (c.dtype == LUVC_F32) LUVC_KV_ATTEND(float); else LUVC_KV_ATTEND(bf16_t);
#undef LUVC_KV_ATTEND
    return check_launch("attention over the cache");
}

}  // namespace luvc
