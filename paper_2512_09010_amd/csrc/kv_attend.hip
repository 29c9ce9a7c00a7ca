// Attention of one new token per sequence over the paged key-value cache (paper Section 3.2, Eq. 3: O = A (V + log s)).
//
//   z_j = scale <q, k_j>,  m = max z_j,  p_j = exp(z_j - m),  o = (sum p_j v_j + sum p_j log s_j) / sum p_j
//
// Every key and value is needed once per query head of its group, 4 G D operations for 2 D elements: HBM bounds it, and the work is to
// keep loads in flight.  A workgroup of four wavefronts takes a run of tokens of one sequence and cache head, a wavefront TOK
// of them at a time, with the running maximum and sum of the softmax; all query heads of the group are columns of its products:
//   S = K Q^T   a tile of 16 tokens x 16 heads (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32); K rows come from memory as
//               the operand wants them, 16 bytes of one token per lane
//   O += V^T P  the result of S is 4 tokens x 1 head per lane, which is what the second product wants of P if its sum over tokens
//               runs in that order; V comes row by row, whole rows to 16 neighbouring lanes, and in bf16 the
//               lane, which then has a few channels of the 8 tokens of its part of the sum, swaps halves of words to get 8 tokens of
//               a channel side by side.  Neither goes through LDS.
// Weights are bf16 for that product in two terms, p = hi + lo with an error of 2^-18: with hi alone the weights would be rounded as
// coarsely as the output, and the matrix cores have the time.
// The maximum is raised (and what has been summed scaled down) only when a logit exceeds it by more than 8 in powers of two: p stays
// below 256, and most steps do without an exchange between lanes.
// Tokens behind the end, without a page or of size below 1 get z = -inf and zeros for values, whatever their rows hold.
//
// The four wavefronts join through LDS.  A sequence longer than a run is joined by the workgroup of its runs that ends last, which adds
// in the order of the runs; hand-over and arrival words as in spu_tiles.hpp.
#include <type_traits>

#include "common.hpp"
#include "kv.hpp"
#include "spu_tiles.hpp"

namespace luvc {

namespace {

typedef __bf16 kv_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 kv_bf16x2 __attribute__((ext_vector_type(2)));
typedef float kv_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv_u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t kv_sizes4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kWaves = 4, kMaxSplits = 256;
constexpr float kLogE = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.0e38f;              // the maximum of nothing: finite, so that differences to it are no NaN

__device__ __forceinline__ float xor16(float v) { return __shfl_xor(v, 16, kWave); }
__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32, kWave); }

// W words of a row of D elements at channel d: in 16- or 8-byte pieces (VEC; D is a multiple of the pieces, and a piece behind the end
// is the row's first: its products are with zeros, or are not stored), or element by element
template <typename T, int W, bool VEC>
__device__ __forceinline__ void load_words(uint32_t* w, const T* row, uint32_t off, int d, int D, bool exact)
{
    constexpr int N = W * 4 / (int)sizeof(T);
    if constexpr (VEC) {
        const T* p = row + (exact || d < D ? off + (uint32_t)d : off);
        if constexpr (W == 4) *(kv_u32x4*)w = *(const kv_u32x4*)p;
        else *(kv_u32x2*)w = *(const kv_u32x2*)p;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (d + e >= D) continue;
            if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(((const float*)row)[off + d + e]);
            else w[e / 2] |= (uint32_t)((const uint16_t*)row)[off + d + e] << (e % 2 * 16);
        }
    }
}

struct KvWork {
    const int32_t* sizes;
    int n_pages, n_heads, log2_page, D, group, chunk, tiles, parts_row;      // tiles: of query heads per cache head; parts_row: floats
    float* parts;                    // [rows, splits, heads of a tile, parts_row]
    tile_tag_t* words;               // [rows]
    tile_tag_t tag;
};

// DP: channels with room (64, 128, 256); QT: tiles of 16 query heads
template <typename T, int DP, int QT, bool VEC>
__global__ void __launch_bounds__(256)
kv_attend(const T* __restrict__ kpool, const T* __restrict__ vpool, KvWork wk, KvAttend a)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int TILES = BF ? 2 : 1, TOK = 16 * TILES;       // tokens of a step
    constexpr int KE = BF ? 8 : 4;                            // elements in 16 bytes
    constexpr int NK = DP / (4 * KE);                         // pieces of a key per lane
    constexpr int VL = DP == 64 ? 4 : KE, VW = VL * (int)sizeof(T) / 4, NV = DP / (16 * VL);      // of a value: elements, words, pieces
    constexpr int VT = 4 * TILES;                             // tokens of a lane's part of the second sum
    constexpr int HEADS = 16 * QT, LD = DP + 4;
    __shared__ __align__(16) float so[kWaves * HEADS * LD];
    __shared__ float sm[kWaves][HEADS], sl[kWaves][HEADS];
    __shared__ __align__(16) float red[256 * 4];
    __shared__ int last_flag;

    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int row = blockIdx.x, qt = row % wk.tiles, sh = row / wk.tiles, h = sh % wk.n_heads, s = sh / wk.n_heads;
    const int split = blockIdx.y, D = wk.D, P1 = (1 << wk.log2_page) - 1;
    const bool exact = D == DP;

    int64_t room = (int64_t)a.max_pages << wk.log2_page;
    room = room < a.max_tokens ? room : a.max_tokens;
    int len = as_scalars(a.lengths)[s];
    len = len < 0 ? 0 : len > room ? (int)room : len;
    const int splits = len > wk.chunk ? (len + wk.chunk - 1) / wk.chunk : 1;
    if (split >= splits) return;
    tile_tag_t* word = wk.words + row;
    tile_tag_t seen = 0;
    if (splits > 1 && threadIdx.x == 0) seen = tag_load(word);
    const int end = split == splits - 1 ? len : (split + 1) * wk.chunk;

    // query heads head0 .. head0 + nh - 1 of the call: columns of the products, zeros behind them
    const int head0 = h * wk.group + qt * HEADS, left = wk.group - qt * HEADS, nh = left < HEADS ? left : HEADS;
    uint32_t qf[QT][NK][4];
#pragma unroll
    for (int u = 0; u < QT; ++u)
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            const int col = 16 * u + c, d = (4 * n + g) * KE;
#pragma unroll
            for (int w = 0; w < 4; ++w) qf[u][n][w] = 0;
            if (col < nh) load_words<T, 4, false>(qf[u][n], (const T*)a.q + s * a.q_stride + (int64_t)(head0 + col) * D, 0, d, D, false);
        }

    kv_f32x4 o[QT][NV * VL] = {};
    float m[QT], l[QT], ls[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) { m[u] = kLowest; l[u] = ls[u] = 0.f; }
    const float scale = a.scale * kLogE;
    const scalar_words table = as_scalars(a.table) + (int64_t)s * a.max_pages;
    auto page_at = [&](int t) { return t < end ? table[t >> wk.log2_page] : -1; };

    for (int t0 = split * wk.chunk + wave * TOK; t0 < end; t0 += kWaves * TOK) {
        uint32_t kf[TILES][NK][4], vf[VT][NV][VW];
        int64_t base[TILES], size_at[TILES];
        uint32_t live = 0;                                    // bit of each of the lane's tokens
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            int page = page_at(t0 + 16 * t);
            const bool ok = page >= 0 && page < wk.n_pages;
            page = ok ? page : 0;
            const int r = (t0 + 16 * t) & P1;
            base[t] = (((int64_t)page * wk.n_heads + h) << wk.log2_page) + r;
            size_at[t] = ((int64_t)page << wk.log2_page) + r;
            const int n = ok ? end - (t0 + 16 * t + 4 * g) : 0;
            live |= (n >= 4 ? 15u : n > 0 ? (1u << n) - 1u : 0u) << (4 * t);
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int n = 0; n < NK; ++n) load_words<T, 4, VEC>(kf[t][n], kpool + base[t] * D, (uint32_t)(c * D), (4 * n + g) * KE, D, exact);
#pragma unroll
        for (int j = 0; j < VT; ++j)
#pragma unroll
            for (int n = 0; n < NV; ++n) load_words<T, VW, VEC>(vf[j][n], vpool + base[j / 4] * D, (uint32_t)((4 * g + j % 4) * D), (16 * n + c) * VL, D, exact);
        float lg[VT] = {};
        if (wk.sizes) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const kv_sizes4 sz = *(const kv_sizes4*)(wk.sizes + size_at[t] + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (sz[i] < 1) live &= ~(1u << (4 * t + i));
                    if (a.enhance) lg[4 * t + i] = __log2f((float)(sz[i] < 1 ? 1 : sz[i]));
                }
            }
        }
        constexpr uint32_t ALL = (1u << VT) - 1u;
        const bool whole = __all(live == ALL);

        // logits, in powers of two
        float p[QT][VT];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                kv_f32x4 z = {};
#pragma unroll
                for (int n = 0; n < NK; ++n) {
                    if constexpr (BF) {
                        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, *(kv_u32x4*)kf[t][n]), __builtin_bit_cast(kv_bf16x8, *(kv_u32x4*)qf[u][n]), z, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int w = 0; w < 4; ++w) z = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[t][n][w]), __uint_as_float(qf[u][n][w]), z, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) p[u][4 * t + i] = z[i] * scale;
            }
            if (!whole) {
#pragma unroll
                for (int j = 0; j < VT; ++j) p[u][j] = live >> j & 1 ? p[u][j] : -__builtin_inff();
            }
            float top = p[u][0];
#pragma unroll
            for (int j = 1; j < VT; ++j) top = fmaxf(top, p[u][j]);
            if (__any(top > m[u] + 8.f)) {
                top = fmaxf(top, xor16(top));
                top = fmaxf(top, xor32(top));
                top = fmaxf(top, m[u]);
                const float f = __builtin_amdgcn_exp2f(m[u] - top);
                m[u] = top;
                l[u] *= f;
                ls[u] *= f;
#pragma unroll
                for (int e = 0; e < NV * VL; ++e) o[u][e] *= f;
            }
#pragma unroll
            for (int j = 0; j < VT; ++j) {
                p[u][j] = __builtin_amdgcn_exp2f(p[u][j] - m[u]);
                l[u] += p[u][j];
                ls[u] += p[u][j] * lg[j];
            }
        }
        if (!whole) {
#pragma unroll
            for (int j = 0; j < VT; ++j)
#pragma unroll
                for (int n = 0; n < NV; ++n)
#pragma unroll
                    for (int w = 0; w < VW; ++w) vf[j][n][w] = live >> j & 1 ? vf[j][n][w] : 0u;
        }
        if constexpr (BF) {
            kv_bf16x8 hi[QT], lo[QT];
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    hi[u][j] = (__bf16)p[u][j];
                    lo[u][j] = (__bf16)(p[u][j] - (float)hi[u][j]);
                }
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int e = 0; e < VL; ++e) {
                    kv_u32x4 w;                                // channel e of the 8 tokens
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(vf[2 * j + 1][n][e / 2], vf[2 * j][n][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        o[u][n * VL + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, w), hi[u], o[u][n * VL + e], 0, 0, 0);
                        o[u][n * VL + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, w), lo[u], o[u][n * VL + e], 0, 0, 0);
                    }
                }
        } else {
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int e = 0; e < VL; ++e)
#pragma unroll
                    for (int u = 0; u < QT; ++u)
#pragma unroll
                        for (int j = 0; j < VT; ++j)
                            o[u][n * VL + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[j][n][e]), p[u][j], o[u][n * VL + e], 0, 0, 0);
        }
    }

    // ---- the four wavefronts' parts; log s goes to every channel
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        l[u] += xor16(l[u]);
        l[u] += xor32(l[u]);
        ls[u] += xor16(ls[u]);
        ls[u] += xor32(ls[u]);
        ls[u] *= kLn2;
        const int col = 16 * u + c;
        if (g == 0) { sm[wave][col] = m[u]; sl[wave][col] = l[u]; }
        if (col < nh)
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < VL; e += 4) {
                        float4 w;
                        w.x = o[u][n * VL + e][i] + ls[u];
                        w.y = o[u][n * VL + e + 1][i] + ls[u];
                        w.z = o[u][n * VL + e + 2][i] + ls[u];
                        w.w = o[u][n * VL + e + 3][i] + ls[u];
                        *(float4*)&so[(wave * HEADS + col) * LD + (16 * n + 4 * g + i) * VL + e] = w;
                    }
    }
    if (splits > 1 && threadIdx.x == 0 && (seen >> 16) != wk.tag) {
        tile_tag_t expect = seen;
        (void)__hip_atomic_compare_exchange_strong(word, &expect, wk.tag << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    const int quads = (D + 3) / 4, items = nh * quads;
    float* mine = wk.parts + ((int64_t)row * gridDim.y + split) * HEADS * wk.parts_row;
    const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(mine, 0, HEADS * wk.parts_row * 4, 0x00020000);
    auto store = [&](int col, int d, float4 v) {
        T* out = (T*)a.out + s * a.out_stride + (int64_t)(head0 + col) * D + d;
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (d + i >= D) continue;
            if constexpr (BF) out[i].bits = f32_to_bf16(e[i]);
            else out[i] = e[i];
        }
    };
    for (int i = threadIdx.x; i < items; i += 256) {
        const int col = i / quads, d = i % quads * 4;
        float top = sm[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][col]);
        float sum = 0.f;
        float4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm[w][col] - top);
            const float4 x = *(const float4*)&so[(w * HEADS + col) * LD + d];
            sum += f * sl[w][col];
            v.x += f * x.x; v.y += f * x.y; v.z += f * x.z; v.w += f * x.w;
        }
        if (splits == 1) {
            const float r = sum > 0.f ? 1.f / sum : 0.f;
            store(col, d, float4{v.x * r, v.y * r, v.z * r, v.w * r});
        } else {
            tile_vec<4>::type w = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
            tile_vec<4>::store(w, to, (uint32_t)((col * wk.parts_row + d) * 4));
            if (d == 0) {
                w = tile_vec<4>::type{__float_as_uint(top), __float_as_uint(sum), 0u, 0u};
                tile_vec<4>::store(w, to, (uint32_t)((col * wk.parts_row + wk.parts_row - 4) * 4));
            }
        }
    }
    if (splits == 1) return;

    // ---- the runs of the sequence, by the workgroup that ends last
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) last_flag = tiles_arrive(word, splits);
    __syncthreads();
    if (!last_flag) return;
    const int part = HEADS * wk.parts_row;
    const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(wk.parts + (int64_t)row * gridDim.y * part, 0, splits * part * 4, 0x00020000);
    static_assert(kMaxSplits <= kWaves * LD, "weights of the runs fit");
    float* weight = so;                                        // [splits][HEADS]
    float* total = sl[0];
    for (int col = wave; col < nh; col += kWaves) {
        float mx[kMaxSplits / 64], sx[kMaxSplits / 64], top = kLowest, sum = 0.f;
#pragma unroll
        for (int k = 0; k < kMaxSplits / 64; ++k) {
            const int i = lane + 64 * k;
            mx[k] = kLowest;
            sx[k] = 0.f;
            if (i < splits) {
                const tile_vec<4>::type w = tile_vec<4>::load(from, (uint32_t)((i * part + col * wk.parts_row + wk.parts_row - 4) * 4));
                mx[k] = __uint_as_float(w[0]);
                sx[k] = __uint_as_float(w[1]);
            }
            top = fmaxf(top, mx[k]);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, kWave));
#pragma unroll
        for (int k = 0; k < kMaxSplits / 64; ++k) {
            const int i = lane + 64 * k;
            const float f = __builtin_amdgcn_exp2f(mx[k] - top);
            sum += f * sx[k];
            if (i < splits) weight[i * HEADS + col] = f;
        }
        sum = wave_sum(sum);
        if (lane == 0) total[col] = sum > 0.f ? 1.f / sum : 0.f;
    }
    __syncthreads();
    // few channels in all: several threads to four of them, each with every groups-th run
    const int groups = items < 256 ? 256 / items : 1;
    for (int i0 = 0; i0 < items; i0 += 256) {
        const int i = groups > 1 ? (int)threadIdx.x % items : i0 + (int)threadIdx.x, grp = groups > 1 ? (int)threadIdx.x / items : 0;
        const bool in = i < items && grp < groups;
        const int col = i / quads, d = i % quads * 4;
        float4 v = {0.f, 0.f, 0.f, 0.f};
        if (in) {
#pragma unroll 4
            for (int k = grp; k < splits; k += groups) {
                const tile_vec<4>::type w = tile_vec<4>::load(from, (uint32_t)((k * part + col * wk.parts_row + d) * 4));
                const float f = weight[k * HEADS + col];
                v.x += f * __uint_as_float(w[0]); v.y += f * __uint_as_float(w[1]); v.z += f * __uint_as_float(w[2]); v.w += f * __uint_as_float(w[3]);
            }
        }
        if (groups > 1) {
            *(float4*)&red[threadIdx.x * 4] = v;
            __syncthreads();
            if (in && grp == 0)
                for (int k = 1; k < groups; ++k) {
                    const float4 x = *(const float4*)&red[(k * items + i) * 4];
                    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                }
        }
        if (in && grp == 0) {
            const float r = total[col];
            store(col, d, float4{v.x * r, v.y * r, v.z * r, v.w * r});
        }
    }
}

// How a call is split: query heads of a workgroup, runs of a sequence
struct AttendPlan {
    int dp, qt, tiles, chunk, splits, parts_row;
    int64_t rows;
    size_t words, bytes;
};
AttendPlan attend_plan(int n_seqs, int n_q_heads, int n_heads, int D, luvc_dtype dt, int max_tokens)
{
    AttendPlan p;
    const int group = n_q_heads / n_heads;
    p.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    p.qt = group > 16 && p.dp < 256 ? 2 : 1;
    p.tiles = (group + 16 * p.qt - 1) / (16 * p.qt);
    p.rows = (int64_t)n_seqs * n_heads * p.tiles;
    const int64_t step = kWaves * (dt == LUVC_F32 ? 16 : 32);
    int64_t want = (512 + p.rows - 1) / p.rows, per = (max_tokens + want - 1) / want;
    per = per < 1024 ? per : 1024;
    if ((max_tokens + per - 1) / per > kMaxSplits) per = (max_tokens + kMaxSplits - 1) / kMaxSplits;
    p.chunk = (int)((per + step - 1) / step * step);
    p.splits = (max_tokens + p.chunk - 1) / p.chunk;
    p.parts_row = (D + 3) / 4 * 4 + 4;
    p.words = align_up((size_t)p.rows * sizeof(tile_tag_t));
    p.bytes = p.words + (p.splits > 1 ? align_up((size_t)p.rows * p.splits * 16 * p.qt * p.parts_row * sizeof(float)) : 0);
    return p;
}

template <typename T, int DP, int QT, bool VEC>
void attend_launch(const AttendPlan& p, const luvc_kv_cache& c, int layer, const KvWork& wk, const KvAttend& a, hipStream_t st)
{
    LUVC_LAUNCH("kv_attend", (kv_attend<T, DP, QT, VEC>), dim3((unsigned)p.rows, p.splits), dim3(256), 0, st,
                (const T*)c.k + layer * c.layer_stride, (const T*)c.v + layer * c.layer_stride, wk, a);
}

template <typename T, bool VEC>
void attend_shape(const AttendPlan& p, const luvc_kv_cache& c, int layer, const KvWork& wk, const KvAttend& a, hipStream_t st)
{
    if (p.dp == 64) { if (p.qt == 1) attend_launch<T, 64, 1, VEC>(p, c, layer, wk, a, st); else attend_launch<T, 64, 2, VEC>(p, c, layer, wk, a, st); }
    else if (p.dp == 128) { if (p.qt == 1) attend_launch<T, 128, 1, VEC>(p, c, layer, wk, a, st); else attend_launch<T, 128, 2, VEC>(p, c, layer, wk, a, st); }
    else attend_launch<T, 256, 1, VEC>(p, c, layer, wk, a, st);
}

}  // namespace

size_t kv_attend_workspace(int n_seqs, int n_q_heads, int n_heads, int D, luvc_dtype dt, int max_tokens)
{
    return attend_plan(n_seqs, n_q_heads, n_heads, D, dt, max_tokens).bytes;
}

luvc_status kv_attend_run(const luvc_kv_cache& c, int layer, const KvAttend& a, void* ws, hipStream_t st)
{
    const AttendPlan p = attend_plan(a.n_seqs, a.n_q_heads, c.n_heads, c.D, c.dtype, a.max_tokens);
    const int64_t es = (int64_t)kv_esize(c);
    const bool vec = (c.D * es) % 16 == 0 && ((uintptr_t)c.k | (uintptr_t)c.v | (uint64_t)(c.layer_stride * es)) % 16 == 0;
    KvWork wk{c.sizes, c.n_pages, c.n_heads, kv_log2_page(c), c.D, a.n_q_heads / c.n_heads, p.chunk, p.tiles, p.parts_row,
              (float*)((char*)ws + p.words), (tile_tag_t*)ws, spu_next_tag()};
    if (c.dtype == LUVC_F32) { if (vec) attend_shape<float, true>(p, c, layer, wk, a, st); else attend_shape<float, false>(p, c, layer, wk, a, st); }
    else                     { if (vec) attend_shape<bf16_t, true>(p, c, layer, wk, a, st); else attend_shape<bf16_t, false>(p, c, layer, wk, a, st); }
    return check_launch("attention over the cache");
}

}  // namespace luvc
