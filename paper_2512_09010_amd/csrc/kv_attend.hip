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
typedef float kv_f32x4 __attribute__((ext_vector_type(4)));
typedef float kv_f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
// of rows that start anywhere
template <typename T, int W> struct kv_piece_t;
template <> struct kv_piece_t<float, 4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct kv_piece_t<bf16_t, 4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct kv_piece_t<bf16_t, 2> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(2))); };
typedef int32_t kv_sizes4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kMaxSplits = 256;
constexpr float kLogE = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.0e38f;              // the maximum of nothing: finite, so that differences to it are no NaN

constexpr int attend_waves(int dp) { return dp == 256 ? 4 : 8; }        // what registers allow to be resident at two, one per SIMD

__device__ __forceinline__ float xor16(float v) { return __shfl_xor(v, 16, kWave); }
__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32, kWave); }

// W words from channel d of a row of D on; SMALL: D is less than 16 bytes, zeros behind it
template <typename T, int W, bool SMALL>
__device__ __forceinline__ void load_words(uint32_t* w, const T* rows, uint32_t row, int d, int D)
{
    if constexpr (!SMALL) {
        typedef typename kv_piece_t<T, W>::type piece;
        const piece p = *(const piece*)(rows + (row + (uint32_t)d));
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = p[i];
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
#pragma unroll
        for (int e = 0; e < W * 4 / (int)sizeof(T); ++e) {
            if (d + e >= D) continue;
            if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(((const float*)rows)[row + d + e]);
            else w[e / 2] |= (uint32_t)((const uint16_t*)rows)[row + d + e] << (e % 2 * 16);
        }
    }
}

struct KvWork {
    const int32_t* sizes;
    int n_pages, n_heads, log2_page, D, group, chunk, tiles, cols, parts_row;      // tiles of at most `cols` query heads; parts_row: floats
    int64_t rows;                    // sequences x cache heads
    float* parts;                    // [rows, tiles, splits, cols, parts_row]
    tile_tag_t* words;               // [rows, tiles]
    tile_tag_t tag;
    bool q_pieces;                   // queries in aligned 16-byte pieces
};

// DP: channels with room (64, 128, 256)
template <typename T, int DP, bool SMALL>
__global__ void __launch_bounds__(attend_waves(DP) * 64)
kv_attend(const T* __restrict__ kpool, const T* __restrict__ vpool, KvWork wk, KvAttend a)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int NW = attend_waves(DP), NT = NW * 64;
    constexpr int TILES = BF ? 2 : 1, TOK = 16 * TILES, STEP = NW * TOK;      // tokens of a wavefront's step, of the workgroup's
    constexpr int KE = BF ? 8 : 4;                            // elements in 16 bytes
    constexpr int NK = DP / (4 * KE);                         // pieces of a key per lane
    constexpr int VL = DP == 64 ? 4 : KE, VW = VL * (int)sizeof(T) / 4, NV = DP / (16 * VL);      // of a value: elements, words, pieces
    constexpr int VT = 4 * TILES;                             // tokens of a lane's part of the second sum
    constexpr int LD = DP + 4, QLD = DP + KE;                 // rows in LDS
    extern __shared__ __align__(16) float lds[];
    __shared__ float sm[NW][16], sl[NW][16];
    __shared__ int last_flag;

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // tiles of one sequence and cache head read the same rows: eight workgroups apart they meet in the L2 of one XCD
    const unsigned band = blockIdx.x / (8 * wk.tiles), in_band = blockIdx.x % (8 * wk.tiles);
    const int qt = in_band / 8;
    const int64_t row = (int64_t)band * 8 + in_band % 8;
    if (row >= wk.rows) return;
    const int h = (int)(row % wk.n_heads), s = (int)(row / wk.n_heads);
    const int split = blockIdx.y, D = wk.D, P1 = (1 << wk.log2_page) - 1;

    // what does not depend on one another is asked for together: the length, the first pages, the queries
    int64_t most = (int64_t)a.max_pages << wk.log2_page;
    const int room = most < a.max_tokens ? (int)most : a.max_tokens;
    const scalar_words table = as_scalars(a.table) + (int64_t)s * a.max_pages;
    int t0 = split * wk.chunk + wave * TOK;
    int now[TILES], next[TILES];
    auto pages_at = [&](int t, int* pages) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) pages[i] = t + 16 * i < room ? table[(t + 16 * i) >> wk.log2_page] : -1;
    };
    pages_at(t0, now);
    pages_at(t0 + STEP, next);
    int len = as_scalars(a.lengths)[s];
    // query heads head0 .. head0 + nh - 1 of the call are columns of the products, zeros behind them
    const int head0 = h * wk.group + qt * wk.cols, left = wk.group - qt * wk.cols, nh = left < wk.cols ? left : wk.cols;
    T* qs = (T*)lds;
    const T* q0 = (const T*)a.q + s * a.q_stride + (int64_t)head0 * D;
    if (wk.q_pieces) {
        constexpr int PIECES = DP / KE;
        for (int i = tid; i < 16 * PIECES; i += NT) {
            const int col = i / PIECES, d = i % PIECES * KE;
            kv_u32x4 w = {};
            if (col < nh && d < D) w = *(const kv_u32x4*)(q0 + col * D + d);
            *(kv_u32x4*)&qs[col * QLD + d] = w;
        }
    } else {
#pragma unroll 1
        for (int i = tid; i < 16 * DP; i += NT) {
            const int col = i / DP, d = i % DP;
            T w{};
            if (col < nh && d < D) w = q0[col * D + d];
            qs[col * QLD + d] = w;
        }
    }
    len = len < 0 ? 0 : len > room ? room : len;
    const int splits = len > wk.chunk ? (len + wk.chunk - 1) / wk.chunk : 1;
    if (split >= splits) return;
    tile_tag_t* word = wk.words + (row * wk.tiles + qt);
    tile_tag_t seen = 0;
    if (splits > 1 && tid == 0) seen = tag_load(word);
    const int end = split == splits - 1 ? len : (split + 1) * wk.chunk;

    // A piece that would reach beyond the row is the row's last one instead: what it repeats meets zeros among the queries, or is the
    // same channel of the output once more
    uint32_t kf[TILES][NK][4], vf[VT][NV][VW];
    kv_sizes4 sz[TILES];
    auto place = [&](int t, int page) -> int64_t {            // page and row as places of a head's tokens in the pool
        page = page >= 0 && page < wk.n_pages ? page : 0;
        return (((int64_t)page * wk.n_heads + h) << wk.log2_page) + (t & P1);
    };
    auto ask_keys = [&](int t, const int* pages) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const T* rows = kpool + place(t + 16 * i, pages[i]) * D;
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                int d = (4 * n + g) * KE;
                d = SMALL ? 0 : d < D - KE ? d : D - KE;
                load_words<T, 4, SMALL>(kf[i][n], rows, (uint32_t)(c * D), d, D);
            }
            if (wk.sizes) {
                const int page = pages[i] >= 0 && pages[i] < wk.n_pages ? pages[i] : 0;
                sz[i] = *(const kv_sizes4*)(wk.sizes + (((int64_t)page << wk.log2_page) + ((t + 16 * i) & P1)) + 4 * g);
            }
        }
    };
    auto ask_values = [&](int t, const int* pages) {
#pragma unroll
        for (int j = 0; j < VT; ++j) {
            const T* rows = vpool + (place(t + 16 * (j / 4), pages[j / 4]) + j % 4) * D;
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                int d = (16 * n + c) * VL;
                d = SMALL || d < D - VL ? d : D - VL;
                load_words<T, VW, SMALL>(vf[j][n], rows, (uint32_t)(4 * g * D), d, D);
            }
        }
    };
    if (t0 < end) {
        ask_keys(t0, now);
        ask_values(t0, now);
    }
    __syncthreads();                                          // the queries are in LDS
    uint32_t qf[NK][4];
#pragma unroll
    for (int n = 0; n < NK; ++n) {
        const int d0 = (4 * n + g) * KE, d1 = SMALL ? 0 : d0 < D - KE ? d0 : D - KE;
        if (d1 == d0) {
            const kv_u32x4 w = *(const kv_u32x4*)&qs[c * QLD + d0];
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[n][i] = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (BF) {
                    const int e = d1 + 2 * i;
                    qf[n][i] = (e >= d0 && e < D ? ((const uint16_t*)qs)[c * QLD + e] : 0u) | (e + 1 >= d0 && e + 1 < D ? (uint32_t)((const uint16_t*)qs)[c * QLD + e + 1] << 16 : 0u);
                } else {
                    const int e = d1 + i;
                    qf[n][i] = e >= d0 && e < D ? ((const uint32_t*)qs)[c * QLD + e] : 0u;
                }
            }
        }
    }

    kv_f32x4 o[NV * VL] = {};
    float m = kLowest, l = 0.f, ls = 0.f;
    const float scale = a.scale * kLogE;
    for (; t0 < end; t0 += STEP) {
        uint32_t live = 0;                                    // a bit for each of the lane's tokens
        float lg[VT] = {};
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const int n = now[i] >= 0 && now[i] < wk.n_pages ? end - (t0 + 16 * i + 4 * g) : 0;
            live |= (n >= 4 ? 15u : n > 0 ? (1u << n) - 1u : 0u) << (4 * i);
            if (wk.sizes) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (sz[i][e] < 1) live &= ~(1u << (4 * i + e));
                    if (a.enhance) lg[4 * i + e] = __log2f((float)(sz[i][e] < 1 ? 1 : sz[i][e]));
                }
            }
        }
        constexpr uint32_t ALL = (1u << VT) - 1u;
        const bool whole = __all(live == ALL);

        // logits, in powers of two
        float p[VT];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            kv_f32x4 z = {};
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                if constexpr (BF) {
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, *(kv_u32x4*)kf[i][n]), __builtin_bit_cast(kv_bf16x8, *(kv_u32x4*)qf[n]), z, 0, 0, 0);
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) z = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i][n][w]), __uint_as_float(qf[n][w]), z, 0, 0, 0);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) p[4 * i + e] = z[e] * scale;
        }
        // the next step's keys take the place of these while the weights are formed, its values that of the values after them
        const int tn = t0 + STEP;
        int after[TILES];
        pages_at(tn + STEP, after);
        if (tn < end) ask_keys(tn, next);
        if (!whole) {
#pragma unroll
            for (int j = 0; j < VT; ++j) p[j] = live >> j & 1 ? p[j] : -__builtin_inff();
        }
        float top = p[0];
#pragma unroll
        for (int j = 1; j < VT; ++j) top = fmaxf(top, p[j]);
        if (__any(top > m + 8.f)) {
            top = fmaxf(top, xor16(top));
            top = fmaxf(top, xor32(top));
            top = fmaxf(top, m);
            const float f = __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= f;
            ls *= f;
#pragma unroll
            for (int e = 0; e < NV * VL; ++e) o[e] *= f;
        }
#pragma unroll
        for (int j = 0; j < VT; ++j) {
            p[j] = __builtin_amdgcn_exp2f(p[j] - m);
            l += p[j];
            ls += p[j] * lg[j];
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
            kv_bf16x8 hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                hi[j] = (__bf16)p[j];
                lo[j] = (__bf16)(p[j] - (float)hi[j]);
            }
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int e = 0; e < VL; ++e) {
                    kv_u32x4 w;                               // channel e of the 8 tokens
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(vf[2 * j + 1][n][e / 2], vf[2 * j][n][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
                    kv_f32x4& acc = o[n * VL + e];
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, w), hi, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, w), lo, acc, 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int e = 0; e < VL; ++e)
#pragma unroll
                    for (int j = 0; j < VT; ++j)
                        o[n * VL + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[j][n][e]), p[j], o[n * VL + e], 0, 0, 0);
        }
        if (tn < end) ask_values(tn, next);
#pragma unroll
        for (int i = 0; i < TILES; ++i) { now[i] = next[i]; next[i] = after[i]; }
    }

    // ---- the wavefronts' parts; log s goes to every channel
    l += xor16(l);
    l += xor32(l);
    ls += xor16(ls);
    ls += xor32(ls);
    ls *= kLn2;
    if (g == 0) { sm[wave][c] = m; sl[wave][c] = l; }
    __syncthreads();                                          // the queries have been read
    if (c < nh) {
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int d = (16 * n + 4 * g + i) * VL;
                d = SMALL || d < D - VL ? d : D - VL;
                if (SMALL && d >= D) continue;
#pragma unroll
                for (int e = 0; e < VL; e += 4) {
                    kv_f32x4u w;
#pragma unroll
                    for (int b = 0; b < 4; ++b) w[b] = o[n * VL + e + b][i] + ls;
                    *(kv_f32x4u*)&lds[(wave * wk.cols + c) * LD + d + e] = w;
                }
            }
    }
    if (splits > 1 && tid == 0 && (seen >> 16) != wk.tag) {
        tile_tag_t expect = seen;
        (void)__hip_atomic_compare_exchange_strong(word, &expect, wk.tag << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    const int quads = (D + 3) / 4, items = nh * quads, part = wk.cols * wk.parts_row;
    float* parts = wk.parts + (row * wk.tiles + qt) * gridDim.y * part;
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(parts, 0, splits * part * 4, 0x00020000);
    auto store = [&](int col, int d, kv_f32x4 v) {
        T* out = (T*)a.out + s * a.out_stride + (int64_t)(head0 + col) * D + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (d + i >= D) continue;
            if constexpr (BF) out[i].bits = f32_to_bf16(v[i]);
            else out[i] = v[i];
        }
    };
    for (int i = tid; i < items; i += NT) {
        const int col = i / quads, d = i % quads * 4;
        float top = sm[0][col];
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, sm[w][col]);
        float sum = 0.f;
        kv_f32x4 v = {};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm[w][col] - top);
            sum += f * sl[w][col];
            v += f * *(const kv_f32x4*)&lds[(w * wk.cols + col) * LD + d];
        }
        if (splits == 1) {
            store(col, d, v * (sum > 0.f ? 1.f / sum : 0.f));
        } else {
            tile_vec<4>::store(__builtin_bit_cast(tile_vec<4>::type, v), all, (uint32_t)((split * part + col * wk.parts_row + d) * 4));
            if (d == 0)
                tile_vec<4>::store(tile_vec<4>::type{__float_as_uint(top), __float_as_uint(sum), 0u, 0u}, all, (uint32_t)((split * part + (col + 1) * wk.parts_row - 4) * 4));
        }
    }
    if (splits == 1) return;

    // ---- the runs of the sequence, by the workgroup that ends last
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) last_flag = tiles_arrive(word, splits);
    __syncthreads();
    if (!last_flag) return;
    float *weight = lds, *total = sl[0], *red = lds + kMaxSplits * 16;      // [splits][cols], [cols], [NT][4]
    // Few channels in all: several threads to four of them, each with every groups-th run.  The first AHEAD runs of a thread are asked for
    // together with the maxima and sums that their weights are formed of.
    constexpr int AHEAD = 16;
    const int groups = items < NT ? NT / items : 1;
    const int lane_item = groups > 1 ? tid % items : tid, grp = groups > 1 ? tid / items : 0;
    kv_f32x4 x[AHEAD];
    auto ask = [&](int i, int k0) {
        const int col = i / quads, d = i % quads * 4;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int run = k0 + k * groups;
            if (run < splits) x[k] = __builtin_bit_cast(kv_f32x4, tile_vec<4>::load(all, (uint32_t)((run * part + col * wk.parts_row + d) * 4)));
        }
    };
    const bool mine = lane_item < items && grp < groups;
    if (mine) ask(lane_item, grp);
    for (int col = wave; col < nh; col += NW) {
        float mx[kMaxSplits / 64], sx[kMaxSplits / 64], top = kLowest, sum = 0.f;
#pragma unroll
        for (int k = 0; k < kMaxSplits / 64; ++k) {
            const int i = lane + 64 * k;
            mx[k] = kLowest;
            sx[k] = 0.f;
            if (i < splits) {
                const tile_vec<4>::type w = tile_vec<4>::load(all, (uint32_t)((i * part + (col + 1) * wk.parts_row - 4) * 4));
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
            if (i < splits) weight[i * 16 + col] = f;
        }
        sum = wave_sum(sum);
        if (lane == 0) total[col] = sum > 0.f ? 1.f / sum : 0.f;
    }
    __syncthreads();
    for (int i0 = 0; i0 < items; i0 += NT) {
        const int i = i0 + lane_item, col = i / quads;
        const bool in = i < items && grp < groups;
        if (in && i0) ask(i, grp);
        kv_f32x4 v = {};
        for (int k0 = grp; in && k0 < splits; k0 += AHEAD * groups) {
            if (k0 != grp) ask(i, k0);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (k0 + k * groups < splits) v += weight[(k0 + k * groups) * 16 + col] * x[k];
        }
        if (groups > 1) {
            *(kv_f32x4*)&red[tid * 4] = v;
            __syncthreads();
            if (in && grp == 0)
                for (int k = 1; k < groups; ++k) v += *(const kv_f32x4*)&red[(k * items + i) * 4];
        }
        if (in && grp == 0) store(col, i % quads * 4, v * total[col]);
    }
}

// How a call is laid out: tiles of query heads, tokens of a run
struct AttendPlan {
    int dp, tiles, cols, chunk, splits, parts_row;
    int64_t rows;
    unsigned blocks;
    size_t words, bytes, lds;
};
AttendPlan attend_plan(int n_seqs, int n_q_heads, int n_heads, int D, luvc_dtype dt, int max_tokens)
{
    AttendPlan p;
    const int group = n_q_heads / n_heads, es = dt == LUVC_F32 ? 4 : 2;
    p.dp = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    p.tiles = (group + 15) / 16;
    p.cols = group < 16 ? group : 16;
    p.rows = (int64_t)n_seqs * n_heads;
    p.blocks = (unsigned)((p.rows + 7) / 8 * 8 * p.tiles);
    const int waves = attend_waves(p.dp), step = waves * (dt == LUVC_F32 ? 16 : 32);
    const int64_t want = (512 + p.rows * p.tiles - 1) / (p.rows * p.tiles);
    int64_t per = (max_tokens + want - 1) / want;
    per = per < 1024 ? per : 1024;
    if ((max_tokens + per - 1) / per > kMaxSplits) per = (max_tokens + kMaxSplits - 1) / kMaxSplits;
    p.chunk = (int)((per + step - 1) / step * step);
    p.splits = (max_tokens + p.chunk - 1) / p.chunk;
    p.parts_row = (D + 3) / 4 * 4 + 4;
    p.words = align_up((size_t)p.rows * p.tiles * sizeof(tile_tag_t));
    p.bytes = p.words + (p.splits > 1 ? align_up((size_t)p.rows * p.tiles * p.splits * p.cols * p.parts_row * sizeof(float)) : 0);
    // queries; parts of the wavefronts; weights of the runs and partial sums over them
    const size_t qs = (size_t)16 * (p.dp * es + 16), parts = (size_t)waves * p.cols * (p.dp + 4) * sizeof(float);
    const size_t join = p.splits > 1 ? (size_t)kMaxSplits * 16 * sizeof(float) + (size_t)waves * 64 * 16 : 0;
    p.lds = qs > parts ? qs : parts;
    p.lds = p.lds > join ? p.lds : join;
    return p;
}

template <typename T, int DP, bool SMALL>
void attend_launch(const AttendPlan& p, const luvc_kv_cache& c, int layer, const KvWork& wk, const KvAttend& a, hipStream_t st)
{
    LUVC_LAUNCH("kv_attend", (kv_attend<T, DP, SMALL>), dim3(p.blocks, p.splits), dim3(attend_waves(DP) * 64), p.lds, st,
                (const T*)c.k + layer * c.layer_stride, (const T*)c.v + layer * c.layer_stride, wk, a);
}

template <typename T>
void attend_shape(const AttendPlan& p, const luvc_kv_cache& c, int layer, const KvWork& wk, const KvAttend& a, hipStream_t st)
{
    if (c.D * sizeof(T) < 16) attend_launch<T, 64, true>(p, c, layer, wk, a, st);
    else if (p.dp == 64) attend_launch<T, 64, false>(p, c, layer, wk, a, st);
    else if (p.dp == 128) attend_launch<T, 128, false>(p, c, layer, wk, a, st);
    else attend_launch<T, 256, false>(p, c, layer, wk, a, st);
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
    const bool q_pieces = (c.D * es) % 16 == 0 && ((uintptr_t)a.q | (uint64_t)(a.q_stride * es)) % 16 == 0;
    const KvWork wk{c.sizes, c.n_pages, c.n_heads, kv_log2_page(c), c.D, a.n_q_heads / c.n_heads, p.chunk, p.tiles, p.cols, p.parts_row, p.rows,
                    (float*)((char*)ws + p.words), (tile_tag_t*)ws, spu_next_tag(), q_pieces};
    if (c.dtype == LUVC_F32) attend_shape<float>(p, c, layer, wk, a, st);
    else attend_shape<bf16_t>(p, c, layer, wk, a, st);
    return check_launch("attention over the cache");
}

}  // namespace luvc
