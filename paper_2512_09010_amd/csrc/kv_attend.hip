// Attention of one new token per sequence over the paged key-value cache (paper Section 3.2, Eq. 3: O = A (V + log s)).
//
//   z_j = scale <q, k_j>,  m = max z_j,  p_j = exp(z_j - m),  o = (sum p_j v_j + sum p_j log s_j) / sum p_j
//
// Every key and value is needed once, for 4 G D operations on 2 D elements (G query heads to a cache head): HBM bounds it, and the work is to
// keep loads in flight (64 sequences of 4096 tokens, 32 query heads on 8 of 128, bf16: 1.07 GB in 162 us, 6.6 TB/s, where a large copy
// reaches 5.1; one sequence of 100000, 4 heads: 205 MB in 38.4 us).  A workgroup of four wavefronts takes a run of tokens of one
// sequence and cache head, a wavefront TOK of them at a time, with the running maximum and sum of the softmax; all query heads of
// the group, up to 16, are columns of its products:
//   S = K Q^T   a tile of 16 tokens x 16 heads (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32); the rows of K are read as rows, and LDS,
//               a part of it for each wavefront, turns them into the operand, 16 bytes of one token per lane.  (Read as the operand
//               wants them, 16 tokens side by side, a step took 2.1 us instead of 1.2: 64 places to look up per load.)
//   O += V^T P  the result of S is 4 tokens x 1 head per lane, which is what the second product wants of P if its sum over tokens
//               runs in that order; V goes from memory to registers row by row, whole rows to 16 neighbouring lanes, and in bf16 the
//               lane, which then has a few channels of the 8 tokens of its part of the sum, swaps halves of words to get 8 tokens of
//               a channel side by side
// The next step's keys are asked for when this one's are in LDS, its values when this one's are used up; four wavefronts of a step each in
// flight, and two or three workgroups to a unit (one above 128 channels), keep memory busy (eight wavefronts to a workgroup were no faster, and
// their join slower).
// With bf16 the second product takes a weight in three bf16 terms, which together are its fp32 value: with one the weights would be rounded as
// coarsely as the output, with two by up to 2^-17, and the matrix cores have the time (64 x 4096: 161 us with two, 161 with three; where steps
// do without memory, nine tokens in ten dead, 55 and 58).
// The maximum is raised (and what has been summed scaled down) only when a logit exceeds it by more than 8 in powers of two: p stays
// below 256, and most steps do without an exchange between lanes.
// Tokens behind the end, without a page or of size below 1 get z = -inf and zeros for values, whatever their rows hold.
//
// The four wavefronts join through LDS.  A sequence longer than a run is joined by the workgroup of its runs that ends last, which adds
// in the order of the runs: the parts are written past the L2 of the XCD, an arrival word per sequence and head counts the workgroups.
// Short calls are bound by trips to memory: 4 us of the launch, then length and page, keys and values, the join's two (1 x 600 tokens: 7 us).
#include <algorithm>
#include <cmath>
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

constexpr int kMaxSplits = 768, kDirect = 32, kFan = 16;      // runs of a sequence: at most, joined at once at most, else in groups of
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.0e38f;              // the maximum of nothing: finite, so that differences to it are no NaN

constexpr int kWaves = 4;

__device__ __forceinline__ float xor16(float v) { return __shfl_xor(v, 16, kWave); }
__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32, kWave); }

// W words at a byte offset; SMALL: the row has D elements, fewer than 16 bytes hold, of which those from d on are taken, zeros behind them.
// Every row is used once: asked for so that it need not be kept (64 x 4096 tokens, 32 / 8 heads: 193 -> 170 us; short calls lose 0.2).
template <typename T, int W, bool SMALL>
__device__ __forceinline__ void load_words(uint32_t* w, const char* rows, uint32_t off, int d, int D)
{
    if constexpr (!SMALL) {
        typedef typename kv_piece_t<T, W>::type piece;
        const piece p = __builtin_nontemporal_load((const piece*)(rows + off));
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = p[i];
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
#pragma unroll
        for (int e = 0; e < W * 4 / (int)sizeof(T); ++e) {
            if (d + e >= D) continue;
            if constexpr (sizeof(T) == 4) w[e] = *(const uint32_t*)(rows + off + 4 * e);
            else w[e / 2] |= (uint32_t)*(const uint16_t*)(rows + off + 2 * e) << (e % 2 * 16);
        }
    }
}

struct KvWork {
    const int32_t* sizes;
    int n_pages, n_heads, log2_page, D, group, chunk, tiles, cols, parts_row;      // tiles of at most `cols` query heads; parts_row: floats
    int words_each;
    int lds_words;                   // where the maxima and sums of the wavefronts lie in LDS
    bool planned;                    // runs by the lengths: splits is not used then, and chunk
    unsigned rows, splits, units;    // sequences x cache heads; the most runs of one; runs of all in the grid
    float* parts;                    // [runs x heads x tiles, cols, parts_row], the runs of one head of a sequence one after the other
    tile_tag_t* words;               // [rows, tiles, words_each]
    tile_tag_t tag;
    float scale, scale_rest;         // of the logits, to powers of two, in two terms; positive
    int sign;                        // of the queries: -1, 0 (as if they were zero), 1
};

// Runs by the lengths, which every wavefront of the grid works out for itself: the steps of all sequences decide how many steps a run has.
// Cut for one workgroup to a compute unit where that makes runs of up to 16 steps, else for two, else for three: one too many is a
// unit with twice the work, so a few longer runs are tried before it goes on to the finer cut, which is kept however many come out.  A
// sequence's runs are of equal length.  Those of sequences with several come before the sequences of one run: the long ones first.
// Sequences of 1 to 32768 tokens, 16 of them, 4 heads of 128, bf16: 107 us without the third cut (544 runs for 512 places), 93 with it;
// 16 of 4096 in fp32, which fit two to a unit: 54 cut for three, 47 for two; five to a unit are no better, and 128 of 1024 take 50 for 43.
// Against runs by the bound on the lengths it is one more trip to memory, 0.7 us, and
//   64 sequences of 1 to 8200 tokens, 8 heads: 68.5 us by the bound (3500 of 4600 runs empty and others waiting for them), 55.5
//   300 of 1 to 2000 with a bound of 32768: 313, 202.  One of 4000 with a bound of 131072: 14.6, 9.4.  One of 32768 and no other: 28.1, 26.6
//   1000 of 100 with a bound of 4096, what it serves worst: 125, 130
// kFinest * kUnits / n_parts + n runs at most, n <= 1024 sequences.  Every 64th sequence belongs to a lane.
constexpr int kUnits = 256, kFinest = 3, kPlanSeqs = 1024;
struct RunOf { int seq, run, runs, chunk, len, before; };     // before: runs of the sequences in front
inline __host__ __device__ int plan_runs(int n_parts) { return (kFinest * kUnits + n_parts - 1) / n_parts; }
__device__ __forceinline__ RunOf run_by_lengths(const int32_t* lengths, int n, int x, int room, int step, int n_parts, int lane)
{
    const int per = (n + 63) / 64;
    int len[kPlanSeqs / 64], runs[kPlanSeqs / 64];
    float steps = 0.f;
#pragma unroll
    for (int k = 0; k < kPlanSeqs / 64; ++k) {
        if (k >= per) break;
        const int i = 64 * k + lane;
        const int l = i < n ? lengths[i] : -1;
        len[k] = i >= n ? -1 : l < 0 ? 0 : l > room ? room : l;
        steps += (float)((len[k] + step - 1) / step);
    }
    // no rounding of the sum may make it smaller than it is: the runs have to fit the grid (a cut that would fit exactly is one step longer so)
    steps = wave_sum(steps) * 1.0001f;
    // workgroups to a unit that the runs are cut for; more than kUnits of each have no chance where there are more sequences
    const float one = steps * (float)n_parts / kUnits;
    int fine = n * n_parts > 2 * kUnits ? kFinest : one <= 16.f && n * n_parts <= kUnits ? 1 : 2, tries = 3;
    auto cut = [&]() { return (int)ceilf(fine == kFinest ? steps / (float)plan_runs(n_parts) : fine == 1 ? one : one * 0.5f); };
    int each = cut();
    uint32_t mine, upto, total;
    for (;;) {
        mine = 0;                                             // runs of sequences with several, sequences with one
#pragma unroll
        for (int k = 0; k < kPlanSeqs / 64; ++k) {
            if (k >= per) break;
            const int a = (len[k] + step - 1) / step;
            runs[k] = len[k] < 0 ? 0 : a <= each ? 1 : (a + each - 1) / each;
            mine += runs[k] > 1 ? (uint32_t)runs[k] << 16 : (uint32_t)runs[k];
        }
        upto = wave_scan_incl(mine);
        total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        if (fine == kFinest || (int)((total >> 16) + (total & 0xffffu)) * n_parts <= fine * kUnits) break;
        if (--tries) {
            each += each < 10 ? 1 : each / 10;
        } else {
            ++fine;
            tries = 3;
            each = cut();
        }
    }
    const int several = (int)(total >> 16);
    RunOf r{-1, 0, 0, 0, 0, 0};
    if (x >= several + (int)(total & 0xffffu)) return r;
    const bool long_one = x < several;
    const int y = long_one ? x : x - several;
    int at = long_one ? (int)((upto - mine) >> 16) : (int)((upto - mine) & 0xffffu);
    bool found = false;
#pragma unroll
    for (int k = 0; k < kPlanSeqs / 64; ++k) {
        if (k >= per) break;
        const int here = (runs[k] > 1) == long_one ? runs[k] : 0;
        if (y >= at && y < at + here) {
            found = true;
            r = RunOf{64 * k + lane, y - at, here, 0, len[k], at + (long_one ? 0 : several)};
        }
        at += here;
    }
    const int src = __ffsll((long long)__ballot(found)) - 1;
    r.seq = __builtin_amdgcn_readlane(r.seq, src);
    r.run = __builtin_amdgcn_readlane(r.run, src);
    r.runs = __builtin_amdgcn_readlane(r.runs, src);
    r.len = __builtin_amdgcn_readlane(r.len, src);
    r.before = __builtin_amdgcn_readlane(r.before, src);
    const int a = (r.len + step - 1) / step;
    r.chunk = (a + r.runs - 1) / r.runs * step;
    return r;
}

// DP: channels with room (64, 128, 256); SMALL: rows shorter than 16 bytes; SIZED: the cache has sizes
template <typename T, int DP, bool SMALL, bool SIZED>
__global__ void __launch_bounds__(kWaves * 64, DP == 256 ? 1 : DP == 64 ? 4 : sizeof(T) == 4 ? 2 : 3)
kv_attend(const T* __restrict__ kpool, const T* __restrict__ vpool, KvWork wk, KvAttend a)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int ES = (int)sizeof(T), NW = kWaves, NT = NW * 64;
    constexpr int TILES = BF ? 2 : 1, TOK = 16 * TILES, STEP = NW * TOK;      // tokens of a wavefront's step, of the workgroup's
    constexpr int KE = 16 / ES;                               // elements in 16 bytes
    constexpr int NK = DP / (4 * KE);                         // pieces of a key per lane
    constexpr int VL = DP == 64 ? 4 : KE, VW = VL * ES / 4, NV = DP / (16 * VL);      // of a value: elements, words, pieces
    constexpr int VT = 4 * TILES;                             // tokens of a lane's part of the second sum
    constexpr int LD = DP + 4, PIECES = DP / KE;              // a row of outputs in LDS; pieces of a query or a key
    constexpr int KU = PIECES / 4, SWZ = PIECES < 16 ? PIECES - 1 : 15;       // loads of a tile of keys, 64 pieces each
    // In LDS, one after the other: the wavefronts' keys, queries; then parts of the outputs; then partial sums of the join
    extern __shared__ __align__(16) char lds[];
    float(*sm)[16] = (float(*)[16])(lds + wk.lds_words), (*sl)[16] = sm + NW;
    int& last_flag = *(int*)(sl + NW);

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // tiles of one run read the same tokens: eight workgroups apart they meet in the L2 of one XCD
    const unsigned band = blockIdx.x / (8 * wk.tiles), in_band = blockIdx.x % (8 * wk.tiles), unit = band * 8 + in_band % 8;
    const int qt = in_band / 8, D = wk.D;
    if (unit >= wk.units) return;
    const int64_t held = (int64_t)a.max_pages << wk.log2_page;
    const int room = held < a.max_tokens ? (int)held : a.max_tokens;
    // Which run of which sequence and cache head: by the lengths, or, where there is little to cut or much too much, by the bound on them
    int s, h, split, splits = 0, chunk = wk.chunk, len;
    int64_t slot;                                             // of the sequence's first run among the parts
    if (wk.planned) {
        const RunOf r = run_by_lengths(a.lengths, a.n_seqs, unit / wk.n_heads, room, STEP, wk.n_heads * wk.tiles, lane);
        if (r.seq < 0) return;
        s = r.seq;
        h = unit % wk.n_heads;
        split = r.run;
        splits = r.runs;
        chunk = r.chunk;
        len = r.len;
        slot = (int64_t)r.before * (wk.n_heads * wk.tiles) + (h * wk.tiles + qt) * splits;
    } else {
        const int row = unit % wk.rows;
        split = unit / wk.rows;
        h = row % wk.n_heads;
        s = row / wk.n_heads;
        len = as_scalars(a.lengths)[s];
        slot = ((int64_t)row * wk.tiles + qt) * wk.splits;
    }

    // what does not depend on one another is asked for together: the length, the first pages, the queries
    const scalar_words table = as_scalars(a.table) + (int64_t)s * a.max_pages;
    int t0 = split * chunk + wave * TOK;
    struct Pages { int first, second; };                      // of a step's tiles
    auto page_at = [&](int t) { return table[(t < room ? t : room - 1) >> wk.log2_page]; };      // behind the end any will do: nothing there is live
    auto pages_at = [&](int t) { return Pages{page_at(t), TILES > 1 ? page_at(t + 16) : 0}; };
    const Pages pages0 = pages_at(t0);
    Pages pages1 = pages_at(t0 + STEP), pages2 = pages_at(t0 + 2 * STEP);
    // Query heads head0 .. head0 + nh - 1 of the call are columns of the products, zeros behind them.  A piece that would reach beyond a
    // row, of queries, keys or values, is the row's last one instead: what it repeats is zero among the queries, and of the values
    // it makes the same channels of the output once more.
    const int head0 = h * wk.group + qt * wk.cols, left = wk.group - qt * wk.cols, nh = left < wk.cols ? left : wk.cols;
    char* const queries = lds + NW * TOK * PIECES * 16;
    const char* q0 = (const char*)((const T*)a.q + s * a.q_stride + (int64_t)head0 * D);
    for (int i = tid; i < 16 * PIECES; i += NT) {
        const int col = i / PIECES, d0 = i % PIECES * KE, d1 = SMALL ? 0 : d0 < D - KE ? d0 : D - KE;
        uint32_t w[4] = {};
        if (col < nh && d0 < D && wk.sign) {
            load_words<T, 4, SMALL>(w, q0, (uint32_t)((col * D + d1) * ES), d1, D);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (BF) w[e] &= (d1 + 2 * e >= d0 ? 0xffffu : 0u) | (d1 + 2 * e + 1 >= d0 ? 0xffff0000u : 0u);
                else w[e] &= d1 + e >= d0 ? 0xffffffffu : 0u;
                w[e] ^= wk.sign < 0 ? (BF ? 0x80008000u : 0x80000000u) : 0u;
            }
        }
        *(kv_u32x4*)(queries + (col * (PIECES + 1) + i % PIECES) * 16) = kv_u32x4{w[0], w[1], w[2], w[3]};
    }
    if (!wk.planned) {
        len = len < 0 ? 0 : len > room ? room : len;
        splits = len > chunk ? (len + chunk - 1) / chunk : 1;
        if (split >= splits) return;
    }
    // Arrival words: the sequence's, then those of its groups of runs.  A word is the launch's tag and a count; one without the tag, whatever an
    // earlier launch or anything else left there, is taken over by whoever may come to it first (thread 0: the word of this run; thread 1 of a
    // group's first run: the sequence's, to which the group comes when all of it has arrived), and whoever completes a count leaves zero
    // behind, so that a captured launch starts over the same way.
    const bool grouped = splits > kDirect;
    tile_tag_t* const words = wk.words + (((int64_t)s * wk.n_heads + h) * wk.tiles + qt) * wk.words_each;
    tile_tag_t* word = words + (grouped ? 1 + split / kFan : 0);
    tile_tag_t* const claimed = splits > 1 && tid == 0 ? word : grouped && tid == 1 && split % kFan == 0 ? words : nullptr;
    const tile_tag_t seen = claimed ? tag_load(claimed) : 0;
    const int end = split == splits - 1 ? len : (split + 1) * chunk;

    // Keys as the product wants them, 16 bytes of one token per lane and the tokens in neighbouring lanes, would be 64 places to look
    // up per load; as neighbouring lanes read them here, rows, they are 16 or fewer, and LDS turns them round.  Piece p of row r lies at
    // p ^ (r % 16) of its row there, so that the 16 rows of one read meet different banks.
    uint32_t kr[TILES][KU][4], vf[VT][NV][VW];
    uint32_t k_off[KU], v_off[4][NV];                         // bytes from the first row of a tile
    char* const keys = lds + wave * (TOK * PIECES * 16);
#pragma unroll
    for (int u = 0; u < KU; ++u) {
        const int r = (64 * u + lane) / PIECES, d = ((lane % PIECES) ^ (r & SWZ)) * KE;
        k_off[u] = (uint32_t)((r * D + (SMALL ? 0 : d < D - KE ? d : D - KE)) * ES);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int d = (16 * n + c) * VL;
            v_off[j][n] = (uint32_t)(((4 * g + j) * D + (SMALL || d < D - VL ? d : D - VL)) * ES);
        }
    const uint32_t row_bytes = (uint32_t)(D * ES), P1 = (1u << wk.log2_page) - 1, page_bytes = (uint32_t)wk.n_heads * row_bytes << wk.log2_page;
    const char* const k0 = (const char*)kpool + ((uint64_t)h * row_bytes << wk.log2_page);
    const char* const v0 = (const char*)vpool + ((uint64_t)h * row_bytes << wk.log2_page);
    auto held_at = [&](int page) { return (uint32_t)page < (uint32_t)wk.n_pages; };
    // One bit for each token of a step that takes part.  With sizes, rows of the others are not read: the request goes to the tile's
    // first bytes instead (a prompt pruned in place may have nine such tokens in ten).  The step is taken all the same: 64 x 4096 tokens take
    // 162 us with none dead, 89 with half of them, 58 with nine in ten, whose bytes take 16.
    constexpr uint32_t ALL = BF ? 0xffffffffu : 0xffffu;
    auto live_at = [&](int t, Pages pg, int size) -> uint32_t {
        const int n = end - t;
        uint32_t m = n >= TOK ? ALL : n > 0 ? (1u << n) - 1u : 0u;
        m &= held_at(pg.first) ? ALL : 0xffff0000u;
        if constexpr (TILES > 1) m &= held_at(pg.second) ? ALL : 0xffffu;
        if constexpr (SIZED) m &= (uint32_t)__ballot(size >= 1);
        return m;
    };
    auto ask_size = [&](int t, Pages pg) -> int {             // of token `lane` of a step
        if constexpr (!SIZED) return 1;
        const uint32_t first = held_at(pg.first) ? pg.first : 0, second = held_at(pg.second) ? pg.second : 0;
        const uint64_t at0 = ((uint64_t)first << wk.log2_page) + ((uint32_t)t & P1), at1 = ((uint64_t)second << wk.log2_page) + ((uint32_t)(t + 16) & P1);
        return wk.sizes[(TILES > 1 && (lane & 16) ? at1 : at0) + (lane & 15)];
    };
    uint64_t tile[TILES];                                     // bytes to the tiles of the step that is asked for
    auto ask_keys = [&](int t, Pages pg, uint32_t live) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {                     // without a page, page 0: its tokens are then not live
            const int page = i ? pg.second : pg.first;
            const uint32_t p = held_at(page) ? page : 0, r = (uint32_t)(t + 16 * i) & P1;
            tile[i] = (uint64_t)p * page_bytes + r * row_bytes;
#pragma unroll
            for (int u = 0; u < KU; ++u) {
                uint32_t off = k_off[u];
                if constexpr (SIZED) off &= (uint32_t)__builtin_amdgcn_sbfe((int)(live >> (16 * i + 64 * u / PIECES)), lane / PIECES, 1);
                load_words<T, 4, SMALL>(kr[i][u], k0 + tile[i], off, ((lane % PIECES) ^ (((64 * u + lane) / PIECES) & SWZ)) * KE, D);
            }
        }
    };
    auto ask_values = [&](uint32_t live) {
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t on = SIZED ? (uint32_t)__builtin_amdgcn_sbfe((int)(live >> (16 * i + j)), 4 * g, 1) : ~0u;
#pragma unroll
                for (int n = 0; n < NV; ++n) load_words<T, VW, SMALL>(vf[4 * i + j][n], v0 + tile[i], SIZED ? v_off[j][n] & on : v_off[j][n], (16 * n + c) * VL, D);
            }
    };
    int size = 1, size_next = 1;
    if (t0 < end) {
        size = ask_size(t0, pages0);
        size_next = ask_size(t0 + STEP, pages1);
        ask_keys(t0, pages0, ~0u);
        ask_values(~0u);
    }
    __syncthreads();                                          // the queries are in LDS
    // Read from there at every step; kept where the sizes' variant has the registers (8 x 1100 tokens: 9.1 us for 9.3; kept in both, the other
    // one's 128 channels go to scratch memory, 64 x 4096: 170 us for 161)
    constexpr bool KEEP = SIZED;
    auto query = [&](int n) { return *(const kv_u32x4*)(queries + (c * (PIECES + 1) + 4 * n + g) * 16); };
    kv_u32x4 kept[KEEP ? NK : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int n = 0; n < NK; ++n) kept[n] = query(n);
    }
    kv_f32x4 o[NV * VL] = {};
    float m = kLowest, l = 0.f, ls = 0.f;
    uint32_t live = live_at(t0, pages0, size);
    // MORE: the next step's keys take the place of this one's while the weights are formed, its values that of the values after them.
    // A step without a successor is code of its own: with the requests behind a condition, the wait for the values would have to be one
    // for everything in flight.
    auto step = [&](auto MORE) {
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int u = 0; u < KU; ++u)
                *(kv_u32x4*)(keys + (i * 16 * PIECES + 64 * u + lane) * 16) = kv_u32x4{kr[i][u][0], kr[i][u][1], kr[i][u][2], kr[i][u][3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // logits but for the scale
        float p[VT];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            // fp32: four sums side by side, which end four times sooner than one and round a quarter as often
            kv_f32x4 z[BF ? 1 : 4] = {};
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                const kv_u32x4 kf = *(const kv_u32x4*)(keys + (i * 16 + c) * PIECES * 16 + (((4 * n + g) ^ (c & SWZ)) * 16));
                const kv_u32x4 qf = KEEP ? kept[KEEP ? n : 0] : query(n);
                if constexpr (BF) {
                    z[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, kf), __builtin_bit_cast(kv_bf16x8, qf), z[0], 0, 0, 0);
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) z[w] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[w]), __uint_as_float(qf[w]), z[w], 0, 0, 0);
                }
            }
            if constexpr (!BF) z[0] = (z[0] + z[1]) + (z[2] + z[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[4 * i + e] = z[0][e];
        }
        uint32_t live_next = 0;
        int size_after = 1;
        Pages pages3{};
        if constexpr (MORE) {
            live_next = live_at(t0 + STEP, pages1, size_next);
            pages3 = pages_at(t0 + 3 * STEP);
            size_after = ask_size(t0 + 2 * STEP, pages2);
            ask_keys(t0 + STEP, pages1, live_next);
        }
        const uint32_t mine = live >> (4 * g);                // bits 0 .. 3, 16 .. 19: the lane's tokens
        auto on = [&](int j) { return mine >> (j % 4 + 16 * (j / 4)) & 1; };
        if (live != ALL) {
#pragma unroll
            for (int j = 0; j < VT; ++j) p[j] = on(j) ? p[j] : -__builtin_inff();
        }
        float top = p[0];
#pragma unroll
        for (int j = 1; j < VT; ++j) top = fmaxf(top, p[j]);
        top *= wk.scale;
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
        for (int j = 0; j < VT; ++j) p[j] = __builtin_amdgcn_exp2f(BF ? fmaf(p[j], wk.scale, -m) : fmaf(p[j], wk.scale_rest, fmaf(p[j], wk.scale, -m)));
        if (live != ALL) {
#pragma unroll
            for (int j = 0; j < VT; ++j) p[j] = on(j) ? p[j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < VT; ++j) l += p[j];
        if (SIZED && a.enhance) {
            const float lg = __log2f((float)(size < 1 ? 1 : size));
#pragma unroll
            for (int j = 0; j < VT; ++j) ls += p[j] * __shfl(lg, 4 * g + j % 4 + 16 * (j / 4), kWave);
        }
        if (live != ALL) {
#pragma unroll
            for (int j = 0; j < VT; ++j)
#pragma unroll
                for (int n = 0; n < NV; ++n)
#pragma unroll
                    for (int w = 0; w < VW; ++w) vf[j][n][w] = on(j) ? vf[j][n][w] : 0u;
        }
        if constexpr (BF) {
            kv_bf16x8 term[3];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float rest = p[j];
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    term[i][j] = (__bf16)rest;
                    rest -= (float)term[i][j];
                }
            }
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int e = 0; e < VL; ++e) {
                    kv_u32x4 w;                               // channel e of the 8 tokens
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(vf[2 * j + 1][n][e / 2], vf[2 * j][n][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
                    kv_f32x4& acc = o[n * VL + e];
#pragma unroll
                    for (int i = 0; i < 3; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(kv_bf16x8, w), term[i], acc, 0, 0, 0);
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
        if constexpr (MORE) {
            ask_values(live_next);
            live = live_next;
            size = size_next;
            size_next = size_after;
            pages1 = pages2;
            pages2 = pages3;
        }
    };
    for (; t0 + STEP < end; t0 += STEP) step(std::true_type{});
    if (t0 < end) step(std::false_type{});

    // ---- the wavefronts' parts; log s goes to every channel
    l += xor16(l);
    l += xor32(l);
    ls += xor16(ls);
    ls += xor32(ls);
    ls *= kLn2;
    if (g == 0) { sm[wave][c] = m; sl[wave][c] = l; }
    __syncthreads();                                          // queries and keys have been read
    float* const so = (float*)lds;
    if (c < nh) {
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < VL; e += 4) {
                    kv_f32x4 w;
#pragma unroll
                    for (int b = 0; b < 4; ++b) w[b] = o[n * VL + e + b][i] + ls;
                    *(kv_f32x4*)&so[(wave * wk.cols + c) * LD + (16 * n + 4 * g + i) * VL + e] = w;
                }
    }
    if (claimed && (seen >> 16) != wk.tag) {
        tile_tag_t expect = seen;
        (void)__hip_atomic_compare_exchange_strong(claimed, &expect, wk.tag << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    // Four channels of a head to a thread, in the order of heads of DP channels; further rows of threads, where heads are few, share runs
    constexpr int QUADS = DP / 4;
    const int log2_items = 31 - __builtin_clz(QUADS) + (nh > 1 ? 32 - __builtin_clz(nh - 1) : 0), part = wk.cols * wk.parts_row;
    const int groups = (1 << log2_items) < NT ? NT >> log2_items : 1, grp = groups > 1 ? tid >> log2_items : 0;
    const int item0 = groups > 1 ? tid & ((1 << log2_items) - 1) : tid;
    float* parts = wk.parts + slot * part;
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(parts, 0, splits * part * 4, 0x00020000);
    auto store = [&](int col, int d, kv_f32x4 v) {
        T* out = (T*)a.out + s * a.out_stride + (int64_t)(head0 + col) * D + d;
        if (d + 4 <= D) {
            if constexpr (BF) {
                typedef uint16_t quad __attribute__((ext_vector_type(4), aligned(2)));
                *(quad*)out = quad{f32_to_bf16(v[0]), f32_to_bf16(v[1]), f32_to_bf16(v[2]), f32_to_bf16(v[3])};
            } else {
                *(kv_f32x4u*)out = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                if (d + i >= D) continue;
                if constexpr (BF) out[i].bits = f32_to_bf16(v[i]);
                else out[i] = v[i];
            }
        }
    };
    // channels d .. d + 3 of a wavefront's part: the piece that would reach beyond the row holds the row's last channels
    const int even = SMALL ? DP : D / VL * VL;
    auto part_of = [&](const float* row_part, int d) {
        if (d + 4 <= even) return *(const kv_f32x4*)(row_part + d);
        kv_f32x4 v;
#pragma unroll
        for (int b = 0; b < 4; ++b) v[b] = row_part[d + b < even ? d + b : d + b < D ? d + b + VL - (D - even) : 0];
        return v;
    };
    struct Sum {                                              // weighted values, their weights' sum, and the maximum both refer to
        float top, sum;
        kv_f32x4 v;
        __device__ __forceinline__ void add(float m, float l, kv_f32x4 x)
        {
            const float t = fmaxf(top, m), f = __builtin_amdgcn_exp2f(top - t), w = __builtin_amdgcn_exp2f(m - t);
            top = t;
            sum = sum * f + l * w;
            v = v * f + x * w;
        }
        __device__ __forceinline__ kv_f32x4 mean() const { return v * (sum > 0.f ? 1.f / sum : 0.f); }
    };
    auto keep = [&](int run, int col, int d, const Sum& t) {
        const uint32_t at = (uint32_t)((run * part + col * wk.parts_row) * 4);
        tile_vec<4>::store(__builtin_bit_cast(tile_vec<4>::type, t.v), all, at + d * 4);
        if (d == 0) tile_vec<2>::store(tile_vec<2>::type{__float_as_uint(t.top), __float_as_uint(t.sum)}, all, at + (wk.parts_row - 4) * 4);
    };
    if (grp == 0)
        for (int i = item0; i < nh * QUADS; i += NT) {
            const int col = i / QUADS, d = i % QUADS * 4;
            if (d >= D) continue;
            Sum t{sm[0][col], sl[0][col], part_of(&so[col * LD], d)};
#pragma unroll
            for (int w = 1; w < NW; ++w) t.add(sm[w][col], sl[w][col], part_of(&so[(w * wk.cols + col) * LD], d));
            if (splits == 1) store(col, d, t.mean());
            else keep(split, col, d, t);
        }
    if (splits == 1) return;

    // ---- the runs of the sequence, or first those of its groups, by the workgroup that ends last
    int first = grouped ? split / kFan * kFan : 0, runs = !grouped ? splits : splits - first < kFan ? splits - first : kFan, apart = 1;
    for (bool done = !grouped;; done = true) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            const tile_tag_t old = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last_flag = (int)(old & 0xffffu) == runs - 1;
            if (last_flag) tag_store(word, 0ull);
        }
        __syncthreads();
        if (!last_flag) return;
        // AHEAD runs of a thread in flight, of one set of four channels or of several where there are more than threads
        auto join = [&](auto SETS, int i0) {
            constexpr int S = decltype(SETS)::value, AHEAD = 8;
            int col[S], d[S];
            bool in[S];
            uint32_t at[S];
            Sum t[S];
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const int i = i0 + j * NT + item0;
                col[j] = i / QUADS;
                d[j] = i % QUADS * 4;
                in[j] = col[j] < nh && d[j] < D;
                at[j] = (uint32_t)((first * part + (in[j] ? col[j] * wk.parts_row : 0)) * 4);
                t[j] = Sum{kLowest, 0.f, {}};
            }
#pragma unroll 1
            for (int k0 = grp; k0 < runs; k0 += AHEAD * groups) {
                tile_vec<4>::type x[S][AHEAD];
                tile_vec<2>::type ml[S][AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int run = k0 + k * groups;
                    const uint32_t from = (uint32_t)((run < runs ? run : runs - 1) * apart * part * 4);
#pragma unroll
                    for (int j = 0; j < S; ++j) {
                        x[j][k] = tile_vec<4>::load(all, from + at[j] + (in[j] ? d[j] * 4 : 0));
                        ml[j][k] = tile_vec<2>::load(all, from + at[j] + (wk.parts_row - 4) * 4);
                    }
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const bool there = k0 + k * groups < runs;
#pragma unroll
                    for (int j = 0; j < S; ++j)
                        t[j].add(there ? __uint_as_float(ml[j][k][0]) : kLowest, there ? __uint_as_float(ml[j][k][1]) : 0.f, there ? __builtin_bit_cast(kv_f32x4, x[j][k]) : kv_f32x4{});
                }
            }
            if (S == 1 && groups > 1) {                       // nh * QUADS < NT: one round
                float* red = so + tid * 8;
                *(kv_f32x4*)red = t[0].v;
                red[4] = t[0].top;
                red[5] = t[0].sum;
                __syncthreads();
#pragma unroll 1
                for (int k = 1; grp == 0 && k < groups; ++k) {
                    red += 8 << log2_items;
                    t[0].add(red[4], red[5], *(const kv_f32x4*)red);
                }
            }
#pragma unroll
            for (int j = 0; j < S; ++j) {
                if (!in[j] || grp) continue;
                if (done) store(col[j], d[j], t[j].mean());
                else keep(first, col[j], d[j], t[j]);
            }
        };
        constexpr int SETS = DP / 64;                         // of 16 heads
        if (nh * QUADS <= NT) join(std::integral_constant<int, 1>{}, 0);
        else if (nh * QUADS <= 2 * NT) join(std::integral_constant<int, SETS < 2 ? 1 : 2>{}, 0);
        else join(std::integral_constant<int, SETS>{}, 0);
        if (done) return;
        // the groups' sums are in the places of their first runs
        first = 0;
        runs = (splits + kFan - 1) / kFan;
        apart = kFan;
        word = words;
    }
}

// Steps of a workgroup, of `all` that the longest sequence has, so that the estimate of the whole is smallest, where a workgroup for
// every step would be 512 of them at most.  All measured, on tokens that come from HBM:
//   - memory delivers 5.9 TB/s, less a share for the parts of runs that are joined and for workgroups that come and go;
//   - a compute unit takes a step of 64 KB in 1.6 us, in 1.7 where it has two workgroups or more;
//   - joining runs takes 3.3 us and 1.2 for every further trip to memory, in groups 5.8 (8 x 300 tokens, 4 heads, 3 steps: 7.0 us with one
//     run, 7.4 with three; 1 x 600, 5 steps: 8.4, 6.7 with five).
// (8 x 1100 tokens, 4 heads of 128, bf16, 9 steps: 10.2 us with 1, 8.4 with 2, 10.4 with 4, 13.3 with 9.)
int attend_steps(int64_t rows, int tiles, int all, int quads, double step_bytes)
{
    const int64_t at_once = 8 * (quads < kWaves * 64 ? kWaves * 64 / quads : 1);
    const double step_us = std::max(0.5, step_bytes / 65536.0), memory = (double)rows * all * step_bytes / 5.9e6;
    int best = 1;
    double least = 1e300;
    for (int n = 1; n <= all; n += n < 4 ? 1 : n / 4) {
        const int64_t runs = (all + n - 1) / n, each = (rows * tiles * runs + 255) / 256, even = (all + runs - 1) / runs;
        const double steps = (double)(even * each) * step_us * (each > 1 ? 1.7 : 1.6);
        double us = memory;
        if (runs > 1) us *= 1.0 + 0.25 / std::sqrt((double)even);
        us = std::max(us, steps);
        if (runs > kDirect) us += 5.8 + 1.2 * (double)((kFan - 1) / at_once + (runs - 1) / kFan / at_once);
        else if (runs > 1) us += 3.3 + 1.2 * (double)((runs - 1) / at_once);
        if (us < least) { least = us; best = (int)even; }
    }
    return best;
}

// Steps of a run where there are more sequences than the kernel plans for: several workgroups to every unit in any case, and one of that
// many steps is not waited for long (2000 sequences of 100 tokens with a bound of 4096: 254 us with runs of 8 steps, 178 with 32).
constexpr int kManySteps = 32;

// How a call is laid out: tiles of query heads, tokens of a run
struct AttendPlan {
    int dp, tiles, cols, chunk, splits, parts_row, lds_words, words_each;
    bool planned;
    int64_t rows, units;
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
    const int step = kWaves * (dt == LUVC_F32 ? 16 : 32), all = (max_tokens + step - 1) / step;
    const int n_parts = n_heads * p.tiles;
    const int64_t parts = p.rows * p.tiles;
    p.planned = all > 1 && n_seqs <= kPlanSeqs && parts * all > 2 * kUnits;
    if (p.planned) {
        p.chunk = 0;
        p.splits = std::min(all, plan_runs(n_parts));
        p.units = std::min<int64_t>((int64_t)n_seqs * all, plan_runs(n_parts) + n_seqs) * n_heads;
    } else {
        int64_t steps;
        if (n_seqs <= kPlanSeqs) steps = attend_steps(p.rows, p.tiles, all, p.cols * ((D + 3) / 4), 2.0 * step * D * es);
        else steps = std::max<int64_t>({kManySteps, (all + kMaxSplits - 1) / kMaxSplits, (parts * all >> 22) + 1});
        p.chunk = (int)std::min<int64_t>(steps, all) * step;
        p.splits = (max_tokens + p.chunk - 1) / p.chunk;
        p.units = p.rows * p.splits;
    }
    p.blocks = (unsigned)((p.units + 7) / 8 * 8 * p.tiles);
    p.parts_row = (D + 3) / 4 * 4 + 4;
    // Workspace for any of the layouts above that n sequences of so many tokens or fewer may get: more of either never need less
    auto words_of = [&](int n) {
        const int runs = n <= kPlanSeqs ? std::min(all, plan_runs(n_parts)) : std::min((all + kManySteps - 1) / kManySteps, kMaxSplits);
        return runs > kDirect ? 1 + (runs + kFan - 1) / kFan : 1;
    };
    auto bytes_of = [&](int n) {
        const int64_t each = (int64_t)n * n_parts, runs = std::min((all + kManySteps - 1) / kManySteps, kMaxSplits);
        const int64_t slots = n > kPlanSeqs ? (runs > 1 ? std::min(each * runs, ((int64_t)1 << 22) + each) : 0) :
                              all > 1 ? std::min<int64_t>((int64_t)n * all, plan_runs(n_parts) + n) * n_parts : 0;
        return align_up((size_t)each * words_of(n) * sizeof(tile_tag_t)) + align_up((size_t)slots * p.cols * p.parts_row * sizeof(float));
    };
    p.words_each = words_of(n_seqs);
    p.words = align_up((size_t)parts * p.words_each * sizeof(tile_tag_t));
    p.bytes = bytes_of(n_seqs);
    if (n_seqs > kPlanSeqs) p.bytes = std::max(p.bytes, bytes_of(kPlanSeqs));
    // keys and queries; parts of the wavefronts; partial sums over runs.  Then maxima, sums, a word
    const size_t front = (size_t)(step + 16) * p.dp * es + 16 * 16, ends = (size_t)kWaves * p.cols * (p.dp + 4) * sizeof(float);
    const size_t join = p.splits > 1 ? (size_t)kWaves * 64 * 8 * sizeof(float) : 0;
    p.lds_words = (int)align_up(std::max({front, ends, join}), 16);
    p.lds = p.lds_words + (2 * (size_t)kWaves * 16 + 4) * sizeof(float);
    return p;
}

template <typename T, int DP, bool SMALL>
void attend_launch(const AttendPlan& p, const luvc_kv_cache& c, int layer, const KvWork& wk, const KvAttend& a, hipStream_t st)
{
    const T *k = (const T*)c.k + layer * c.layer_stride, *v = (const T*)c.v + layer * c.layer_stride;
    const dim3 grid(p.blocks), block(kWaves * 64);
    if (c.sizes) LUVC_LAUNCH("kv_attend", (kv_attend<T, DP, SMALL, true>), grid, block, p.lds, st, k, v, wk, a);
    else LUVC_LAUNCH("kv_attend", (kv_attend<T, DP, SMALL, false>), grid, block, p.lds, st, k, v, wk, a);
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
    const tile_tag_t tag = spu_next_tag();
    const double log2e = 1.4426950408889634074, full = a.scale == 0.0 ? 1.0 : std::fabs(a.scale) * log2e;
    const float scale = (float)full, rest = (float)(full - scale);
    const KvWork wk{c.sizes, c.n_pages, c.n_heads, kv_log2_page(c), c.D, a.n_q_heads / c.n_heads, p.chunk, p.tiles, p.cols, p.parts_row, p.words_each, p.lds_words, p.planned,
                    (unsigned)p.rows, (unsigned)p.splits, (unsigned)p.units,
                    (float*)((char*)ws + p.words), (tile_tag_t*)ws, tag,
                    scale, rest, a.scale < 0.f ? -1 : a.scale > 0.f};
    if (c.dtype == LUVC_F32) attend_shape<float>(p, c, layer, wk, a, st);
    else attend_shape<bf16_t>(p, c, layer, wk, a, st);
    return check_launch("attention over the cache");
}

}  // namespace luvc
