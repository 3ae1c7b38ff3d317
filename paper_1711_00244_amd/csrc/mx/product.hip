// Products with microscaled 4-bit matrices on the scaled matrix instructions: one matrix for all rows of X, or one per expert
// for the rows that were routed to it.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "mx_common.hpp"

namespace cl {
namespace mx {

// What a product kernel reads and writes.  Matrices are codes [row][block][16 bytes] and scales [row][block], `blocks` of them
// to a row, a multiple of four.
struct ProductArgs {
    const uint8_t *w_codes, *w_scales;
    const uint8_t *x_codes, *x_scales;
    const float *bias;
    void *Y;
    const int32_t *order;                                    // pairs in the order of the experts; null: row n of X makes row n of Y
    const int2 *tiles;
    const int32_t *tile_count;
    const float *weights;                                    // of rows of Y, where outputs are WEIGHTED
    int blocks, M, rows, experts, act;
    int out_width;                                           // elements of a row of Y
    Div x_div;                                               // pair / x_div is its row of X
    float *part;                                             // not null: sums of a share of k, [split][row of Y][pitch], to be finished
    int splits, pitch;
    int split_steps, split_more;                             // steps of 128 k of a share of k, and how many shares have one more
    Div row_tiles, band_tiles;                               // tiles of a column of tiles, and of a band of columns
    int past_caches;                                         // what the product stores would not stay in the caches until it is read again
    int tile0;                                               // tile of the launch's blockIdx.y of 0
    int skip_unrouted;                                       // the rows of Y of pairs without an expert are not read
};

// The columns of a tile: which rows of X and Y they are, and whose weights.
struct Columns {
    int first, count, expert;                                // of the order, or of X
};

template <int WIDTH> __device__ __forceinline__ bool columns_of(const ProductArgs &a, int tile, Columns &c)
{
    if (!a.order) {
        c = Columns{tile * WIDTH, min(WIDTH, a.rows - tile * WIDTH), 0};
        return true;
    }
    if (tile >= *a.tile_count) return false;
    const int2 t = a.tiles[tile];
    c = Columns{t.y, t.x & 0xffff, t.x >> 16};
    return !(c.expert == a.experts && a.skip_unrouted);
}

// The bias of four consecutive rows of the matrix from m on (zero where there is no expert, whose sums are zero as well).
__device__ __forceinline__ f32x4 bias_of(const ProductArgs &a, int expert, int m)
{
    f32x4 b = {0, 0, 0, 0};
    if (!a.bias || (a.order && expert >= a.experts)) return b;
    const float *at = a.bias + (int64_t)expert * a.M;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = at[min(m + i, a.M - 1)];          // (nothing waits for them here, as it would at a branch of lanes)
    return b;
}

// The outputs of four consecutive rows of the matrix, from m on, in one row of Y; WEIGHTED: times its weight, rounded to 32 bits as in the kernels that
// sum over k pairs.
template <class T, bool WEIGHTED> __device__ __forceinline__ void store_outputs(const ProductArgs &a, int64_t row, int m, f32x4 v, f32x4 bias, float weight)
{
    if (m >= a.M) return;
    if (a.bias) v += bias;
    T *y = (T *)a.Y + row * a.out_width;
    if (a.act == CL_ACT_GATED) {
        // rows 2 i and 2 i + 1 of the matrix: gate and value of output i
        const float g[2] = {v[0] / (1.0f + expf(-v[0])) * v[1], v[2] / (1.0f + expf(-v[2])) * v[3]};
        const T out[2] = {(T)(WEIGHTED ? product32(weight, g[0]) : g[0]), (T)(WEIGHTED ? product32(weight, g[1]) : g[1])};
        y += m / 2;
        if (m / 2 + 2 <= a.out_width) store_values<2>(y, out);
        else y[0] = out[0];
        return;
    }
    T out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = a.act == CL_ACT_RELU && v[i] < 0.0f ? 0.0f : v[i];       // (NaN stays)
        out[i] = (T)(WEIGHTED ? product32(weight, r) : r);
    }
    y += m;
    if (m + 4 <= a.out_width) {
        if (std::is_same_v<T, float> && a.past_caches) __builtin_nontemporal_store(f32x4{(float)out[0], (float)out[1], (float)out[2], (float)out[3]}, (f32x4 *)y);
        else store_values<4>(y, out);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (m + i < a.out_width) y[i] = out[i];
    }
}

// Four sums of a share of k.  (A row of partial sums is padded to whole fours.)
__device__ __forceinline__ void store_part(const ProductArgs &a, int split, int64_t row, int m, f32x4 v)
{
    if (m >= a.M) return;
    f32x4 *at = (f32x4 *)(a.part + ((int64_t)split * a.rows + row) * a.pitch + m);
    if (a.past_caches) __builtin_nontemporal_store(v, at);
    else *at = v;
}

// A workgroup of up to sixteen wavefronts makes 16 outputs (blockIdx.x) of 16 NT columns (blockIdx.y).  The wavefronts share out the
// row's runs of 16 blocks; of a run, a lane's group has four consecutive blocks - 64 bytes and one word of scales - which
// are its 32 k of four matrix instructions (the order of k does not matter as long as both operands have the same).
// Their sums meet in LDS and are added in the order of the wavefronts.  No operand is shared, so that nothing waits for a barrier until the
// end: 37 x 1000 x 4096 5.4 us, which are the launch and two trips to memory (2.2 MB); with more columns reading W again for every
// sixteen costs more than a tile's start (256 x 4096 x 9216 90 us, 64 x 64 18.7).
constexpr int kRowsWaves = 16;

template <int NT, class T, bool WEIGHTED> __global__ __launch_bounds__(kRowsWaves * 64) void mx_rows_kernel(ProductArgs a)
{
    __shared__ f32x4 part[kRowsWaves][NT][64];
    Columns c;
    if (!columns_of<16 * NT>(a, a.tile0 + (int)blockIdx.y, c)) return;
    const int waves = (int)blockDim.x / 64, wave = threadIdx.x / 64, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int m0 = (int)blockIdx.x * 16;
    f32x4 acc[NT] = {};
    if (!a.order || c.expert < a.experts) {                  // (the pairs without an expert: zeros)
        const int64_t w_row = (int64_t)c.expert * a.M + min(m0 + r, a.M - 1);
        const uint8_t *wc = a.w_codes + w_row * a.blocks * 16, *ws = a.w_scales + w_row * a.blocks;
        const uint8_t *xc[NT], *xs[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int n = c.first + min(t * 16 + r, c.count - 1);
            const int64_t x_row = a.order ? (int64_t)a.x_div.quotient((uint32_t)a.order[n]) : n;
            xc[t] = a.x_codes + x_row * a.blocks * 16;
            xs[t] = a.x_scales + x_row * a.blocks;
        }
        for (int b = wave * 16 + g * 4; b - g * 4 < a.blocks; b += waves * 16) {
            const bool in = b < a.blocks;                    // (four blocks are in or out together)
            const int bb = in ? b : 0;
            i32x4 w[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) w[s] = in ? ((const i32x4 *)(wc + (int64_t)bb * 16))[s] : i32x4{};
            const int sw = in ? *(const int *)(ws + bb) : 0;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                i32x4 x[4];
#pragma unroll
                for (int s = 0; s < 4; ++s) x[s] = in ? ((const i32x4 *)(xc[t] + (int64_t)bb * 16))[s] : i32x4{};
                const int sx = in ? *(const int *)(xs[t] + bb) : 0;
                acc[t] = mfma_fp4<0>(w[0], x[0], acc[t], sw, sx);
                acc[t] = mfma_fp4<1>(w[1], x[1], acc[t], sw, sx);
                acc[t] = mfma_fp4<2>(w[2], x[2], acc[t], sw, sx);
                acc[t] = mfma_fp4<3>(w[3], x[3], acc[t], sw, sx);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    for (int e = threadIdx.x; e < NT * 64; e += (int)blockDim.x) {
        const int t = e / 64, l = e & 63, n = t * 16 + (l & 15);
        if (n >= c.count) continue;
        f32x4 v = part[0][t][l];
        for (int w = 1; w < waves; ++w) v += part[w][t][l];
        const int64_t y_row = a.order ? a.order[c.first + n] : c.first + n;
        if (a.part) store_part(a, 0, y_row, m0 + 4 * (l >> 4), v);
        else store_outputs<T, WEIGHTED>(a, y_row, m0 + 4 * (l >> 4), v, bias_of(a, c.expert, m0 + 4 * (l >> 4)), WEIGHTED && c.expert < a.experts ? a.weights[y_row] : 0.0f);
    }
}

#include "few_kernel.hpp"
#include "tile_kernel.hpp"

// The sum over the splits of a product's parts, in order, and from it four outputs of one row (two, of a gated product).  Parts come from
// the caches: 146 x 2084, two parts, 3.9 us, of which the launch is two.
template <class T> __global__ __launch_bounds__(256) void mx_finish_kernel(ProductArgs a, Div quads, int row0, int rows)
{
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = quads.quotient(at);
    if (row >= (uint32_t)rows) return;
    const int m = (int)(at - row * quads.d) * 4;
    const int64_t t = (int64_t)row0 + row, stride = (int64_t)a.rows * a.pitch;
    const float *p = a.part + t * a.pitch + m;
    f32x4 part[8];                                           // (at most eight)
#pragma unroll
    for (int s = 0; s < 8; ++s) part[s] = *(const f32x4 *)(p + min(s, a.splits - 1) * stride);
#pragma unroll
    for (int s = 1; s < 8; ++s)
        if (s < a.splits) part[0] += part[s];
    store_outputs<T, false>(a, t, m, part[0], bias_of(a, 0, m), 1.0f);
}

// Y[t] = sum over j, in order, of weights[t][j] times what the product made of pair t k + j, of the pairs that have an expert.
// A thread makes four consecutive outputs of one token and has asked for TOGETHER pairs' before it uses the first.  Memory bounds it:
// 8192 tokens, four pairs each, 2048 outputs, 302 MB in 50 us, 6.0 TB/s; 3463, two, 2900 15.7 (with bias and activation here, and a
// 64-bit division, 44).
struct JoinArgs {
    const float *pairs, *weights;                            // rows of pitch elements
    const int32_t *experts_of;
    void *Y;
    int token0, tokens, k, experts, width, pitch;
    Div quads;                                               // fours of a row
};

template <class T, int TOGETHER> __global__ __launch_bounds__(256) void mx_join_kernel(JoinArgs a)
{
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, token = a.quads.quotient(at);
    if (token >= (uint32_t)a.tokens) return;
    const int m = (int)(at - token * a.quads.d) * 4;
    const int64_t t = (int64_t)a.token0 + token;
    f32x4 sum = {0, 0, 0, 0};
    for (int j0 = 0; j0 < a.k; j0 += TOGETHER) {
        int e[TOGETHER];
        float weight[TOGETHER];
        f32x4 v[TOGETHER];
#pragma unroll
        for (int i = 0; i < TOGETHER; ++i) {
            const int64_t pair = t * a.k + min(j0 + i, a.k - 1);
            e[i] = a.experts_of[pair];
            weight[i] = a.weights[pair];
            v[i] = *(const f32x4 *)(a.pairs + pair * a.pitch + m);
        }
#pragma unroll
        for (int i = 0; i < TOGETHER; ++i) {
            if (j0 + i >= a.k || e[i] < 0 || e[i] >= a.experts) continue;
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] = fmaf(weight[i], v[i][c], sum[c]);
        }
    }
    T *y = (T *)a.Y + t * a.width + m;
    if (m + 4 <= a.width) {
        const T v[4] = {(T)sum[0], (T)sum[1], (T)sum[2], (T)sum[3]};
        store_values<4>(y, v);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (m + i < a.width) y[i] = (T)sum[i];
    }
}

enum Form { kRows, kTile64, kTile128, kTile256x128, kTile256 };
constexpr int kFormRows[] = {16, 64, 128, 256, 256}, kFormThreads[] = {0, 256, 512, 512, 512};      // of a workgroup (kRows: as many as run_waves says)

template <Form F, int BN, int WM, int WN, int D, class T, bool WEIGHTED> static int32_t launch_tiles(ProductArgs a, int64_t tiles, hipStream_t st)
{
    constexpr int BM = kFormRows[F];
    using C = Tile<BM, BN, WM, WN, D>;
    static_assert(C::kThreads == kFormThreads[F], "");
    auto kernel = mx_tile_kernel<BM, BN, WM, WN, D, T, WEIGHTED>;
    static LdsLimit seen;
    if (int32_t rc = allow_lds((const void *)kernel, C::kLds, seen)) return rc;
    const int64_t row_tiles = (a.M + BM - 1) / BM;
    a.row_tiles = make_div((uint32_t)row_tiles);
    a.band_tiles = make_div((uint32_t)row_tiles * (a.order ? 1u : 4u));
    a.split_steps = a.blocks / 4 / a.splits;
    a.split_more = a.blocks / 4 % a.splits;
    hipLaunchKernelGGL(kernel, dim3((unsigned)round_up(row_tiles * tiles, 8), (unsigned)a.splits), dim3(C::kThreads), C::kLds, st, a, (int)row_tiles);
    MX_HIP_TRY(hipGetLastError());
    return CL_OK;
}

// ------------------------------------------------------------------------- //
// which kernel
// ------------------------------------------------------------------------- //
struct Choice {
    Form form;
    int width;                                               // columns of a tile: an index of kTileWidth
    int splits;
    float us;
};

// What a form takes in microseconds, fitted to measurements of 450 shapes of M 100 .. 4096, K 100 .. 25088, 20 .. 16000 columns, one
// matrix and 4 to 128: over 550 others the choice took 1.4 % longer, in the mean of logarithms, than the best of the forms.  (That was with
// 128 x 128 on four wavefronts; on eight it is 7-14 % faster at small K, and its row is as it was.  A row fits its shapes on the whole: a step of 64 x 64
// alone on a compute unit is 0.16 here and 0.18 at 256 x 4096 x 9216.)
// Tiles: a start (launch, what its columns are, first loads, last stores), and per step of 128 k what a workgroup takes alone on
// its compute unit, or its share of a full one where the launch has more workgroups than the chip has compute units; that
// is another with experts, whose matrices change within a launch.
struct Price { int bm, bn, width; float start, alone, shared, shared_experts; };
constexpr Price kPrices[] = {{64, 64, 1, 5.1f, 0.16f, 0.31f, 0.24f}, {128, 128, 2, 7.5f, 0.35f, 0.63f, 0.52f}, {256, 128, 2, 9.0f, 0.60f, 0.51f, 0.80f},
                             {256, 256, 3, 12.0f, 0.90f, 1.20f, 1.10f}};
constexpr int kCus = 256;
constexpr int64_t kCaches = 128 << 20;                       // half of what the caches hold (past them 268 MB of pairs: 312 us in all, through them 325)

// rows: columns of the product in all; experts: how many matrices share them (0: one matrix); most_splits: 1 where there is no room for parts.
static Choice choose(int M, int blocks, int64_t rows, int experts, int most_splits = 8)
{
    const int steps = blocks / 4, runs = (blocks + 15) / 16;
    // the matrices that have columns, and those that have more than i tiles of them, their numbers spread about the mean
    const float mean = experts ? (float)rows / experts : 0.0f, spread = std::sqrt(mean) + mean / 8;
    auto tiles_of = [&](int bn) {
        if (!experts) return (float)((rows + bn - 1) / bn);
        if (spread > bn) return (mean / bn + 0.5f) * experts;            // (what the sum comes to, with many terms)
        const float whole = std::max(0.0f, std::floor((mean - 4 * spread) / bn));
        float n = (1.0f - std::exp(-mean)) + whole;
        for (float i = whole + 1; i * bn < mean + 4 * spread; ++i) n += 1.0f / (1.0f + std::exp(1.7f * (i * bn - mean) / spread));
        return n * experts;
    };
    // columns sixteen at a time: every workgroup reads all it multiplies itself
    const float wgs = (float)(((int64_t)M + 15) / 16) * tiles_of(16);
    Choice best{kRows, 0, 1, 2.5f + std::max(1.08e-3f * wgs * runs, 2.6f * ((runs + kRowsWaves - 1) / kRowsWaves))};
    for (int f = kTile64; f <= kTile256; ++f) {
        const Price &p = kPrices[f - kTile64];
        const float n = tiles_of(p.bn) * (((int64_t)M + p.bm - 1) / p.bm);
        const bool alone = f >= kTile256x128;                // (one workgroup to a compute unit: whole rounds; else two, which hide starts)
        for (int splits = 1; splits <= most_splits && (splits == 1 || steps / splits >= 4); splits *= 2) {
            if (splits > 1 && (experts || n * splits > 2 * kCus)) break;
            const float full = n * splits / kCus, rounds = std::max(1.0f, std::ceil(full));
            const float each = full <= 1.0f ? p.alone : std::max(p.alone, (experts ? p.shared_experts : p.shared) * (alone ? rounds : full));
            float us = p.start * (alone ? rounds : 1.0f + 0.4f * std::max(0.0f, full / 2 - 1)) + each * (steps + splits - 1) / splits;
            if (splits > 1) us += 1.7f + (float)(2 * splits - 1) * rows * M * 0.66e-6f;        // (the parts, there and back, and a launch)
            if (us < best.us) best = Choice{(Form)f, p.width, splits, us};
        }
    }
    return best;
}

// Wavefronts that share out the runs of 16 blocks of a row: as many rounds as sixteen would need, and no more than that takes.
// (The same in both kernels that do: the same sums, bit for bit.)
static int run_waves(int blocks)
{
    const int runs = (blocks + 15) / 16, rounds = (runs + kRowsWaves - 1) / kRowsWaves;
    return (runs + rounds - 1) / rounds;
}

// Whether the launch has less than 2^32 threads along each axis, for `tiles` columns of tiles.
static int32_t check_grid(const Choice &c, int32_t M, int blocks, int64_t tiles)
{
    const int64_t rows = kFormRows[c.form], row_tiles = (M + rows - 1) / rows;
    const int64_t wgs = c.form == kRows ? row_tiles : (int64_t)round_up(row_tiles * tiles, 8), threads = c.form == kRows ? run_waves(blocks) * 64 : kFormThreads[c.form];
    if (wgs > (int64_t)UINT32_MAX / threads) return fail(CL_EUNSUPPORTED, "a launch of %lld workgroups does not fit a grid", (long long)wgs);
    return CL_OK;
}
static int64_t column_tiles(const Choice &c, int64_t rows) { return (rows + kTileWidth[c.width] - 1) / kTileWidth[c.width]; }

// The tiles of a product: rows of X in order, or what the lists have.
template <class T, bool WEIGHTED> static int32_t launch_product(ProductArgs a, const Choice &c, const ExpertLists *L, hipStream_t st)
{
    int64_t tiles = column_tiles(c, a.rows);
    if (L) {
        a.tiles = L->tiles[c.width];
        a.tile_count = L->tile_count + c.width;
        tiles = L->max_tiles[c.width];
    }
    a.splits = c.splits;
    switch (c.form) {
    case kTile64: return launch_tiles<kTile64, 64, 2, 2, 8, T, WEIGHTED>(a, tiles, st);
    case kTile128: return launch_tiles<kTile128, 128, 2, 4, 4, T, WEIGHTED>(a, tiles, st);
    case kTile256x128: return launch_tiles<kTile256x128, 128, 4, 2, 4, T, WEIGHTED>(a, tiles, st);
    case kTile256: return launch_tiles<kTile256, 256, 2, 4, 4, T, WEIGHTED>(a, tiles, st);
    default: break;
    }
    // (a grid is at most 65535 high: taller ones go in pieces)
    for (int64_t t0 = 0; t0 < tiles; t0 += 65535) {
        a.tile0 = (int)t0;
        hipLaunchKernelGGL((mx_rows_kernel<1, T, WEIGHTED>), dim3((unsigned)((a.M + 15) / 16), (unsigned)std::min<int64_t>(tiles - t0, 65535)), dim3(run_waves(a.blocks) * 64), 0, st, a);
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
}

// Rows of each of a token's matrices that a workgroup has (even: a gated product's rows come in pairs).
static int few_rows_each(int k) { return 32 / k / 2 * 2; }

// Wavefronts of a workgroup of few_kernel: those that multiply, and more where there is much to quantise.
static int few_waves(int blocks, int columns) { return std::max(run_waves(blocks), std::min(kFewWaves, (columns * blocks * 4 + 255) / 256)); }

// Whether few_kernel takes a call: by what it takes in microseconds (fitted to M 119 .. 4096, K 106 .. 25088, 1 .. 256 columns or 1 .. 1245
// tokens) against the launches that it replaces, of which each costs the host, besides, some 4 us.  kLaunch of those count: between calls one by one,
// which pay them, and calls recorded in a graph, which do not.  (37 rows of bf16 by 1000 x 4096: 9.4 and 9.3 by price, so two launches, 8.4 of
// kernels and 13.1 a call.)
constexpr int64_t kFewMostWgs = UINT32_MAX / (kFewWaves * 64);         // (a launch has less than 2^32 threads along an axis)
constexpr float kQuantise = 2.2f, kLists = 5.5f, kJoin = 3.0f, kLaunch = 2.0f;
static bool few_fc(int M, int blocks, int batch, int32_t x_type)
{
    const int columns = std::min(batch, kFewColumns);
    const int64_t groups = ((int64_t)batch + kFewColumns - 1) / kFewColumns, row_wgs = ((int64_t)M + 15) / 16, wgs = groups * row_wgs;
    if (x_type == CL_MX4 || groups > 65535 || row_wgs > kFewMostWgs || few_lds(blocks, columns) > kFewLds) return false;
    // a workgroup's quantisation, the share of a chip that is full of them, or reading the matrix
    const float own = (float)columns * blocks, us = std::max(std::max(4.3f + 2.5e-3f * own, 3.0f + 3.9e-3f * own * wgs / kCus), 2.7f + (float)wgs * 16 * blocks * 17 / 5e6f);
    return us <= kQuantise + choose(M, blocks, batch, 0).us + kLaunch;
}
static bool few_experts(int M, int blocks, int32_t x_type, int experts, const cl_mx_experts_call &call)
{
    if (x_type == CL_MX4 || call.d_lists || call.k > 16 || call.tokens > 65535 || few_lds(blocks, call.x_per_pair ? call.k : 1) > kFewLds) return false;
    const int64_t rows_each = few_rows_each(call.k), row_wgs = (M + rows_each - 1) / rows_each;
    if (row_wgs > kFewMostWgs) return false;
    // workgroups as fast as they are launched, or reading a matrix for every token that is sent to it
    const float wgs = (float)call.tokens * row_wgs, us = 4.0f + std::max(1.45e-3f * wgs, (float)call.tokens * call.k * M * blocks * 17 / 4e6f);
    return us <= kLists + choose(M, blocks, (int64_t)call.tokens * call.k, experts).us + kLaunch + (call.d_weights && call.k > 1 ? kJoin + kLaunch : 0.0f);
}

static int32_t launch_few(FewArgs a, int32_t x_type, int32_t y_type, bool experts, dim3 grid, hipStream_t st)
{
    a.waves = run_waves(a.p.blocks);
    const int threads = 64 * few_waves(a.p.blocks, a.columns);
    const size_t lds = few_lds(a.p.blocks, a.columns) + (size_t)a.waves * (experts ? 2 : 1) * 64 * sizeof(f32x4);
    return with_type(x_type, [&](auto x) -> int32_t {
        return with_type(y_type, [&](auto y) -> int32_t {
            using X = decltype(x);
            using Y = decltype(y);
            auto kernel = experts ? mx_few_kernel<X, Y, true> : mx_few_kernel<X, Y, false>;
            static LdsLimit seen[2];
            if (int32_t rc = allow_lds((const void *)kernel, kFewLds + kFewWaves * 2 * 64 * sizeof(f32x4), seen[experts])) return rc;
            hipLaunchKernelGGL(kernel, grid, dim3((unsigned)threads), lds, st, a);
            MX_HIP_TRY(hipGetLastError());
            return CL_OK;
        });
    });
}

// launch(row0, rows, workgroups) over rows of `quads` threads each, in pieces whose threads' numbers have 32 bits.
template <class F> static int32_t launch_rows(int32_t rows, uint32_t quads, F launch)
{
    const int32_t most = (int32_t)std::min<int64_t>(rows, (1ll << 31) / quads);
    for (int32_t row0 = 0, n; row0 < rows; row0 += n) {
        n = std::min(most, rows - row0);
        launch(row0, n, dim3((uint32_t)(((int64_t)n * quads + 255) / 256)));
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
}

// The product of one matrix; a.part is where the sums of a split product go.
static int32_t run_product(const ProductArgs &a, const Choice &c, int32_t y_type, hipStream_t st)
{
    if (!a.part) return with_type(y_type, [&](auto t) { return launch_product<decltype(t), false>(a, c, nullptr, st); });
    ProductArgs p = a;
    p.splits = c.splits;
    p.past_caches = (int64_t)c.splits * a.rows * a.pitch * 4 > kCaches;
    if (int32_t rc = launch_product<float, false>(p, c, nullptr, st)) return rc;
    p.past_caches = 0;
    const Div quads = make_div((uint32_t)a.pitch / 4);
    return with_type(y_type, [&](auto t) -> int32_t {
        return launch_rows(a.rows, quads.d, [&](int row0, int rows, dim3 grid) {
            hipLaunchKernelGGL(mx_finish_kernel<decltype(t)>, grid, dim3(256), 0, st, p, quads, row0, rows);
        });
    });
}

// The products of the pairs, to `pairs` (fp32) and from there to the weighted sums, or straight to Y.
static int32_t run_experts(const ProductArgs &a, const Choice &c, const ExpertLists &L, const cl_mx_experts_call &call, float *pairs, int32_t y_type, hipStream_t st)
{
    if (!call.d_weights) return with_type(y_type, [&](auto t) { return launch_product<decltype(t), false>(a, c, &L, st); });
    ProductArgs p = a;
    if (call.k == 1) {                                       // nothing to join
        p.weights = call.d_weights;
        return with_type(y_type, [&](auto t) { return launch_product<decltype(t), true>(p, c, &L, st); });
    }
    p.Y = pairs;
    p.out_width = (int)round_up(a.out_width, 4);
    p.skip_unrouted = 1;
    p.past_caches = (int64_t)a.rows * p.out_width * 4 > kCaches;
    if (int32_t rc = launch_product<float, false>(p, c, &L, st)) return rc;
    JoinArgs f{pairs, call.d_weights, call.d_experts, a.Y, 0, 0, call.k, a.experts, a.out_width, p.out_width, make_div((uint32_t)p.out_width / 4)};
    return with_type(y_type, [&](auto t) -> int32_t {
        return launch_rows(call.tokens, f.quads.d, [&](int row0, int rows, dim3 grid) {
            f.token0 = row0;
            f.tokens = rows;
            if (f.k <= 2) hipLaunchKernelGGL((mx_join_kernel<decltype(t), 2>), grid, dim3(256), 0, st, f);
            else hipLaunchKernelGGL((mx_join_kernel<decltype(t), 4>), grid, dim3(256), 0, st, f);
        });
    });
}

static int32_t check_matrix(const cl_mx_matrix *W)
{
    if (!W) return fail(CL_EINVAL, "null pointer");
    if (W->rows < 1 || W->K < 1) return fail(CL_EINVAL, "bad matrix: %d x %d", (int)W->rows, (int)W->K);
    if (W->K > CL_MX_MAX_K) return fail(CL_EUNSUPPORTED, "rows of more than %d elements", (int)CL_MX_MAX_K);
    return CL_OK;
}

static int32_t check_pointers(const cl_mx_matrix *W, const cl_mx_input *X, const void *Y, int64_t rows)
{
    if (!W->d_codes || !W->d_scales || !X->d_X || !Y) return fail(CL_EINVAL, "null pointer");
    if (!aligned(W->d_codes, 16) || !aligned(W->d_scales, 4)) return fail(CL_EINVAL, "codes must be 16-byte and scales 4-byte aligned");
    if (X->type == CL_MX4) {
        if (!X->d_scales) return fail(CL_EINVAL, "null pointer");
        if (!aligned(X->d_X, 16) || !aligned(X->d_scales, 4)) return fail(CL_EINVAL, "codes must be 16-byte and scales 4-byte aligned");
    } else {
        if (!aligned(X->d_X, type_bytes(X->type))) return fail(CL_EINVAL, "elements are not aligned");
        if (rows > 1 && X->stride < W->K) return fail(CL_EINVAL, "rows of %d elements overlap at a stride of %lld", (int)W->K, (long long)X->stride);
    }
    return CL_OK;
}

static int32_t check_forward(const cl_mx_matrix *W, int32_t x_type, int32_t y_type, int32_t act)
{
    if (int32_t rc = check_matrix(W)) return rc;
    if (!known_type(x_type) && x_type != CL_MX4) return fail(CL_EINVAL, "unknown element type %d", (int)x_type);
    if (!known_type(y_type)) return fail(CL_EINVAL, "unknown element type %d", (int)y_type);
    if (act != CL_ACT_NONE && act != CL_ACT_RELU && act != CL_ACT_GATED) return fail(CL_EINVAL, "unknown activation %d", (int)act);
    if (act == CL_ACT_GATED && W->rows % 2) return fail(CL_EINVAL, "a gated product needs an even number of rows, got %d", (int)W->rows);
    return CL_OK;
}

// Scratch of a call, by what is in it.
struct Scratch {
    size_t x_codes = 0, x_scales = 0, pairs = 0, lists = 0, bytes = 0;
    size_t take(size_t n) { const size_t at = bytes; bytes += round_up(n, 256); return at; }
};

static void scratch_input(Scratch &s, int32_t x_type, int64_t rows, int32_t K)
{
    if (x_type == CL_MX4) return;
    s.x_codes = s.take((size_t)rows * row_blocks(K) * 16);
    s.x_scales = s.take((size_t)rows * row_blocks(K));
}

static int32_t check_scratch(const Scratch &s, const void *ws, size_t bytes)
{
    if (s.bytes && !ws) return fail(CL_EINVAL, "null workspace");
    if (bytes < s.bytes) return fail(CL_EINVAL, "workspace needs %zu bytes, got %zu", s.bytes, bytes);
    if (s.bytes && !aligned(ws, 256)) return fail(CL_EINVAL, "workspace must be 256-byte aligned");
    return CL_OK;
}

// The 4-bit rows of the input: its own, or made in the workspace.
static int32_t quantised_input(ProductArgs &a, const cl_mx_input *X, int64_t rows, int32_t K, const Scratch &s, void *ws, hipStream_t st)
{
    if (X->type == CL_MX4) {
        a.x_codes = (const uint8_t *)X->d_X;
        a.x_scales = (const uint8_t *)X->d_scales;
        return CL_OK;
    }
    uint8_t *codes = (uint8_t *)ws + s.x_codes, *scales = (uint8_t *)ws + s.x_scales;
    a.x_codes = codes;
    a.x_scales = scales;
    return launch_quantize(X->d_X, X->type, X->stride, rows, K, codes, scales, st);
}

static size_t part_bytes(int32_t M, int64_t rows, int splits) { return (size_t)splits * rows * round_up(M, 4) * 4; }

static Scratch fc_scratch(const Choice &c, int32_t M, int32_t K, int32_t x_type, int32_t batch)
{
    Scratch s;
    scratch_input(s, x_type, batch, K);
    if (c.splits > 1) s.pairs = s.take(part_bytes(M, batch, c.splits));
    return s;
}

// What is asked for a batch is enough for all smaller ones: X's codes grow with it, where they have no room beside them for parts a product is not
// split, and where one launch would do it is asked what a smaller batch needs that takes more.
static size_t fc_need(const Choice &c, const cl_mx_matrix &W, int32_t x_type, int32_t batch)
{
    const int blocks = row_blocks(W.K);
    if (!few_fc(W.rows, blocks, batch, x_type)) return fc_scratch(c, W.rows, W.K, x_type, batch).bytes;
    // (from kFewColumns on, few_kernel takes as long for all batches of a group, and the other forms at least as long as for its first)
    for (int32_t b = batch - 1; b > 0; b = b <= kFewColumns ? b - 1 : std::max((b - 2) / kFewColumns * kFewColumns + 1, kFewColumns))
        if (!few_fc(W.rows, blocks, b, x_type)) return fc_scratch(Choice{kRows, 0, 1, 0.0f}, W.rows, W.K, x_type, batch).bytes;
    return 0;
}

static Scratch experts_scratch(int32_t M, int32_t K, int32_t x_type, int32_t experts, const cl_mx_experts_call &call)
{
    Scratch s;
    scratch_input(s, x_type, (int64_t)call.tokens * (call.x_per_pair ? call.k : 1), K);
    if (call.d_weights && call.k > 1) s.pairs = s.take(part_bytes(call.act == CL_ACT_GATED ? M / 2 : M, (int64_t)call.tokens * call.k, 1));
    if (!call.d_lists) s.lists = s.take(expert_lists_at(nullptr, call.tokens, call.k, experts).bytes);
    return s;
}

}  // namespace mx
}  // namespace cl

using namespace cl;
using namespace cl::mx;

extern "C" int32_t cl_mx_fc_workspace_bytes(const cl_mx_matrix *W, int32_t batch, int32_t x_type, size_t *out)
{
    if (!out) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, x_type, CL_F32, CL_ACT_NONE)) return rc;
    if (batch < 0) return fail(CL_EINVAL, "batch of %d", (int)batch);
    const Choice c = choose(W->rows, row_blocks(W->K), batch, 0);
    if (!few_fc(W->rows, row_blocks(W->K), batch, x_type))
        if (int32_t rc = check_grid(c, W->rows, row_blocks(W->K), column_tiles(c, batch))) return rc;
    *out = fc_need(c, *W, x_type, batch);
    clear_error();
    return CL_OK;
}

static_assert(CL_MX_FORM_ROWS == 1 + kRows && CL_MX_FORM_TILE_64 == 1 + kTile64 && CL_MX_FORM_TILE_256 == 1 + kTile256, "");

extern "C" int32_t cl_mx_fc_resolved_form(const cl_mx_matrix *W, int32_t batch, int32_t x_type, int32_t *form, int32_t *splits)
{
    if (!form || !splits) return fail(CL_EINVAL, "null pointer");
    size_t bytes;
    if (int32_t rc = cl_mx_fc_workspace_bytes(W, batch, x_type, &bytes)) return rc;
    const bool few = few_fc(W->rows, row_blocks(W->K), batch, x_type);
    const Choice c = choose(W->rows, row_blocks(W->K), batch, 0);
    *form = few ? CL_MX_FORM_FEW : 1 + c.form;
    *splits = few ? 1 : c.splits;
    return CL_OK;
}

extern "C" int32_t cl_mx_fc_forward(const cl_mx_matrix *W, const cl_mx_input *X, const float *d_bias, void *d_Y, int32_t y_type, int32_t batch, int32_t act,
                                    void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!X) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, X->type, y_type, act)) return rc;
    if (batch < 0) return fail(CL_EINVAL, "batch of %d", (int)batch);
    if (batch == 0) return CL_OK;
    if (int32_t rc = check_pointers(W, X, d_Y, batch)) return rc;
    hipStream_t st = (hipStream_t)stream;
    ProductArgs a{};
    a.w_codes = (const uint8_t *)W->d_codes;
    a.w_scales = (const uint8_t *)W->d_scales;
    a.bias = d_bias;
    a.blocks = row_blocks(W->K);
    a.M = W->rows;
    a.rows = batch;
    a.act = act;
    a.out_width = act == CL_ACT_GATED ? W->rows / 2 : W->rows;
    if (few_fc(a.M, a.blocks, batch, X->type)) {
        a.Y = d_Y;
        const FewArgs f{a, X->d_X, X->stride, W->K, std::min(batch, kFewColumns), nullptr, nullptr, 1, 0, 0, 0};
        if (int32_t rc = launch_few(f, X->type, y_type, false, dim3((unsigned)((a.M + 15) / 16), (unsigned)((batch + kFewColumns - 1) / kFewColumns)), st)) return rc;
        clear_error();
        return CL_OK;
    }
    Choice c = choose(W->rows, a.blocks, batch, 0);
    Scratch s = fc_scratch(c, W->rows, W->K, X->type, batch);
    if (c.splits > 1 && workspace_bytes < s.bytes) {
        c = choose(W->rows, a.blocks, batch, 0, 1);
        s = fc_scratch(c, W->rows, W->K, X->type, batch);
    }
    if (int32_t rc = check_grid(c, a.M, a.blocks, column_tiles(c, batch))) return rc;
    if (int32_t rc = check_scratch(s, d_workspace, workspace_bytes)) return rc;
    if (int32_t rc = quantised_input(a, X, batch, W->K, s, d_workspace, st)) return rc;
    a.part = c.splits > 1 ? (float *)((uint8_t *)d_workspace + s.pairs) : nullptr;
    a.pitch = (int)round_up(W->rows, 4);
    a.Y = d_Y;
    if (int32_t rc = run_product(a, c, y_type, st)) return rc;
    clear_error();
    return CL_OK;
}

static int32_t check_experts(const cl_mx_matrix *W, int32_t experts, int32_t tokens, int32_t k)
{
    if (experts < 1 || tokens < 0 || k < 1) return fail(CL_EINVAL, "%d tokens, %d of %d experts", (int)tokens, (int)k, (int)experts);
    if (experts > CL_ROUTE_MAX_EXPERTS) return fail(CL_EUNSUPPORTED, "%d experts: at most %d", (int)experts, CL_ROUTE_MAX_EXPERTS);
    if ((int64_t)tokens * k > CL_EXPERTS_MAX_PAIRS) return fail(CL_EUNSUPPORTED, "more than 2^30 pairs of token and expert");
    return CL_OK;
}

extern "C" int32_t cl_mx_experts_workspace_bytes(const cl_mx_matrix *W, int32_t experts, const cl_mx_experts_call *call, int32_t x_type, size_t *out)
{
    if (!out || !call) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, x_type, CL_F32, call->act)) return rc;
    if (int32_t rc = check_experts(W, experts, call->tokens, call->k)) return rc;
    // (enough for fewer tokens too: where one launch would do, what the most tokens below need that take more)
    cl_mx_experts_call most = *call;
    while (most.tokens > 0 && few_experts(W->rows, row_blocks(W->K), x_type, experts, most)) --most.tokens;
    if (most.tokens == call->tokens) {
        const Choice c = choose(W->rows, row_blocks(W->K), (int64_t)call->tokens * call->k, experts);
        if (int32_t rc = check_grid(c, W->rows, row_blocks(W->K), expert_lists_at(nullptr, call->tokens, call->k, experts).max_tiles[c.width])) return rc;
    }
    *out = most.tokens > 0 ? experts_scratch(W->rows, W->K, x_type, experts, most).bytes : 0;
    clear_error();
    return CL_OK;
}

extern "C" int32_t cl_mx_experts_resolved_form(const cl_mx_matrix *W, int32_t experts, const cl_mx_experts_call *call, int32_t x_type, int32_t *form)
{
    if (!form) return fail(CL_EINVAL, "null pointer");
    size_t bytes;
    if (int32_t rc = cl_mx_experts_workspace_bytes(W, experts, call, x_type, &bytes)) return rc;
    const bool few = few_experts(W->rows, row_blocks(W->K), x_type, experts, *call);
    *form = few ? CL_MX_FORM_FEW : 1 + choose(W->rows, row_blocks(W->K), (int64_t)call->tokens * call->k, experts).form;
    return CL_OK;
}

extern "C" int32_t cl_mx_experts_forward(const cl_mx_matrix *W, int32_t experts, const cl_mx_input *X, const cl_mx_experts_call *call, void *d_Y, int32_t y_type,
                                         void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!X || !call) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, X->type, y_type, call->act)) return rc;
    if (int32_t rc = check_experts(W, experts, call->tokens, call->k)) return rc;
    const int32_t tokens = call->tokens, k = call->k;
    if (tokens == 0) return CL_OK;
    const int64_t x_rows = (int64_t)tokens * (call->x_per_pair ? k : 1);
    if (int32_t rc = check_pointers(W, X, d_Y, x_rows)) return rc;
    if (!call->d_experts) return fail(CL_EINVAL, "null pointer");
    if (call->d_lists && !aligned(call->d_lists, 256)) return fail(CL_EINVAL, "lists must be 256-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    ProductArgs a{};
    a.w_codes = (const uint8_t *)W->d_codes;
    a.w_scales = (const uint8_t *)W->d_scales;
    a.bias = call->d_bias;
    a.blocks = row_blocks(W->K);
    a.M = W->rows;
    a.rows = tokens * k;
    a.experts = experts;
    a.act = call->act;
    a.out_width = call->act == CL_ACT_GATED ? W->rows / 2 : W->rows;
    if (few_experts(a.M, a.blocks, X->type, experts, *call)) {
        a.Y = d_Y;
        const int rows_each = few_rows_each(k);
        const FewArgs f{a, X->d_X, X->stride, W->K, call->x_per_pair ? k : 1, call->d_experts, call->d_weights, k, rows_each, call->x_per_pair, 0};
        if (int32_t rc = launch_few(f, X->type, y_type, true, dim3((unsigned)((a.M + rows_each - 1) / rows_each), (unsigned)tokens), st)) return rc;
        clear_error();
        return CL_OK;
    }
    const Choice c = choose(a.M, a.blocks, (int64_t)tokens * k, experts);
    if (int32_t rc = check_grid(c, a.M, a.blocks, expert_lists_at(nullptr, tokens, k, experts).max_tiles[c.width])) return rc;
    const Scratch s = experts_scratch(W->rows, W->K, X->type, experts, *call);
    if (int32_t rc = check_scratch(s, d_workspace, workspace_bytes)) return rc;
    const ExpertLists L = expert_lists_at(call->d_lists ? const_cast<void *>(call->d_lists) : (uint8_t *)d_workspace + s.lists, tokens, k, experts);
    if (call->d_lists) {
        if (int32_t rc = quantised_input(a, X, x_rows, W->K, s, d_workspace, st)) return rc;
    } else if (X->type == CL_MX4) {
        if (int32_t rc = launch_expert_lists(call->d_experts, tokens, k, experts, L, nullptr, st)) return rc;
        if (int32_t rc = quantised_input(a, X, x_rows, W->K, s, d_workspace, st)) return rc;
    } else {
        const QuantiseRows rows{X->d_X, X->type, X->stride, x_rows, W->K, (uint8_t *)d_workspace + s.x_codes, (uint8_t *)d_workspace + s.x_scales};
        a.x_codes = rows.codes;
        a.x_scales = rows.scales;
        if (int32_t rc = launch_expert_lists(call->d_experts, tokens, k, experts, L, &rows, st)) return rc;
    }
    a.x_div = make_div(call->x_per_pair ? 1u : (uint32_t)k);
    a.order = L.order;
    a.Y = d_Y;
    if (int32_t rc = run_experts(a, c, L, *call, (float *)((uint8_t *)d_workspace + s.pairs), y_type, st)) return rc;
    clear_error();
    return CL_OK;
}
