// Products with 8-bit matrices that have a scale for each block of 128 x 128, on the 8-bit matrix instructions.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "f8_common.hpp"

namespace cl {
namespace f8 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// What a product kernel reads and writes.  Rows are `blocks` blocks of 128 bytes; scales have `pitch_scales` numbers to a row of blocks.
//
// y[n][o] = act(sum over blocks j of sx[n][j] sw[o / 128][j] p_j + v[o]) with p_j the sum of 128 products of 8-bit values: one matrix instruction, whose
// sums start at zero, and a multiplication by both scales where its result joins the others.  Rows of a gated product: `width` gates and
// as many values, each with blocks of its own.
struct ProductArgs {
    const uint8_t *w, *x;
    const float *w_scales, *x_scales, *bias;
    void *Y;
    float *y_scales;
    int blocks, pitch_scales;
    int width;                                               // outputs of a row
    int rows, act;
    int value_tall;                                          // gated: where the values' rows of scales start
    float *part;                                             // not null: sums of a share of k, [split][row of Y][pitch], gates and values apart, to be finished
    int pitch, value_at;
    int splits;
    int split_fours, split_more;                             // fours of steps of 128 k of a share of k, and how many shares have one more
    Div band_tiles;                                          // of a band of four columns of tiles
};

// Eight 8-bit values in 16 bits.
__device__ __forceinline__ bf16x8 wide(int lo, int hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The sum over 128 k of A[row][k] B[col][k], 8 bits each.  Lane l has row (A) and column (B) l % 16 and 32 of the k, whole runs of eight of them (which ones does
// not matter, as long as it is the same in both).  Of the result, [i] is row 4 (l / 16) + i, column l % 16.
//
// The 8-bit instructions line up the products of each run of eight k by the largest and cut off what is more than 13 bits below it (measured: a product of
// 2^-14 of the largest is lost, beside a product of another run one of 2^-23 is not); sums of runs are 32 bits.  So a run is off by less than 7 * 2^-13 of its
// largest product - with activations and weights as they are, 1.4e-5 to 5e-5 of a sum (2-norm), a hundredth of the rounding of an output in bf16, a
// tenth of one in fp16.  An output in fp32 has the bits to show it; so has, behind a second product, one in 8 bits: a value next to the middle of two steps goes to
// one or the other by the last bits of its sum (outputs in bf16 of two layers one after the other were up to 5.7e-3 off instead of the rounding's 1.7e-3, of 32 rows of
// 194 numbers).  For these WIDE takes the operands to bf16, which is exact, and multiplies on the bf16 instructions,
// whose products and sums are 32 bits, at half the rate.
template <bool WIDE> struct OperandOf { typedef i32x8 type; };
template <> struct OperandOf<true> { struct type { bf16x8 v[4]; }; };
template <bool WIDE> using Operand = typename OperandOf<WIDE>::type;

template <bool WIDE> __device__ __forceinline__ Operand<WIDE> operand(i32x8 a)
{
    if constexpr (!WIDE) return a;
    else return {{wide(a[0], a[1]), wide(a[2], a[3]), wide(a[4], a[5]), wide(a[6], a[7])}};
}

template <bool WIDE> __device__ __forceinline__ f32x4 mfma_f8(const Operand<WIDE> &a, const Operand<WIDE> &b)
{
    if constexpr (!WIDE) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
    } else {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], acc, 0, 0, 0);
        return acc;
    }
}

__device__ __forceinline__ i32x8 both(i32x4 lo, i32x4 hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

struct F8Out {};

// bias of four outputs from o on (of the values: at = width)
__device__ __forceinline__ f32x4 bias_of(const ProductArgs &a, int at, int o)
{
    f32x4 b = {0, 0, 0, 0};
    if (!a.bias) return b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = a.bias[at + min(o + i, a.width - 1)];
    return b;
}

// g / (1 + exp(-g)), by the hardware's exponential and reciprocal, each off by one unit in the last place.  The exponential's argument is off by |g| 2^-24, which an
// output in 16 bits does not show (at its worst 2^-17 of it).  EXACT, for fp32 and 8 bits: what rounding leaves of -g log2(e), and log2(e) itself, goes in as a
// factor (the minimum, of floats as whole numbers, which keeps negative ones: an infinite gate leaves NaN); the whole is then within 9 2^-24 (62 without).  Of 4096 rows of 2 x 9216 with 8-bit outputs that takes 3 us of 538
// (K 4096), 7 of 166 (K 1024), with fp32 outputs none; for 128 outputs a lane, the library's exponential and a division take 4 of a tile's 40 us.  Gates below -87, whose output is
// below 2^-119 of the value, come out as zeros.
template <bool EXACT> __device__ __forceinline__ float silu(float g)
{
    const float log2e = 1.44269504f, rest = 1.92596299e-8f, ln2 = 0.693147181f;
    if (!EXACT) return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-log2e * g));
    const float c = __int_as_float(min(__float_as_int(g), __float_as_int(100.0f))), t = -log2e * c, left = fmaf(-rest, c, fmaf(-log2e, c, -t));
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t) * fmaf(left, ln2, 1.0f));
}

// T: the output's type.
template <class T, bool GATED> __device__ __forceinline__ f32x4 activated(const ProductArgs &a, int o, f32x4 v, f32x4 u)
{
    if (a.bias) v += bias_of(a, 0, o);
    if (GATED) {
        if (a.bias) u += bias_of(a, a.width, o);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = silu<!std::is_same_v<T, bf16_t> && !std::is_same_v<T, f16_t>>(v[i]) * u[i];
    } else if (a.act == CL_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];            // (NaN stays)
    }
    return v;
}

// The outputs o .. o + 3 of one row of Y.
template <class T> __device__ __forceinline__ void store_outputs(const ProductArgs &a, int64_t row, int o, f32x4 v)
{
    if (o >= a.width) return;
    T *y = (T *)a.Y + row * a.width + o;
    const T out[4] = {(T)product32(v[0], 1.0f), (T)product32(v[1], 1.0f), (T)product32(v[2], 1.0f), (T)product32(v[3], 1.0f)};
    if (o + 4 <= a.width) {
        store_values<4>(y, out);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (o + i < a.width) y[i] = out[i];
    }
}

// Four sums of a share of k.  (A row of partial sums is padded to whole fours.)
__device__ __forceinline__ void store_part(const ProductArgs &a, int split, int64_t row, int o, f32x4 v, int at)
{
    if (o < a.width) *(f32x4 *)(a.part + ((int64_t)split * a.rows + row) * a.pitch + at + o) = v;
}

#include "few_kernel.hpp"
#include "tile_kernel.hpp"
#include "small_tile_kernel.hpp"

// The sum over the splits of a product's parts, in order, and from it four outputs of one row.  8-bit outputs: 32 lanes have a block.
template <class T, bool GATED> __global__ __launch_bounds__(256) void f8_finish_kernel(ProductArgs a, Div quads, int row0, int rows)
{
    constexpr bool kF8 = std::is_same_v<T, F8Out>;
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = quads.quotient(at);
    if (row >= (uint32_t)rows) return;                       // (8-bit outputs: the lanes of a block together)
    const int o = (int)(at - row * quads.d) * 4;
    const int64_t t = (int64_t)row0 + row, stride = (int64_t)a.rows * a.pitch;
    f32x4 v = {0, 0, 0, 0}, u = {0, 0, 0, 0};
    if (o < a.width) {
        const float *p = a.part + t * a.pitch + o;
        v = *(const f32x4 *)p;
        if (GATED) u = *(const f32x4 *)(p + a.value_at);
        for (int s = 1; s < a.splits; ++s) {
            v += *(const f32x4 *)(p + s * stride);
            if (GATED) u += *(const f32x4 *)(p + a.value_at + s * stride);
        }
        v = activated<T, GATED>(a, o, v, u);
    }
    if constexpr (kF8) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = o + i < a.width ? v[i] : 0.0f;
        const Scale s = scale_of(top_of_lanes<32>(top_bits<4>(y)));
        const int y_blocks = (int)quads.d / 32, b = o / kBlock;
        *(uint32_t *)((uint8_t *)a.Y + t * y_blocks * kBlock + o) = to_f8(y, s.inverse);
        if (o % kBlock == 0) {
            const int pitch = (y_blocks + 3) / 4 * 4;
            float *to = a.y_scales + t * pitch;
            to[b] = s.scale;
            if (b == y_blocks - 1)
                for (int i = y_blocks; i < pitch; ++i) to[i] = 0.0f;
        }
    } else {
        store_outputs<T>(a, t, o, v);
    }
}

// ------------------------------------------------------------------------- //
// which kernel
// ------------------------------------------------------------------------- //
constexpr int kCus = 256;
enum Form { kFew, kTile64, kTile128, kTile256 };
constexpr int kFormRows[] = {16, 64, 128, 256}, kFormThreads[] = {0, 256, 512, 512};        // of a workgroup: rows of W; threads (kFew: as many as few_threads says)
constexpr int form_columns(Form form, bool wide) { return form == kTile256 && wide ? 128 : kFormRows[form]; }      // rows of X

// A call, by what the choice of a kernel depends on.
struct Shape {
    int32_t width, blocks, batch;
    bool gated, wide;                                        // wide: sums of 32 bits within a block
    int32_t x_type, y_type;
};
struct Choice {
    Form form;
    int splits;
    bool own;                                                // kFew: quantises X itself
    float us;
};

// Outputs that show the 8-bit instruction's sums (see mfma_f8).
static bool is_wide(int32_t y_type) { return y_type == CL_F32 || y_type == CL_F8; }

static bool few_own(const Shape &s) { return s.x_type != CL_F8 && few_lds(s.blocks, std::min(s.batch, kFewColumns)) <= kFewLds; }

// Wavefronts of a workgroup of few_kernel that share out the blocks of a row, and all: more where there is much to quantise.
static int few_waves(int blocks) { return std::min(kFewWaves, blocks); }
static int few_threads(const Shape &s, bool own)
{
    const int columns = std::min(s.batch, kFewColumns);
    return 64 * std::max(few_waves(s.blocks), own ? (int)std::min<int64_t>(kFewWaves, ((int64_t)columns * s.blocks * 16 + 127) / 128) : 1);
}

static int64_t row_tiles_of(Form form, int32_t width, bool gated)
{
    const int64_t outputs = form == kFew || !gated ? kFormRows[form] : kFormRows[form] / 2;
    return (width + outputs - 1) / outputs;
}

static int64_t columns_of(Form form, int64_t rows, bool wide) { return (rows + form_columns(form, wide) - 1) / form_columns(form, wide); }

// Whether 8-bit outputs are made where the product ends: where a workgroup has all 128 of a block.
static bool ends_in_f8(const Shape &s, const Choice &c) { return s.y_type == CL_F8 && c.splits == 1 && (c.form == kTile256 || (c.form == kTile128 && !s.gated)); }
static bool needs_parts(const Shape &s, const Choice &c) { return c.splits > 1 || (s.y_type == CL_F8 && !ends_in_f8(s, c)); }

// Whether the launch has less than 2^32 threads along each axis.
static bool fits_grid(const Choice &c, const Shape &s)
{
    const int64_t row_tiles = row_tiles_of(c.form, s.width, s.gated), columns = columns_of(c.form, s.batch, s.wide);
    const int64_t wgs = c.form == kFew ? row_tiles : (int64_t)round_up(row_tiles * columns, 8), threads = c.form == kFew ? few_threads(s, c.own) : kFormThreads[c.form];
    return wgs <= (int64_t)UINT32_MAX / threads;
}

template <Form F, class T, bool GATED, bool WIDE> static int32_t launch_tiles(ProductArgs a, const Choice &c, hipStream_t st)
{
    using C = std::conditional_t<F == kTile256, std::conditional_t<WIDE, Tile<256, 128, 4, 2>, Tile<256, 256, 2, 4>>,
                                 std::conditional_t<F == kTile128, SmallTile<128, 128, 2, 4>, SmallTile<64, 64, 2, 2>>>;
    static_assert(C::kThreads == kFormThreads[F], "");
    constexpr size_t kLds = C::kLds + (std::is_same_v<T, F8Out> ? C::kTops : 0);
    void (*kernel)(ProductArgs, int);
    if constexpr (F == kTile256 && WIDE) kernel = f8_tile_kernel<256, 128, 4, 2, T, GATED, WIDE>;
    else if constexpr (F == kTile256) kernel = f8_tile_kernel<256, 256, 2, 4, T, GATED, WIDE>;
    else if constexpr (F == kTile128) kernel = f8_small_tile_kernel<128, 128, 2, 4, T, GATED, WIDE>;
    else kernel = f8_small_tile_kernel<64, 64, 2, 2, T, GATED, WIDE>;
    static LdsLimit seen;
    if (int32_t rc = allow_lds((const void *)kernel, kLds, seen)) return rc;
    const int64_t row_tiles = row_tiles_of(F, a.width, GATED), columns = columns_of(F, a.rows, WIDE);
    a.band_tiles = make_div((uint32_t)row_tiles * 4u);
    const int fours = (a.blocks + 3) / 4;
    if (c.splits < 1 || c.splits > fours) return fail(CL_EINVAL, "%d blocks of k in %d shares", a.blocks, c.splits);      // (a share without steps would read off its operands)
    a.split_fours = fours / c.splits;
    a.split_more = fours % c.splits;
    const size_t wgs = round_up(row_tiles * columns, 8);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(F == kTile256 ? std::min<size_t>(wgs, kCus) : wgs), (unsigned)c.splits), dim3(C::kThreads), kLds, st, a, (int)row_tiles);
    MX_HIP_TRY(hipGetLastError());
    return CL_OK;
}

// x: what few_kernel quantises itself; else a.x.
template <class X, class T, bool GATED, bool WIDE> static int32_t launch_few(const ProductArgs &a, const Shape &s, const cl_f8_input &x, int32_t K, hipStream_t st)
{
    constexpr bool kOwn = !std::is_same_v<X, F8In>;
    auto kernel = f8_few_kernel<X, T, GATED, WIDE>;
    const int columns = std::min(s.batch, kFewColumns);
    const size_t sums = (size_t)few_waves(s.blocks) * (GATED ? 2 : 1) * 64 * sizeof(f32x4);
    static LdsLimit seen;
    if (int32_t rc = allow_lds((const void *)kernel, kFewLds + kFewWaves * 2 * 64 * sizeof(f32x4), seen)) return rc;
    const FewArgs f{a, x.d_X, x.stride, make_div((uint32_t)s.blocks * (kBlock / 8)), K, columns, few_waves(s.blocks)};
    hipLaunchKernelGGL(kernel, dim3((unsigned)((s.width + 15) / 16), (unsigned)((s.batch + kFewColumns - 1) / kFewColumns)), dim3((unsigned)few_threads(s, kOwn)),
                       (kOwn ? few_lds(s.blocks, columns) : 0) + sums, st, f);
    MX_HIP_TRY(hipGetLastError());
    return CL_OK;
}

// T: what the kernel stores.
template <class T, bool GATED, bool WIDE> static int32_t launch_product(const ProductArgs &a, const Shape &s, const Choice &c, const cl_f8_input &x, int32_t K, hipStream_t st)
{
    switch (c.form) {
    case kTile64: return launch_tiles<kTile64, T, GATED, WIDE>(a, c, st);
    case kTile128: return launch_tiles<kTile128, T, GATED, WIDE>(a, c, st);
    case kTile256: return launch_tiles<kTile256, T, GATED, WIDE>(a, c, st);
    default: break;
    }
    if (!c.own) return launch_few<F8In, T, GATED, WIDE>(a, s, x, K, st);
    return with_type(x.type, [&](auto t) { return launch_few<decltype(t), T, GATED, WIDE>(a, s, x, K, st); });
}

// launch(row0, rows, workgroups) over rows of `quads` threads each, in pieces whose threads' numbers have 32 bits.
template <class F> static int32_t launch_rows(int32_t rows, uint32_t quads, F launch)
{
    const int32_t most = (int32_t)std::min<int64_t>(rows, std::max<int64_t>(1, (1ll << 31) / quads));
    for (int32_t row0 = 0, n; row0 < rows; row0 += n) {
        n = std::min(most, rows - row0);
        launch(row0, n, dim3((uint32_t)(((int64_t)n * quads + 255) / 256)));
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
}

template <bool GATED> static int32_t run_product(ProductArgs a, const Shape &s, const Choice &c, const cl_f8_input &x, int32_t K, hipStream_t st)
{
    a.splits = c.splits;
    if (!a.part) {
        if (s.y_type == CL_F32) return launch_product<float, GATED, true>(a, s, c, x, K, st);
        if (s.y_type == CL_BF16) return launch_product<bf16_t, GATED, false>(a, s, c, x, K, st);
        if (s.y_type == CL_F16) return launch_product<f16_t, GATED, false>(a, s, c, x, K, st);
        if (c.form == kTile256) return launch_tiles<kTile256, F8Out, GATED, true>(a, c, st);
        if constexpr (!GATED) return launch_tiles<kTile128, F8Out, false, true>(a, c, st);
    }
    if (int32_t rc = s.wide ? launch_product<float, GATED, true>(a, s, c, x, K, st) : launch_product<float, GATED, false>(a, s, c, x, K, st)) return rc;
    auto finish = [&](auto t, uint32_t quads) {
        return launch_rows(a.rows, quads, [&](int row0, int rows, dim3 grid) {
            hipLaunchKernelGGL((f8_finish_kernel<decltype(t), GATED>), grid, dim3(256), 0, st, a, make_div(quads), row0, rows);
        });
    };
    if (s.y_type == CL_F8) return finish(F8Out{}, (uint32_t)blocks_of(a.width) * 32);
    return with_type(s.y_type, [&](auto t) { return finish(t, (uint32_t)(a.width + 3) / 4); });
}

static int32_t check_forward(const cl_f8_matrix *W, int32_t batch, int32_t x_type, int32_t y_type, int32_t act)
{
    if (!W) return fail(CL_EINVAL, "null pointer");
    if (W->rows < 1 || W->K < 1) return fail(CL_EINVAL, "bad matrix: %d x %d", (int)W->rows, (int)W->K);
    if (W->K > CL_F8_MAX_K) return fail(CL_EUNSUPPORTED, "rows of more than %d elements", (int)CL_F8_MAX_K);
    if (W->rows > INT_MAX - 512) return fail(CL_EUNSUPPORTED, "a matrix of %d rows", (int)W->rows);
    if (batch < 0) return fail(CL_EINVAL, "batch of %d", (int)batch);
    if (!known_type(x_type) && x_type != CL_F8) return fail(CL_EINVAL, "unknown element type %d", (int)x_type);
    if (!known_type(y_type) && y_type != CL_F8) return fail(CL_EINVAL, "unknown element type %d", (int)y_type);
    if (act != CL_ACT_NONE && act != CL_ACT_RELU && act != CL_ACT_GATED) return fail(CL_EINVAL, "unknown activation %d", (int)act);
    if (act == CL_ACT_GATED && W->rows % 2) return fail(CL_EINVAL, "a gated product needs an even number of rows, got %d", (int)W->rows);
    return CL_OK;
}

static int32_t check_pointers(const cl_f8_matrix *W, const cl_f8_input *X, const void *Y, const void *y_scales, int32_t y_type, int64_t rows)
{
    if (!W->d_values || !W->d_scales || !X->d_X || !Y) return fail(CL_EINVAL, "null pointer");
    if (Y == X->d_X) return fail(CL_EINVAL, "the output and the input are one");
    if (!aligned(W->d_values, 16) || !aligned(W->d_scales, 16)) return fail(CL_EINVAL, "values and scales must be 16-byte aligned");
    if (X->type == CL_F8) {
        if (!X->d_scales) return fail(CL_EINVAL, "null pointer");
        if (!aligned(X->d_X, 16) || !aligned(X->d_scales, 16)) return fail(CL_EINVAL, "values and scales must be 16-byte aligned");
    } else {
        if (!aligned(X->d_X, type_bytes(X->type))) return fail(CL_EINVAL, "elements are not aligned");
        if (rows > 1 && X->stride < W->K) return fail(CL_EINVAL, "rows of %d elements overlap at a stride of %lld", (int)W->K, (long long)X->stride);
    }
    if (y_type == CL_F8) {
        if (!y_scales) return fail(CL_EINVAL, "null pointer");
        if (!aligned(Y, 16) || !aligned(y_scales, 16)) return fail(CL_EINVAL, "values and scales must be 16-byte aligned");
    } else if (!aligned(Y, type_bytes(y_type))) {
        return fail(CL_EINVAL, "elements are not aligned");
    }
    return CL_OK;
}

// Scratch of a call, by what is in it.
struct Scratch {
    size_t x_values = 0, x_scales = 0, parts = 0, bytes = 0;
    size_t take(size_t n) { const size_t at = bytes; bytes += round_up(n, 256); return at; }
};

static size_t part_pitch(int32_t width, bool gated) { return round_up(width, 4) * (gated ? 2 : 1); }

static Scratch scratch_of(const Shape &s, const Choice &c, int32_t K)
{
    Scratch at;
    if (s.x_type != CL_F8 && !c.own) {
        at.x_values = at.take((size_t)s.batch * s.blocks * kBlock);
        at.x_scales = at.take((size_t)s.batch * scales_of(K) * 4);
    }
    if (needs_parts(s, c)) at.parts = at.take((size_t)c.splits * s.batch * part_pitch(s.width, s.gated) * 4);
    return at;
}

// What a form takes in microseconds, fitted to measurements of 1800 shapes - 100 .. 4096 rows of W (gated: twice 100 .. 9216), K 100 .. 25088, 1 .. 4096 rows of X, outputs of
// bf16 and of fp32 -: the choice then takes 1.1 % longer, in the mean of logarithms, than the best of up to thirteen.
// Tiles: a start (launch, first loads, last stores), and per step of 128 k what a workgroup takes alone on its compute unit; 64 x 64: its share of a full one, where the launch has more
// workgroups than the chip has compute units; the larger, of which a compute unit has one at a time: how much of a last round that is not full counts; what each further
// workgroup of a compute unit adds.
struct Price { float start, alone, shared, last, more; };
constexpr Price kPrices[2][4] = {{{}, {3.1f, 0.273f, 0.259f, 0, 1.0f}, {4.0f, 0.447f, 0, 0.84f, 3.9f}, {7.0f, 1.25f, 0, 0.82f, 8.2f}},
                                 {{}, {3.35f, 0.535f, 0.432f, 0, 1.7f}, {4.7f, 0.99f, 0, 0.47f, 7.7f}, {6.4f, 1.69f, 0, 0.77f, 9.8f}}};
// few_kernel: a start; per block of 128 k and 256 workgroups of rows of W and of X (from 0.6 or 0.7 of that on, which is as fast as a workgroup gets); what it quantises.
struct FewPrice { float start, row, column, at_least, quantise; };
constexpr FewPrice kFewPrices[2] = {{2.55f, 0.103f, 0.003f, 0.71f, 0.0015f}, {3.4f, 0.095f, 0.014f, 0.6f, 0.0022f}};       // X in 8 bits; in numbers
// The quantisation of X, the sum of partial sums.  A launch costs the host, besides, some 4 us, which calls one by one pay, and calls recorded in a graph do not: half of it counts.
constexpr float kLaunch = 2.0f;
constexpr int32_t kFewMostRows = 256;                        // (beyond, tiles are always faster)
static_assert(kFewMostRows / kFewColumns < 65536, "");       // (the height of its grid)

static float price_of(const Shape &s, const Choice &c)
{
    const int64_t row_tiles = row_tiles_of(c.form, s.width, s.gated), columns = columns_of(c.form, s.batch, s.wide);
    const float M = (float)s.width * (s.gated ? 2 : 1), n = (float)row_tiles * columns * c.splits / kCus;
    float us;
    if (c.form == kFew) {
        const FewPrice &p = kFewPrices[c.own];
        const int cols = std::min(s.batch, kFewColumns);
        us = p.start + s.blocks * ((p.row * (s.gated ? 2 : 1) + p.column * cols) * std::max(n, p.at_least) + p.quantise * cols);
    } else {
        const Price &p = kPrices[s.wide][c.form];
        const int fours = (s.blocks + 3) / 4, steps = std::min(s.blocks, (fours + c.splits - 1) / c.splits * 4);
        if (c.form == kTile64) {
            us = p.start + steps * std::max(p.alone, p.shared * n) + p.more * std::max(0.0f, n - 1);
        } else {
            const float rounds = std::max(1.0f, n + p.last * (std::ceil(n) - n));
            us = p.start + steps * p.alone * rounds + p.more * (rounds - 1);
        }
    }
    if (s.x_type != CL_F8 && !c.own) us += 2.9f + kLaunch + 2.1e-7f * s.batch * s.blocks * kBlock * type_bytes(s.x_type);
    if (needs_parts(s, c)) us += 1.7f + kLaunch + 0.85e-6f * (2 * c.splits + 1) * s.batch * M;
    return us;
}

// The cheapest form that fits a grid and whose scratch has at most `most` bytes; us < 0: there is none.  What one form needs for a batch is enough for the same form, not split, and a smaller batch: so
// is what is asked for.
static Choice choose(const Shape &s, int32_t K, size_t most)
{
    Choice best{kFew, 1, false, -1.0f};
    auto offer = [&](Form form, int splits, bool own) {
        Choice c{form, splits, own, 0.0f};
        c.us = price_of(s, c);
        if ((best.us < 0.0f || c.us < best.us) && fits_grid(c, s) && scratch_of(s, c, K).bytes <= most) best = c;
    };
    if (s.batch <= kFewMostRows) {
        offer(kFew, 1, false);
        if (few_own(s)) offer(kFew, 1, true);
    }
    const int fours = (s.blocks + 3) / 4;
    for (int form = kTile64; form <= kTile256; ++form) {
        const int64_t n = row_tiles_of((Form)form, s.width, s.gated) * columns_of((Form)form, s.batch, s.wide);
        for (int splits = 1; splits <= 8 && splits <= fours && (splits == 1 || n * splits <= 4 * kCus); splits *= 2) offer((Form)form, splits, false);
    }
    return best;
}

static int32_t fail_with_grid(const Shape &s) { return fail(CL_EUNSUPPORTED, "%d rows of %d outputs do not fit a grid", (int)s.batch, (int)s.width); }

static Shape shape_of(const cl_f8_matrix &W, int32_t batch, int32_t x_type, int32_t y_type, int32_t act)
{
    const bool gated = act == CL_ACT_GATED;
    return Shape{gated ? W.rows / 2 : W.rows, blocks_of(W.K), batch, gated, is_wide(y_type), x_type, y_type};
}

}  // namespace f8
}  // namespace cl

using namespace cl;
using namespace cl::f8;

extern "C" int32_t cl_eight_fc_workspace_bytes(const cl_f8_matrix *W, int32_t batch, int32_t x_type, int32_t y_type, int32_t act, size_t *out)
{
    if (!out) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, batch, x_type, y_type, act)) return rc;
    const Shape s = shape_of(*W, batch, x_type, y_type, act);
    const Choice c = choose(s, W->K, SIZE_MAX);
    if (c.us < 0.0f) return fail_with_grid(s);
    *out = scratch_of(s, c, W->K).bytes;
    clear_error();
    return CL_OK;
}

static_assert(CL_F8_FORM_FEW == 1 + kFew && CL_F8_FORM_TILE_64 == 1 + kTile64 && CL_F8_FORM_TILE_256 == 1 + kTile256, "");

extern "C" int32_t cl_eight_fc_resolved_form(const cl_f8_matrix *W, int32_t batch, int32_t x_type, int32_t y_type, int32_t act, int32_t *form, int32_t *splits)
{
    if (!form || !splits) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, batch, x_type, y_type, act)) return rc;
    const Shape s = shape_of(*W, batch, x_type, y_type, act);
    const Choice c = choose(s, W->K, SIZE_MAX);
    if (c.us < 0.0f) return fail_with_grid(s);
    *form = c.own ? CL_F8_FORM_FEW_NUMBERS : 1 + c.form;
    *splits = c.splits;
    clear_error();
    return CL_OK;
}

extern "C" int32_t cl_eight_fc_forward(const cl_f8_matrix *W, const cl_f8_input *X, const float *d_bias, void *d_Y, float *d_y_scales, int32_t y_type, int32_t batch, int32_t act,
                                       void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!X) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, batch, X->type, y_type, act)) return rc;
    if (batch == 0) return CL_OK;
    if (int32_t rc = check_pointers(W, X, d_Y, d_y_scales, y_type, batch)) return rc;
    hipStream_t st = (hipStream_t)stream;
    const Shape s = shape_of(*W, batch, X->type, y_type, act);
    const Choice c = choose(s, W->K, d_workspace ? workspace_bytes : 0);
    if (c.us < 0.0f) {
        const Choice any = choose(s, W->K, SIZE_MAX);
        if (any.us < 0.0f) return fail_with_grid(s);
        return fail(CL_EINVAL, "workspace needs %zu bytes, got %zu", scratch_of(s, any, W->K).bytes, d_workspace ? workspace_bytes : 0);
    }
    const Scratch at = scratch_of(s, c, W->K);
    if (at.bytes && !aligned(d_workspace, 256)) return fail(CL_EINVAL, "workspace must be 256-byte aligned");
    uint8_t *ws = (uint8_t *)d_workspace;
    ProductArgs a{};
    a.w = (const uint8_t *)W->d_values;
    a.w_scales = W->d_scales;
    a.bias = d_bias;
    a.Y = d_Y;
    a.y_scales = d_y_scales;
    a.blocks = s.blocks;
    a.pitch_scales = scales_of(W->K);
    a.width = s.width;
    a.rows = batch;
    a.act = act;
    a.value_tall = (s.width + kBlock - 1) / kBlock;
    if (X->type == CL_F8) {
        a.x = (const uint8_t *)X->d_X;
        a.x_scales = X->d_scales;
    } else if (!c.own) {
        a.x = ws + at.x_values;
        a.x_scales = (const float *)(ws + at.x_scales);
        if (int32_t rc = launch_rows_to_f8(X->d_X, X->type, X->stride, batch, W->K, ws + at.x_values, (float *)(ws + at.x_scales), st)) return rc;
    }
    if (needs_parts(s, c)) a.part = (float *)(ws + at.parts);
    a.pitch = (int)part_pitch(s.width, s.gated);
    a.value_at = (int)round_up(s.width, 4);
    if (int32_t rc = s.gated ? run_product<true>(a, s, c, *X, W->K, st) : run_product<false>(a, s, c, *X, W->K, st)) return rc;
    clear_error();
    return CL_OK;
}
