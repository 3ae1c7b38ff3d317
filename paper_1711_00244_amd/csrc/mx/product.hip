// Products with microscaled 4-bit matrices on the scaled matrix instructions: one matrix for all rows of X, or one per expert
// for the rows that were routed to it.
#include <algorithm>

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
    const int32_t *tile_count, *offsets;
    int blocks, M, rows, experts, act;
    int out_width;                                           // elements of a row of Y
    int x_div;                                               // pair / x_div is its row of X
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
    c = Columns{t.y, min(WIDTH, a.offsets[t.x + 1] - t.y), t.x};
    return !(c.expert == a.experts && a.skip_unrouted);
}

// Four consecutive outputs of one row of Y, from output m on.
template <class T> __device__ __forceinline__ void store_outputs(const ProductArgs &a, int expert, int64_t row, int m, f32x4 v)
{
    if (m >= a.M) return;
    if (a.bias) {
        const float *b = a.bias + (int64_t)expert * a.M + m;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m + i < a.M) v[i] += b[i];
    }
    T *y = (T *)a.Y + row * a.out_width;
    if (a.act == CL_ACT_GATED) {
        // rows 2 i and 2 i + 1 of the matrix: gate and value of output i
        y += m / 2;
#pragma unroll
        for (int i = 0; i < 4; i += 2)
            if (m + i + 1 < a.M) y[i / 2] = (T)(v[i] / (1.0f + expf(-v[i])) * v[i + 1]);
        return;
    }
    y += m;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (m + i < a.M) y[i] = (T)(a.act == CL_ACT_RELU && v[i] < 0.0f ? 0.0f : v[i])   /* (NaN stays) */;
}

// A workgroup of eight wavefronts makes 16 outputs (blockIdx.x) of 16 NT columns (blockIdx.y).  The wavefronts share out the
// row's runs of 16 blocks; of a run, a lane's group has four consecutive blocks - 64 bytes and one word of scales - which
// are its 32 k of four matrix instructions (the order of k does not matter as long as both operands have the same).
// Their sums meet in LDS and are added in the order of the wavefronts.
constexpr int kRowsWaves = 8;

template <int NT, class T> __global__ __launch_bounds__(kRowsWaves * 64) void mx_rows_kernel(ProductArgs a)
{
    __shared__ f32x4 part[kRowsWaves][NT][64];
    Columns c;
    if (!columns_of<16 * NT>(a, a.tile0 + (int)blockIdx.y, c)) return;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int m0 = (int)blockIdx.x * 16;
    f32x4 acc[NT] = {};
    if (!a.order || c.expert < a.experts) {                  // (the pairs without an expert: zeros)
        const int64_t w_row = (int64_t)c.expert * a.M + min(m0 + r, a.M - 1);
        const uint8_t *wc = a.w_codes + w_row * a.blocks * 16, *ws = a.w_scales + w_row * a.blocks;
        const uint8_t *xc[NT], *xs[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int n = c.first + min(t * 16 + r, c.count - 1);
            const int64_t x_row = a.order ? a.order[n] / a.x_div : n;
            xc[t] = a.x_codes + x_row * a.blocks * 16;
            xs[t] = a.x_scales + x_row * a.blocks;
        }
        for (int b = wave * 16 + g * 4; b - g * 4 < a.blocks; b += kRowsWaves * 16) {
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
    for (int e = threadIdx.x; e < NT * 64; e += kRowsWaves * 64) {
        const int t = e / 64, l = e & 63, n = t * 16 + (l & 15);
        if (n >= c.count) continue;
        f32x4 v = part[0][t][l];
#pragma unroll
        for (int w = 1; w < kRowsWaves; ++w) v += part[w][t][l];
        const int64_t y_row = a.order ? a.order[c.first + n] : c.first + n;
        if (a.order && c.expert == a.experts) {              // no expert: zeros, whatever the activation makes of zero and a bias
            T *y = (T *)a.Y + y_row * a.out_width;
            const int step = a.act == CL_ACT_GATED ? 2 : 1, m = m0 + 4 * (l >> 4);
            for (int i = 0; i < 4; i += step)
                if (m + i + step <= a.M) y[(m + i) / step] = (T)0.0f;
        } else {
            store_outputs<T>(a, c.expert, y_row, m0 + 4 * (l >> 4), v);
        }
    }
}

// Y[t] = sum over j of weights[t][j] P[t k + j], in the order of j, of the pairs that have an expert.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ P, const int32_t *__restrict__ experts_of, const float *__restrict__ weights,
                                                   T *__restrict__ Y, int k, int experts, int width)
{
    const int m = (int)(blockIdx.x * 256u + threadIdx.x);
    if (m >= width) return;
    const int64_t t = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
    float sum = 0.0f;
    for (int j = 0; j < k; ++j) {
        const int e = experts_of[t * k + j];
        if (e >= 0 && e < experts) sum += weights[t * k + j] * P[(t * k + j) * width + m];
    }
    Y[t * width + m] = (T)sum;
}

template <class T> static int32_t launch_product(const ProductArgs &a, int64_t tiles, hipStream_t st)
{
    const int64_t gx = (a.M + 15) / 16;
    // (a grid is at most 65535 high: taller ones go in pieces)
    for (int64_t t0 = 0; t0 < tiles; t0 += 65535) {
        ProductArgs p = a;
        p.tile0 = (int)t0;
        hipLaunchKernelGGL((mx_rows_kernel<4, T>), dim3((unsigned)gx, (unsigned)std::min<int64_t>(tiles - t0, 65535)), dim3(kRowsWaves * 64), 0, st, p);
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
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

static Scratch experts_scratch(int32_t M, int32_t K, int32_t x_type, int64_t x_rows, int32_t tokens, int32_t k, int32_t experts, bool join, bool own_lists, int32_t act)
{
    Scratch s;
    scratch_input(s, x_type, x_rows, K);
    if (join) s.pairs = s.take((size_t)tokens * k * (act == CL_ACT_GATED ? M / 2 : M) * 4);
    if (own_lists) s.lists = s.take(expert_lists_at(nullptr, tokens, k, experts).bytes);
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
    Scratch s;
    scratch_input(s, x_type, batch, W->K);
    *out = s.bytes;
    clear_error();
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
    Scratch s;
    scratch_input(s, X->type, batch, W->K);
    if (int32_t rc = check_scratch(s, d_workspace, workspace_bytes)) return rc;
    hipStream_t st = (hipStream_t)stream;
    ProductArgs a{};
    if (int32_t rc = quantised_input(a, X, batch, W->K, s, d_workspace, st)) return rc;
    a.w_codes = (const uint8_t *)W->d_codes;
    a.w_scales = (const uint8_t *)W->d_scales;
    a.bias = d_bias;
    a.Y = d_Y;
    a.blocks = row_blocks(W->K);
    a.M = W->rows;
    a.rows = batch;
    a.act = act;
    a.out_width = act == CL_ACT_GATED ? W->rows / 2 : W->rows;
    const int32_t rc = with_type(y_type, [&](auto t) { return launch_product<decltype(t)>(a, ((int64_t)batch + 63) / 64, st); });
    if (rc) return rc;
    clear_error();
    return CL_OK;
}

static int32_t check_experts(const cl_mx_matrix *W, int32_t experts, int32_t tokens, int32_t k)
{
    if (experts < 1 || tokens < 0 || k < 1) return fail(CL_EINVAL, "%d tokens, %d of %d experts", (int)tokens, (int)k, (int)experts);
    if (experts > CL_ROUTE_MAX_EXPERTS) return fail(CL_EUNSUPPORTED, "%d experts: at most %d", (int)experts, CL_ROUTE_MAX_EXPERTS);
    if ((int64_t)tokens * k > (int64_t)INT32_MAX - kListChunk) return fail(CL_EUNSUPPORTED, "more than 2^31 pairs of token and expert");
    return CL_OK;
}

extern "C" int32_t cl_mx_experts_workspace_bytes(const cl_mx_matrix *W, int32_t experts, const cl_mx_experts_call *call, int32_t x_type, size_t *out)
{
    if (!out || !call) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_forward(W, x_type, CL_F32, call->act)) return rc;
    if (int32_t rc = check_experts(W, experts, call->tokens, call->k)) return rc;
    const int64_t x_rows = (int64_t)call->tokens * (call->x_per_pair ? call->k : 1);
    *out = experts_scratch(W->rows, W->K, x_type, x_rows, call->tokens, call->k, experts, call->d_weights != nullptr, call->d_lists == nullptr, call->act).bytes;
    clear_error();
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
    const bool join = call->d_weights != nullptr;
    const Scratch s = experts_scratch(W->rows, W->K, X->type, x_rows, tokens, k, experts, join, call->d_lists == nullptr, call->act);
    if (int32_t rc = check_scratch(s, d_workspace, workspace_bytes)) return rc;
    hipStream_t st = (hipStream_t)stream;
    ProductArgs a{};
    const ExpertLists L = expert_lists_at(call->d_lists ? const_cast<void *>(call->d_lists) : (uint8_t *)d_workspace + s.lists, tokens, k, experts);
    if (!call->d_lists)
        if (int32_t rc = launch_expert_lists(call->d_experts, tokens, k, experts, L, st)) return rc;
    if (int32_t rc = quantised_input(a, X, x_rows, W->K, s, d_workspace, st)) return rc;
    a.w_codes = (const uint8_t *)W->d_codes;
    a.w_scales = (const uint8_t *)W->d_scales;
    a.bias = call->d_bias;
    a.blocks = row_blocks(W->K);
    a.M = W->rows;
    a.rows = tokens * k;
    a.experts = experts;
    a.act = call->act;
    a.out_width = call->act == CL_ACT_GATED ? W->rows / 2 : W->rows;
    a.x_div = call->x_per_pair ? 1 : k;
    a.order = L.order;
    a.offsets = L.offsets;
    a.tiles = L.tiles[1];
    a.tile_count = L.tile_count + 1;
    a.skip_unrouted = join;
    a.Y = join ? (uint8_t *)d_workspace + s.pairs : d_Y;
    int32_t rc = with_type(join ? (int32_t)CL_F32 : y_type, [&](auto t) { return launch_product<decltype(t)>(a, L.max_tiles[1], st); });
    if (rc) return rc;
    if (join) {
        rc = with_type(y_type, [&](auto t) -> int32_t {
            using T = decltype(t);
            const unsigned gy = (unsigned)std::min(tokens, 32768), gz = 1;
            for (int32_t t0 = 0; t0 < tokens; t0 += (int32_t)gy) {
                const unsigned n = (unsigned)std::min<int64_t>(gy, tokens - t0);
                hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)((a.out_width + 255) / 256), n, gz), dim3(256), 0, st,
                                   (const float *)a.Y + (int64_t)t0 * k * a.out_width, call->d_experts + (int64_t)t0 * k, call->d_weights + (int64_t)t0 * k,
                                   (T *)d_Y + (int64_t)t0 * a.out_width, k, experts, a.out_width);
                MX_HIP_TRY(hipGetLastError());
            }
            return CL_OK;
        });
        if (rc) return rc;
    }
    clear_error();
    return CL_OK;
}
