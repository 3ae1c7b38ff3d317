// Rows of numbers to blocks of 32 four-bit floats under one power-of-two scale (OCP MXFP4: E2M1 elements, E8M0 scale), and back.
#include "mx_common.hpp"

namespace cl {
namespace mx {

// Division of a 32-bit number by a run-time constant: a high product and two shifts (round-up method; exact for all n).
struct Div {
    uint32_t mul, shift1, shift2, d;
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const
    {
        const uint32_t t = __umulhi(n, mul);
        return (t + ((n - t) >> shift1)) >> shift2;
    }
};

static Div make_div(uint32_t d)
{
    uint32_t s = 0;
    while (s < 32 && (1ull << s) < d) ++s;
    return Div{(uint32_t)((((1ull << s) - d) << 32) / d + 1), s > 0 ? 1u : 0u, s > 0 ? s - 1 : 0u, d};
}

// A unit per lane.
template <class T, bool ALIGNED>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ X, int64_t stride, uint32_t units, Div per_row, int K,
                                                          uint32_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    if (u >= units) return;                                  // (a row has whole blocks: the four lanes of one leave together)
    const uint32_t row = per_row.quotient(u);
    const int k0 = (int)(u - row * per_row.d) * kUnit;
    float x[kUnit];
    load_unit<T>(X + (int64_t)row * stride + k0, K - k0, ALIGNED, x);
    uint32_t byte;
    codes[u] = quantise_unit(x, byte);
    if ((u & 3) == 0) scales[u >> 2] = (uint8_t)byte;
}

template <class T, bool ALIGNED>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, uint32_t units,
                                                            Div per_row, int K, T *__restrict__ Y, int64_t stride)
{
    const uint32_t u = blockIdx.x * 256u + threadIdx.x;
    if (u >= units) return;
    const uint32_t row = per_row.quotient(u);
    const int k0 = (int)(u - row * per_row.d) * kUnit, left = K - k0;
    if (left <= 0) return;
    const uint32_t c = codes[u];
    const float s = scale_value(scales[u >> 2]);
    f32x2 v[4];
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    T y[kUnit];
#pragma unroll
    for (int i = 0; i < kUnit; ++i) y[i] = (T)(v[i / 2][i % 2] * s);
    T *out = Y + (int64_t)row * stride + k0;
    if (ALIGNED && left >= kUnit) {
        __builtin_memcpy(__builtin_assume_aligned(out, 16), y, sizeof y);
    } else {
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
            if (i < left) out[i] = y[i];
    }
}

// Rows of one launch: at most 2^30 units, so that their numbers and the grid fit 32 bits.
static int64_t rows_per_launch(uint32_t units_per_row) { return std::max<int64_t>(1, ((int64_t)1 << 30) / units_per_row); }

int32_t launch_quantize(const void *X, int32_t type, int64_t stride, int64_t rows, int32_t K, uint8_t *codes, uint8_t *scales, hipStream_t st)
{
    const uint32_t upr = (uint32_t)row_blocks(K) * 4;
    const int64_t step = rows_per_launch(upr);
    return with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        const bool ok = aligned(X, 16) && (stride * (int64_t)sizeof(T)) % 16 == 0;
        auto kernel = ok ? mx_quantize_kernel<T, true> : mx_quantize_kernel<T, false>;
        for (int64_t r = 0; r < rows; r += step) {
            const uint32_t units = (uint32_t)std::min(step, rows - r) * upr;
            hipLaunchKernelGGL(kernel, dim3((units + 255) / 256), dim3(256), 0, st, (const T *)X + r * stride, stride, units, make_div(upr), K,
                               (uint32_t *)codes + r * upr, scales + r * (upr / 4));
            MX_HIP_TRY(hipGetLastError());
        }
        return CL_OK;
    });
}

}  // namespace mx
}  // namespace cl

using namespace cl;
using namespace cl::mx;

static int32_t check_rows(const void *x, const void *codes, const void *scales, int32_t type, int64_t stride, int64_t rows, int32_t K)
{
    if (!known_type(type)) return fail(CL_EINVAL, "unknown element type %d", (int)type);
    if (rows < 0 || K < 1) return fail(CL_EINVAL, "bad matrix: %lld rows of %d", (long long)rows, (int)K);
    if (K > CL_MX_MAX_K) return fail(CL_EUNSUPPORTED, "rows of more than %d elements", (int)CL_MX_MAX_K);
    if (rows == 0) return CL_OK;
    if (!x || !codes || !scales) return fail(CL_EINVAL, "null pointer");
    if (rows > 1 && stride < K) return fail(CL_EINVAL, "rows of %d elements overlap at a stride of %lld", (int)K, (long long)stride);
    if (!aligned(codes, 16) || !aligned(scales, 4)) return fail(CL_EINVAL, "codes must be 16-byte and scales 4-byte aligned");
    if (!aligned(x, type_bytes(type))) return fail(CL_EINVAL, "elements are not aligned");
    return CL_OK;
}

extern "C" int32_t cl_mx_quantize(const void *d_X, int32_t type, int64_t x_stride, int64_t rows, int32_t K, void *d_codes, void *d_scales, void *stream)
{
    if (int32_t rc = check_rows(d_X, d_codes, d_scales, type, x_stride, rows, K)) return rc;
    if (int32_t rc = launch_quantize(d_X, type, x_stride, rows, K, (uint8_t *)d_codes, (uint8_t *)d_scales, (hipStream_t)stream)) return rc;
    clear_error();
    return CL_OK;
}

extern "C" int32_t cl_mx_dequantize(const void *d_codes, const void *d_scales, int64_t rows, int32_t K, void *d_Y, int32_t type, int64_t y_stride, void *stream)
{
    if (int32_t rc = check_rows(d_Y, d_codes, d_scales, type, y_stride, rows, K)) return rc;
    const uint32_t upr = (uint32_t)row_blocks(K) * 4;
    const int64_t step = rows_per_launch(upr);
    const int32_t rc = with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        const bool ok = aligned(d_Y, 16) && (y_stride * (int64_t)sizeof(T)) % 16 == 0;
        auto kernel = ok ? mx_dequantize_kernel<T, true> : mx_dequantize_kernel<T, false>;
        for (int64_t r = 0; r < rows; r += step) {
            const uint32_t units = (uint32_t)std::min(step, rows - r) * upr;
            hipLaunchKernelGGL(kernel, dim3((units + 255) / 256), dim3(256), 0, (hipStream_t)stream, (const uint32_t *)d_codes + r * upr,
                               (const uint8_t *)d_scales + r * (upr / 4), units, make_div(upr), K, (T *)d_Y + r * y_stride, y_stride);
            MX_HIP_TRY(hipGetLastError());
        }
        return CL_OK;
    });
    if (rc) return rc;
    clear_error();
    return CL_OK;
}
