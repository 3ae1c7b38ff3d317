// Rows of numbers to blocks of 32 four-bit floats under one power-of-two scale (OCP MXFP4: E2M1 elements, E8M0 scale), and back.
#include "quantize_kernel.hpp"

namespace cl {
namespace mx {

template <class T, bool STREAM> __global__ __launch_bounds__(256) void mx_quantize_kernel(QuantiseArgs a) { quantise_units<T, STREAM>(blockIdx.x, a); }

template <class T, bool STREAM>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const void *__restrict__ codes, const uint8_t *__restrict__ scales, uint32_t units,
                                                            Div per_row, int K, T *__restrict__ Y, int64_t stride)
{
    typedef Unit<T> U;
    constexpr int V = U::kValues, kLanes = 32 / V;
    uint32_t c[kUnits], byte[kUnits];
    const uint32_t first = blockIdx.x * (256u * kUnits) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = min(first + i * 256u, units - 1);
        c[i] = ((const typename U::Codes *)codes)[u];
        byte[i] = scales[u / kLanes];
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = first + i * 256u;
        if (u >= units) return;
        const uint32_t row = per_row.quotient(u);
        const int k0 = (int)(u - row * per_row.d) * V, left = K - k0;
        if (left <= 0) continue;
        const float s = scale_value(byte[i]);
        f32x2 v[4];
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], 1.0f, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], 1.0f, 1);
        if (V == 8) {
            v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], 1.0f, 2);
            v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], 1.0f, 3);
        }
        T y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = (T)product32(v[j / 2][j % 2], s);
        T *out = Y + (int64_t)row * stride + k0;
        if (left >= V) {
            typename U::Bytes b;
            __builtin_memcpy(&b, y, 16);
            if (STREAM) __builtin_nontemporal_store(b, (typename U::Bytes *)out);
            else *(typename U::Bytes *)out = b;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < left) out[j] = y[j];
        }
    }
}

// launch(rows before it, units, kernel of these types) for pieces of at most 2^30 units, so that their numbers and the grid fit 32
// bits.
template <class T, class F> static int32_t in_pieces(int64_t rows, int32_t K, F launch)
{
    const uint32_t per_row = (uint32_t)(row_blocks(K) * (32 / Unit<T>::kValues));
    const int64_t step = std::max<int64_t>(1, ((int64_t)1 << 30) / per_row);
    const bool stream = past_caches(rows * K * (int64_t)sizeof(T));
    for (int64_t r = 0; r < rows; r += step) {
        const uint32_t units = (uint32_t)std::min(step, rows - r) * per_row;
        const dim3 grid((units + 256 * kUnits - 1) / (256 * kUnits));
        if (stream) launch(std::true_type{}, grid, r, units, make_div(per_row));
        else launch(std::false_type{}, grid, r, units, make_div(per_row));
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
}

int32_t launch_quantize(const void *X, int32_t type, int64_t stride, int64_t rows, int32_t K, uint8_t *codes, uint8_t *scales, hipStream_t st)
{
    const int64_t kb = row_blocks(K);
    return with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        return in_pieces<T>(rows, K, [&](auto stream, dim3 grid, int64_t r, uint32_t units, Div per_row) {
            const QuantiseArgs a{(const T *)X + r * stride, codes + r * kb * 16, scales + r * kb, stride, per_row, units, K};
            hipLaunchKernelGGL((mx_quantize_kernel<T, stream.value>), grid, dim3(256), 0, st, a);
        });
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
    const int64_t kb = row_blocks(K);
    const int32_t rc = with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        return in_pieces<T>(rows, K, [&](auto past, dim3 grid, int64_t r, uint32_t units, Div per_row) {
            hipLaunchKernelGGL((mx_dequantize_kernel<T, past.value>), grid, dim3(256), 0, (hipStream_t)stream,
                               (const void *)((const uint8_t *)d_codes + r * kb * 16), (const uint8_t *)d_scales + r * kb, units, per_row, K,
                               (T *)d_Y + r * y_stride, y_stride);
        });
    });
    if (rc) return rc;
    clear_error();
    return CL_OK;
}
