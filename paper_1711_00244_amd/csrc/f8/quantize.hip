// Rows of numbers to 8-bit values (E4M3) under a scale for each block of 128 of a row, or of 128 x 128, and back.
#include "f8_common.hpp"

namespace cl {
namespace f8 {

struct ToArgs {
    const void *X;
    uint8_t *values;
    float *scales;
    int64_t stride;
    Div per_row;                                             // units of a row
    uint32_t units;
    int K, pitch;                                            // scales from row to row
};

// 16 bytes of numbers.
template <class T, bool STREAM> __device__ __forceinline__ void load_numbers(const T *p, int left, float *x)
{
    constexpr int V = Unit<T>::kValues;
    if (STREAM && left >= V) {
        const typename Unit<T>::Bytes v = __builtin_nontemporal_load((const typename Unit<T>::Bytes *)p);
        T t[V];
        __builtin_memcpy(t, &v, 16);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = to_float(t[j]);
    } else {
        load_unit<V>(p, left, x);
    }
}

template <int V> __device__ __forceinline__ void store_f8(uint8_t *at, const float *x, float inverse)
{
    if constexpr (V == 4) *(uint32_t *)at = to_f8(x, inverse);
    else *(u32x2 *)at = u32x2{to_f8(x, inverse), to_f8(x + 4, inverse)};
}

// The scale of block b of `blocks` of a row, and behind the last the zeros that pad the row.
__device__ __forceinline__ void store_scale(float *row, int b, int blocks, int pitch, float scale)
{
    row[b] = scale;
    if (b == blocks - 1)
        for (int i = blocks; i < pitch; ++i) row[i] = 0.0f;
}

// Blocks of one row: a lane has 16 bytes of numbers at a time - 16 or 32 lanes to a block -, of what goes past the caches kUnits times (4096 rows of
// 25088 bf16, 308 MB, 51 us, 6.0 TB/s; once 54), else once (333 rows of 1100 fp16 2.6 us, else 3.5; 4096 of 4096 bf16 9.6, else 10.1).  Memory bounds the first, a launch and
// one trip there and back the smallest.
template <class T, bool STREAM> __global__ __launch_bounds__(256) void f8_rows_kernel(ToArgs a)
{
    constexpr int V = Unit<T>::kValues, kLanes = kBlock / V;
    constexpr int kTimes = STREAM ? kUnits : 1;
    float x[kTimes][V];
    const uint32_t first = blockIdx.x * (256u * kTimes) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const uint32_t u = min(first + i * 256u, a.units - 1), row = a.per_row.quotient(u);
        const int k0 = (int)(u - row * a.per_row.d) * V;
        load_numbers<T, STREAM>((const T *)a.X + (int64_t)row * a.stride + k0, a.K - k0, x[i]);
    }
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const uint32_t u = first + i * 256u;
        const Scale s = scale_of(top_of_lanes<kLanes>(top_bits<V>(x[i])));       // (a row has whole blocks: the lanes of one are beyond the end together)
        if (u >= a.units) continue;
        store_f8<V>(a.values + (uint64_t)u * V, x[i], s.inverse);
        if (u % kLanes == 0) {
            const uint32_t row = a.per_row.quotient(u);
            store_scale(a.scales + (uint64_t)row * a.pitch, (int)((u - row * a.per_row.d) / kLanes), (int)(a.per_row.d / kLanes), a.pitch, s.scale);
        }
    }
}

// Blocks of 128 x 128: a workgroup has one, in registers.  Memory bounds it: 4096 x 25088 fp32, 514 MB, 80 us, 6.4 TB/s.
template <class T, bool STREAM> __global__ __launch_bounds__(256) void f8_blocks_kernel(ToArgs a, int64_t rows, int blocks)
{
    constexpr int V = Unit<T>::kValues, kLanes = kBlock / V, kRows = 256 / kLanes, kTimes = kBlock / kRows;
    __shared__ uint32_t tops[4];
    const uint32_t tall = a.per_row.quotient(blockIdx.x);
    const int b = (int)(blockIdx.x - tall * a.per_row.d), k0 = b * kBlock + (int)threadIdx.x % kLanes * V, left = a.K - k0;
    const int64_t row0 = (int64_t)tall * kBlock + threadIdx.x / kLanes;
    float x[kTimes][V];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const int64_t row = row0 + i * kRows;
        load_numbers<T, STREAM>((const T *)a.X + row * a.stride + k0, row < rows ? left : 0, x[i]);
    }
#pragma unroll
    for (int i = 0; i < kTimes; ++i) top = max(top, top_bits<V>(x[i]));
    top = top_of_lanes<32>(top);
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
    __syncthreads();
    const Scale s = scale_of(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const int64_t row = row0 + i * kRows;
        if (row < rows) store_f8<V>(a.values + row * blocks * kBlock + k0, x[i], s.inverse);
    }
    if (threadIdx.x == 0) store_scale(a.scales + (int64_t)tall * a.pitch, b, blocks, a.pitch, s.scale);
}

// Back: a lane makes 16 bytes of numbers, of what goes past the caches kUnits times.  Memory bounds it: 4096 x 25088 from blocks of 128 x 128 to fp32, 514 MB, 81 us, 6.3 TB/s;
// to bf16, 308 MB, 50 us, 6.2 TB/s.
template <class T, bool STREAM>
__global__ __launch_bounds__(256) void f8_back_kernel(const uint8_t *__restrict__ values, const float *__restrict__ scales, int64_t row0, int block_rows, uint32_t units,
                                                      Div per_row, int K, int pitch, T *__restrict__ Y, int64_t stride)
{
    constexpr int V = Unit<T>::kValues, kLanes = kBlock / V;
    constexpr int kTimes = STREAM ? kUnits : 1;
    uint32_t c[kTimes][V / 4];
    float s[kTimes];
    const uint32_t first = blockIdx.x * (256u * kTimes) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const uint32_t u = min(first + i * 256u, units - 1), row = per_row.quotient(u);
        __builtin_memcpy(c[i], values + (uint64_t)u * V, V);
        s[i] = scales[(row0 + row) / block_rows * pitch + (u - row * per_row.d) / kLanes];
    }
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const uint32_t u = first + i * 256u;
        if (u >= units) return;
        const uint32_t row = per_row.quotient(u);
        const int k0 = (int)(u - row * per_row.d) * V, left = K - k0;
        if (left <= 0) continue;
        T y[V];
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i][j / 4], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i][j / 4], true);
            y[j] = (T)product32(lo[0], s[i]);
            y[j + 1] = (T)product32(lo[1], s[i]);
            y[j + 2] = (T)product32(hi[0], s[i]);
            y[j + 3] = (T)product32(hi[1], s[i]);
        }
        T *out = Y + (int64_t)row * stride + k0;
        if (left >= V) {
            typename Unit<T>::Bytes v;
            __builtin_memcpy(&v, y, 16);
            if (STREAM) __builtin_nontemporal_store(v, (typename Unit<T>::Bytes *)out);
            else *(typename Unit<T>::Bytes *)out = v;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < left) out[j] = y[j];
        }
    }
}

// launch(first row, units) for pieces of at most 2^30 units, so that their numbers and the grid fit 32 bits.
template <class F> static int32_t in_pieces(int64_t rows, uint32_t per_row, F launch)
{
    const int64_t step = std::max<int64_t>(1, ((int64_t)1 << 30) / per_row);
    for (int64_t r = 0; r < rows; r += step) {
        launch(r, (uint32_t)std::min(step, rows - r) * per_row);
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
}

static dim3 grid_of(uint32_t units, bool stream)
{
    const uint32_t each = 256 * (stream ? kUnits : 1);
    return dim3((units + each - 1) / each);
}

int32_t launch_rows_to_f8(const void *X, int32_t type, int64_t stride, int64_t rows, int32_t K, uint8_t *values, float *scales, hipStream_t st)
{
    const int64_t blocks = blocks_of(K);
    const int pitch = scales_of(K);
    return with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        const uint32_t per_row = (uint32_t)(blocks * kBlock / Unit<T>::kValues);
        const bool stream = past_caches(rows * K * (int64_t)sizeof(T));
        return in_pieces(rows, per_row, [&](int64_t r, uint32_t units) {
            const ToArgs a{(const T *)X + r * stride, values + r * blocks * kBlock, scales + r * pitch, stride, make_div(per_row), units, K, pitch};
            if (stream) hipLaunchKernelGGL((f8_rows_kernel<T, true>), grid_of(units, true), dim3(256), 0, st, a);
            else hipLaunchKernelGGL((f8_rows_kernel<T, false>), grid_of(units, false), dim3(256), 0, st, a);
        });
    });
}

static int32_t launch_blocks_to_f8(const void *X, int32_t type, int64_t stride, int64_t rows, int32_t K, uint8_t *values, float *scales, hipStream_t st)
{
    const int64_t blocks = blocks_of(K), tall = (rows + kBlock - 1) / kBlock;
    const int pitch = scales_of(K);
    return with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        const bool stream = past_caches(rows * K * (int64_t)sizeof(T));
        const int64_t step = std::max<int64_t>(1, ((int64_t)1 << 23) / blocks);        // (a grid has less than 2^32 threads)
        for (int64_t b = 0; b < tall; b += step) {
            const int64_t r = b * kBlock, n = std::min(step, tall - b);
            const ToArgs a{(const T *)X + r * stride, values + r * blocks * kBlock, scales + b * pitch, stride, make_div((uint32_t)blocks), 0, K, pitch};
            const dim3 grid((unsigned)(n * blocks));
            if (stream) hipLaunchKernelGGL((f8_blocks_kernel<T, true>), grid, dim3(256), 0, st, a, rows - r, (int)blocks);
            else hipLaunchKernelGGL((f8_blocks_kernel<T, false>), grid, dim3(256), 0, st, a, rows - r, (int)blocks);
            MX_HIP_TRY(hipGetLastError());
        }
        return CL_OK;
    });
}

}  // namespace f8
}  // namespace cl

using namespace cl;
using namespace cl::f8;

static int32_t check_rows(const void *x, const void *values, const void *scales, int32_t type, int64_t stride, int64_t rows, int32_t K, int32_t block_rows)
{
    if (!known_type(type)) return fail(CL_EINVAL, "unknown element type %d", (int)type);
    if (rows < 0 || K < 1) return fail(CL_EINVAL, "bad matrix: %lld rows of %d", (long long)rows, (int)K);
    if (block_rows != 1 && block_rows != kBlock) return fail(CL_EINVAL, "blocks of %d rows: 1 or %d", (int)block_rows, kBlock);
    if (K > CL_F8_MAX_K) return fail(CL_EUNSUPPORTED, "rows of more than %d elements", (int)CL_F8_MAX_K);
    if (rows == 0) return CL_OK;
    if (!x || !values || !scales) return fail(CL_EINVAL, "null pointer");
    if (x == values || x == scales || values == scales) return fail(CL_EINVAL, "numbers, values and scales: two of them are one");
    if (rows > 1 && stride < K) return fail(CL_EINVAL, "rows of %d elements overlap at a stride of %lld", (int)K, (long long)stride);
    if (!aligned(values, 16) || !aligned(scales, 16)) return fail(CL_EINVAL, "values and scales must be 16-byte aligned");
    if (!aligned(x, type_bytes(type))) return fail(CL_EINVAL, "elements are not aligned");
    return CL_OK;
}

extern "C" int32_t cl_eight_quantize(const void *d_X, int32_t type, int64_t x_stride, int64_t rows, int32_t K, int32_t block_rows, void *d_values, float *d_scales, void *stream)
{
    if (int32_t rc = check_rows(d_X, d_values, d_scales, type, x_stride, rows, K, block_rows)) return rc;
    if (int32_t rc = (block_rows == 1 ? launch_rows_to_f8 : launch_blocks_to_f8)(d_X, type, x_stride, rows, K, (uint8_t *)d_values, d_scales, (hipStream_t)stream)) return rc;
    clear_error();
    return CL_OK;
}

extern "C" int32_t cl_eight_dequantize(const void *d_values, const float *d_scales, int64_t rows, int32_t K, int32_t block_rows, void *d_Y, int32_t type, int64_t y_stride,
                                    void *stream)
{
    if (int32_t rc = check_rows(d_Y, d_values, d_scales, type, y_stride, rows, K, block_rows)) return rc;
    const int64_t blocks = blocks_of(K);
    const int32_t rc = with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        const uint32_t per_row = (uint32_t)(blocks * kBlock / Unit<T>::kValues);
        const bool stream_it = past_caches(rows * K * (int64_t)sizeof(T));
        return in_pieces(rows, per_row, [&](int64_t r, uint32_t units) {
            auto kernel = stream_it ? f8_back_kernel<T, true> : f8_back_kernel<T, false>;
            hipLaunchKernelGGL(kernel, grid_of(units, stream_it), dim3(256), 0, (hipStream_t)stream, (const uint8_t *)d_values + r * blocks * kBlock, d_scales, r, (int)block_rows, units,
                               make_div(per_row), (int)K, (int)scales_of(K), (T *)d_Y + r * y_stride, y_stride);
        });
    });
    if (rc) return rc;
    clear_error();
    return CL_OK;
}
