// What the kernels of 8-bit matrices with a scale for each block of 128 share: the format, conversions, argument checks.
#pragma once
#include "mx/mx_common.hpp"
#include "mx/quantize_kernel.hpp"

namespace cl {
namespace f8 {

using namespace cl::mx;

constexpr int kBlock = 128;                                  // elements of a row under one scale
constexpr float kLargest = 448.0f;                           // of E4M3
constexpr float kLeastScale = 0x1p-126f;

inline int32_t blocks_of(int32_t K) { return (int32_t)CL_F8_ROW_BLOCKS((int64_t)K); }
inline int32_t scales_of(int32_t K) { return (int32_t)CL_F8_ROW_SCALES((int64_t)K); }

// The scale of a block and what its values are multiplied by, from the bits of its largest magnitude (Inf and NaN are above all finite
// ones).  Two divisions rounded to nearest, of which the reciprocal's rounding can move a value that lies within 2^-23 of a tie
// to the other side: half a step of 2^-4 more than such a value's own rounding, and a multiplication instead of a division for each
// value (a division is ten instructions, and memory leaves time for about as many).
struct Scale { float scale, inverse; };
__device__ __forceinline__ Scale scale_of(uint32_t top_bits)
{
    if (top_bits >= 0x7f800000u) return Scale{__uint_as_float(0x7fc00000u), 0.0f};
    const float top = __uint_as_float(top_bits);
    if (top < kLargest * kLeastScale) return Scale{kLeastScale, 1.0f / kLeastScale};
    return Scale{top / kLargest, kLargest / top};
}

// The largest of the lanes of a run of 16 or 32, in all of them.
template <int LANES> __device__ __forceinline__ uint32_t top_of_lanes(uint32_t top)
{
    static_assert(LANES == 16 || LANES == 32, "");
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2 of a quad
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));      // lanes 2 3 0 1
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x141, 0xF, 0xF, true));     // the other quad of eight lanes
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x140, 0xF, 0xF, true));     // the other eight of sixteen
    if (LANES == 32) top = max(top, (uint32_t)__builtin_amdgcn_ds_swizzle((int)top, 0x401F));        // lane ^ 16
    return top;
}

template <int N> __device__ __forceinline__ uint32_t top_bits(const float *x)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    return top;
}

// Four values to 8 bits each: nearest, ties to even.  (What is multiplied comes to at most 448 (1 + 2^-22), and rounds to 448.)  inverse 0: a
// block that is not finite, whose codes are zeros.
__device__ __forceinline__ uint32_t to_f8(const float *x, float inverse)
{
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inverse, x[1] * inverse, 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inverse, x[3] * inverse, c, true);
    return inverse == 0.0f ? 0u : (uint32_t)c;
}

// quantize.hip: rows of X (stride in elements) to values and scales of 128 of a row, no checks.
int32_t launch_rows_to_f8(const void *X, int32_t type, int64_t stride, int64_t rows, int32_t K, uint8_t *values, float *scales, hipStream_t st);

}  // namespace f8
}  // namespace cl
