// What the kernels of microscaled 4-bit matrices and of routed experts share: element types,
// the scaled matrix instruction, the format's constants, argument checks.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <atomic>
#include <climits>
#include <cstdint>

#include "layer.hpp"

namespace cl {
namespace mx {

#define MX_HIP_TRY(expr)                                                                      \
    do {                                                                                      \
        hipError_t e_ = (expr);                                                               \
        if (e_ != hipSuccess) return fail(CL_EHIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

using bf16_t = __bf16;
using f16_t = _Float16;

// An E8M0 scale of NaN: a block with a value that is not finite.
constexpr uint32_t kScaleNaN = 255;

// A row of K elements in whole steps of the 128-wide matrix instruction, four blocks of 32 each.
inline int32_t row_blocks(int32_t K) { return (int32_t)CL_MX_ROW_BLOCKS((int64_t)K); }

// 2^(byte - 127): a power of two, the subnormal 2^-127 for 0, NaN for 255.
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    const uint32_t bits = byte == 0 ? 0x00400000u : byte == kScaleNaN ? 0x7fc00000u : byte << 23;
    return __uint_as_float(bits);
}

// The scale byte of a block from the bits of its largest magnitude: the biased exponent less 2 (the largest code, 6, is
// 1.5 * 2^2), not below 0, so that subnormal maxima need no case of their own.  255 where the maximum is Inf or NaN, whose
// bits are above all finite ones.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits)
{
    const uint32_t e = top_bits >> 23;
    return e == 255 ? kScaleNaN : e > 2 ? e - 2 : 0;
}

// 2^(127 - byte) for a scale byte of a finite block (0 .. 252): what a value is multiplied by before it is rounded to a
// code.  (A block that is not finite has codes of zero.)
__device__ __forceinline__ float scale_inverse(uint32_t byte)
{
    return byte == kScaleNaN ? 0.0f : __uint_as_float((254u - byte) << 23);
}

// The upper half of the instruction's 256-bit operand belongs to wider formats and is not read for 4-bit ones.
__device__ __forceinline__ i32x8 widen(i32x4 a) { return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1); }

// acc += sum over 128 k of A[row][k] B[col][k], both 4-bit with a scale per 32 k.  Lane l has row (A) and column (B) l % 16
// and the 32 k of its group l / 16; byte S of its scale word is that block's.  acc[i] is row 4 (l / 16) + i, column l % 16.
template <int S> __device__ __forceinline__ f32x4 mfma_fp4(i32x4 a, i32x4 b, f32x4 acc, int scale_a, int scale_b)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widen(a), widen(b), acc, 4, 4, S, scale_a, S, scale_b);
}

// a b as a 32-bit number before anything else is done with it.  (A product that is rounded to 16 bits next may else become one instruction, a b + 0
// rounded to fp16, whose last bit can differ and which makes zeros of negative ones.)
__device__ __forceinline__ float product32(float a, float b)
{
    float r = a * b;
    asm("" : "+v"(r));
    return r;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16_t x) { return (float)x; }
__device__ __forceinline__ float to_float(f16_t x) { return (float)x; }

// Between accesses of a wavefront's lanes to what its other lanes have in LDS.  A wavefront's LDS accesses are served in order, so this
// costs nothing at run time; it keeps the compiler from exchanging them.  (A wave barrier alone is no fence for memory.)
__device__ __forceinline__ void lanes_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// N consecutive values at any element's address, with one access (gfx950 takes any alignment).
template <int N, class T> __device__ __forceinline__ void load_values(const T *p, T *v) { __builtin_memcpy(v, p, N * sizeof(T)); }
template <int N, class T> __device__ __forceinline__ void store_values(T *p, const T *v) { __builtin_memcpy(p, v, N * sizeof(T)); }

// V consecutive elements of a row, of which `left` exist.
template <int V, class T> __device__ __forceinline__ void load_unit(const T *p, int left, float *x)
{
    if (left >= V) {
        T v[V];
        load_values<V>(p, v);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = to_float(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = i < left ? to_float(p[i]) : 0.0f;
    }
}

// The codes of a lane's V values (four or eight) and the scale byte of their block, whose 32 values 32 / V neighbouring lanes have.
// The maximum is taken on the bits of the magnitudes (in order for finite values, Inf and NaN above them).  The instruction
// rounds to nearest, ties to even, and takes what is above 6 to 6; the values are scaled beforehand, which is exact but for
// those that round to zero either way.
template <int V> __device__ __forceinline__ uint32_t quantise_unit(const float *x, uint32_t &byte)
{
    static_assert(V == 4 || V == 8, "");
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2 of a quad
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));      // lanes 2 3 0 1
    if (V == 4) top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x141, 0xF, 0xF, true));     // the other quad of eight lanes
    byte = scale_byte(top);
    const float inv = scale_inverse(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0] * inv, x[1] * inv, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2] * inv, x[3] * inv, 1.0f, 1);
    if (V == 8) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4] * inv, x[5] * inv, 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6] * inv, x[7] * inv, 1.0f, 3);
    }
    return byte == kScaleNaN ? 0u : c;                       // (Inf * 0 is no code)
}

inline bool known_type(int32_t type) { return type == CL_F32 || type == CL_BF16 || type == CL_F16; }
inline size_t type_bytes(int32_t type) { return type == CL_F32 ? 4 : 2; }

// f(element of the type) for the type that a call names.
template <class F> static int32_t with_type(int32_t type, F f)
{
    switch (type) {
    case CL_F32: return f(float{});
    case CL_BF16: return f(bf16_t{});
    default: return f(f16_t{});
    }
}

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

inline size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }
inline bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Raises a kernel's limit of dynamic LDS, once per device (the attribute stays).  `seen` belongs to one kernel.
struct LdsLimit { std::atomic<bool> done[64]; };
inline int32_t allow_lds(const void *kernel, size_t bytes, LdsLimit &seen)
{
    int dev = 0;
    MX_HIP_TRY(hipGetDevice(&dev));
    const bool tracked = dev >= 0 && dev < 64;
    if (tracked && seen.done[dev].load(std::memory_order_relaxed)) return CL_OK;
    MX_HIP_TRY(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (tracked) seen.done[dev].store(true, std::memory_order_relaxed);
    return CL_OK;
}

// quantize.hip: rows of X (stride in elements) to codes and scales, no checks.
int32_t launch_quantize(const void *X, int32_t type, int64_t stride, int64_t rows, int32_t K, uint8_t *codes, uint8_t *scales, hipStream_t st);

// route.hip: what expert_lists() writes, and where in its buffer.
struct ExpertLists {
    int32_t *offsets;                // experts + 2: first pair of each expert, of the pairs without one, and the end
    int32_t *order;                  // tokens * k pairs (token * k + j), expert by expert, ascending within one
    int32_t *tile_count;             // kTileWidths: tiles of each width
    int2 *tiles[4];                  // per width: (expert << 16 | pairs, first pair) of each tile; an expert's pairs begin a tile
    int32_t *chunk_counts;           // scratch of the launches that build it
    int64_t max_tiles[4];
    size_t bytes;
};
constexpr int kTileWidths = 4;
constexpr int kTileWidth[kTileWidths] = {16, 64, 128, 256};
ExpertLists expert_lists_at(void *base, int32_t tokens, int32_t k, int32_t experts);
// Rows to quantise in the same launches.
struct QuantiseRows {
    const void *X;
    int32_t type;
    int64_t stride, rows;
    int32_t K;
    uint8_t *codes, *scales;
};
int32_t launch_expert_lists(const int32_t *experts_of, int32_t tokens, int32_t k, int32_t experts, const ExpertLists &L, const QuantiseRows *rows_or_null, hipStream_t st);

}  // namespace mx
}  // namespace cl
