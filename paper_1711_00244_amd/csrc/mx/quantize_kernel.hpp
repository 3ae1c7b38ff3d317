// Quantisation of rows, for the kernels that do nothing else and for one that builds lists beside.
#pragma once
#include <algorithm>
#include <type_traits>

#include "mx_common.hpp"

namespace cl {
namespace mx {

// A lane has 16 bytes of numbers at a time - a unit: four or eight, eight or four lanes to a block - so that each load and store
// of a wavefront is consecutive, and kUnits of those.  STREAM: numbers go past the caches (matrices that would not stay in
// them).  Memory bounds both: 4096 x 25088 fp32, there and back, 142 us, 931 MB at 6.5 TB/s (a large copy: 5.1).  With eight
// values a lane - two stores that each fill half of every line - and through the caches it was 223, back alone 133.
constexpr int kUnits = 2;

// (An element's alignment is enough for an access of 16 bytes.)
template <int BYTES> struct UnitOf;
template <> struct UnitOf<4> {
    static constexpr int kValues = 4;
    typedef uint16_t Codes;
    typedef uint32_t Bytes __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct UnitOf<2> {
    static constexpr int kValues = 8;
    typedef uint32_t Codes;
    typedef uint32_t Bytes __attribute__((ext_vector_type(4), aligned(2)));
};
template <class T> using Unit = UnitOf<(int)sizeof(T)>;

struct QuantiseArgs {
    const void *X;
    void *codes;
    uint8_t *scales;
    int64_t stride;
    Div per_row;
    uint32_t units;
    int K;
};

// kUnits units of each thread of workgroup `block`.
template <class T, bool STREAM>
__device__ __forceinline__ void quantise_units(uint32_t block, const QuantiseArgs &a)
{
    typedef Unit<T> U;
    constexpr int V = U::kValues, kLanes = 32 / V;
    float x[kUnits][V];
    const uint32_t first = block * (blockDim.x * kUnits) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = min(first + i * blockDim.x, a.units - 1), row = a.per_row.quotient(u);
        const int k0 = (int)(u - row * a.per_row.d) * V, left = a.K - k0;
        const T *p = (const T *)a.X + (int64_t)row * a.stride + k0;
        if (STREAM && left >= V) {
            const typename U::Bytes v = __builtin_nontemporal_load((const typename U::Bytes *)p);
            T t[V];
            __builtin_memcpy(t, &v, 16);
#pragma unroll
            for (int j = 0; j < V; ++j) x[i][j] = to_float(t[j]);
        } else {
            load_unit<V>(p, left, x[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = first + i * blockDim.x;
        uint32_t byte;
        const uint32_t c = quantise_unit<V>(x[i], byte);     // (a row has whole blocks: the lanes of one are beyond the end together)
        if (u < a.units) {
            ((typename U::Codes *)a.codes)[u] = (typename U::Codes)c;
            if (u % kLanes == 0) a.scales[u / kLanes] = (uint8_t)byte;
        }
    }
}

// Numbers go past the caches where they take more than a quarter of the last one (256 MB).
inline bool past_caches(int64_t bytes) { return bytes > (64 << 20); }

}  // namespace mx
}  // namespace cl
