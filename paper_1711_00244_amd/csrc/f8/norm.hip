// Root-mean-square norm of rows, with the addition of a residual before it and an 8-bit output after it.
#include "f8_common.hpp"

namespace cl {
namespace f8 {

struct NormArgs {
    const void *X, *residual, *gain;
    void *sum, *Y;
    float *scales;
    int64_t x_stride, residual_stride, sum_stride, y_stride, rows;
    int K, units, blocks, pitch;                             // units of a row; its blocks and scales (8-bit output)
    int lanes;                                               // that share a row: a power of two
    int gain_f32;
    float eps;
};

struct F8Out {};

// h = x + r, rounded to the type that the sum is stored in (so that what is normalised is what the next layer adds to); y = h / sqrt(mean h^2 + eps) gain.
// Squares are added in 32 bits: a lane's own in order, then lanes by exchanges, then wavefronts in order.
//
// `lanes` lanes have a row, 16 bytes of numbers at a time, U times - all in registers, so that a row is read once.  U = 0: rows that do not fit,
// read again for the output.  TAIL: K is no multiple of a unit (the others do without, and are up to 13 % faster for it).  STREAM: what is read and the sum go past
// the caches (matrices that would not stay in them).  Memory bounds it: 16384 rows of 4096 bf16 with sum and 8-bit output, 470 MB, 78 us, 6.0 TB/s.
template <class T, class Y, int U, bool STREAM, bool TAIL> __global__ __launch_bounds__(1024) void rms_norm_kernel(NormArgs a)
{
    constexpr int V = Unit<T>::kValues, kLanes = kBlock / V, R = U ? U : 1;
    constexpr bool kF8 = std::is_same_v<Y, F8Out>;
    typedef typename Unit<T>::Bytes Bytes;
    __shared__ float parts[16];
    const int lanes = a.lanes, lane = (int)threadIdx.x & (lanes - 1);
    const int64_t row = (int64_t)blockIdx.x * ((int)blockDim.x / lanes) + (int)threadIdx.x / lanes;
    const bool in = row < a.rows;                            // (the lanes of a row together)
    const T *x = (const T *)a.X + row * a.x_stride, *r = (const T *)a.residual + row * a.residual_stride;
    T *sum = (T *)a.sum + row * a.sum_stride;
    Bytes h[R];

    auto left_of = [&](int u) { return in ? a.K - u * V : 0; };
    // A unit of a row; of one that the row ends in (TAIL) the row's last V numbers, which settle() moves down when they are there.  (One load for all lanes: with up to
    // seven for a row's last numbers, 789041 rows of 69 bf16 with sum, 435 MB, take 183 us instead of 143.)
    auto load = [&](const T *p, int u) {
        const int left = left_of(u);
        Bytes b = {0, 0, 0, 0};
        if (!TAIL || a.K >= V) {
            const Bytes *at = (const Bytes *)(p + (TAIL ? min(u * V, a.K - V) : u * V));
            if (left > 0) b = STREAM ? __builtin_nontemporal_load(at) : *at;
        } else {
            T v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = j < left ? p[u * V + j] : (T)0.0f;
            __builtin_memcpy(&b, v, 16);
        }
        return b;
    };
    auto settle = [&](int u, Bytes &b) {
        const int left = left_of(u);
        if (TAIL && left > 0 && left < V && a.K >= V) {
            uint64_t h[2];
            __builtin_memcpy(h, &b, 16);
            const int by = (V - left) * (int)sizeof(T) * 8;
            h[0] = by < 64 ? h[0] >> by | h[1] << (64 - by) : h[1] >> (by - 64);
            h[1] = by < 64 ? h[1] >> by : 0;
            __builtin_memcpy(&b, h, 16);
        }
    };
    auto values = [&](const Bytes &b, float *f) {
        T v[V];
        __builtin_memcpy(v, &b, 16);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = to_float(v[j]);
    };
    auto store = [&](auto *p, int u, const auto *v, bool stream) {
        using S = std::remove_reference_t<decltype(*p)>;
        const int left = left_of(u);
        if (left >= (TAIL ? V : 1)) {
            typedef uint32_t Wide __attribute__((ext_vector_type(V * sizeof(S) / 4), aligned(sizeof(S))));
            Wide b;
            __builtin_memcpy(&b, v, sizeof(b));
            if (stream) __builtin_nontemporal_store(b, (Wide *)(p + u * V));
            else *(Wide *)(p + u * V) = b;
        } else if (TAIL) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < left) p[u * V + j] = v[j];
        }
    };
    auto add_residual = [&](int u, Bytes &b, const Bytes &with) {
        float f[V], g[V];
        values(b, f);
        values(with, g);
        T v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (T)(f[j] + g[j]);
        __builtin_memcpy(&b, v, 16);
        store(sum, u, v, STREAM);
    };
    float squares = 0.0f;
    auto add_squares = [&](const Bytes &b) {
        float f[V];
        values(b, f);
#pragma unroll
        for (int j = 0; j < V; ++j) squares = fmaf(f[j], f[j], squares);
    };
    if constexpr (U > 0) {
#pragma unroll
        for (int i = 0; i < U; ++i) h[i] = load(x, i * lanes + lane);
        if (a.residual) {
            Bytes w[U];
#pragma unroll
            for (int i = 0; i < U; ++i) w[i] = load(r, i * lanes + lane);
#pragma unroll
            for (int i = 0; i < U; ++i) {
                settle(i * lanes + lane, h[i]);
                settle(i * lanes + lane, w[i]);
                add_residual(i * lanes + lane, h[i], w[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) settle(i * lanes + lane, h[i]);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) add_squares(h[i]);
    } else {
        for (int u = lane; u < a.units; u += lanes) {
            h[0] = load(x, u);
            settle(u, h[0]);
            if (a.residual) {
                Bytes w = load(r, u);
                settle(u, w);
                add_residual(u, h[0], w);
            }
            add_squares(h[0]);
        }
    }
    for (int o = 1; o < min(lanes, 64); o *= 2) squares += __shfl_xor(squares, o);
    if (lanes > 64) {
        if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64] = squares;
        __syncthreads();
        const int first = (int)threadIdx.x / lanes * (lanes / 64);
        squares = parts[first];
        for (int i = 1; i < lanes / 64; ++i) squares += parts[first + i];
    }
    const float by = 1.0f / sqrtf(squares / (float)a.K + a.eps);

    auto finish = [&](int u, const Bytes &b) {
        if (u >= a.units) return;                            // (the lanes of a block together)
        const int left = left_of(u);
        float y[V];
        values(b, y);
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] *= by;
        if (a.gain) {
            float gain[V];
            if (a.gain_f32) load_unit<V>((const float *)a.gain + u * V, left, gain);
            else load_unit<V>((const T *)a.gain + u * V, left, gain);
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] *= gain[j];
        }
        if constexpr (kF8) {
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = j < left ? y[j] : 0.0f;           // (beyond the row's end, in a row that is not finite)
            const Scale s = scale_of(top_of_lanes<kLanes>(top_bits<V>(y)));
            if (!in) return;
            uint8_t *at = (uint8_t *)a.Y + (row * a.blocks * kLanes + u) * V;
            if constexpr (V == 4) *(uint32_t *)at = to_f8(y, s.inverse);
            else *(u32x2 *)at = u32x2{to_f8(y, s.inverse), to_f8(y + 4, s.inverse)};
            if (u % kLanes == 0) {
                float *to = a.scales + row * a.pitch;
                const int b = u / kLanes;
                to[b] = s.scale;
                if (b == a.blocks - 1)
                    for (int i = a.blocks; i < a.pitch; ++i) to[i] = 0.0f;
            }
        } else {
            Y out[V];
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = (Y)product32(y[j], 1.0f);
            store((Y *)a.Y + row * a.y_stride, u, out, false);
        }
    };
    if constexpr (U > 0) {
#pragma unroll
        for (int i = 0; i < U; ++i) finish(i * lanes + lane, h[i]);
    } else {
        const T *from = a.residual ? sum : x;
        for (int u = lane; u < a.units; u += lanes) {
            h[0] = load(from, u);
            settle(u, h[0]);
            finish(u, h[0]);
        }
    }
}

template <class T, class Y> static int32_t launch_norm(NormArgs a, hipStream_t st)
{
    constexpr int V = Unit<T>::kValues;
    a.units = std::is_same_v<Y, F8Out> ? a.blocks * (kBlock / V) : (a.K + V - 1) / V;
    // many rows: a lane has 64 bytes or 16 (16384 rows of 4096 bf16 with sum and 8-bit output, 4 times 77 us, 2 times 81, 8 times 82, once 94; 65536 of 1024 76, once
    // 91); few: as many lanes as there is work for (512 rows of 4096 5.3, four times 6.5; one row 3.4 and 6.9).  Lanes and times, which are the order that squares are added in,
    // go by the units of whole blocks, a block's at the least, whatever the output's type: so 8 bits are those of the fp32 result.
    const int whole = a.blocks * (kBlock / V), want = a.rows >= (1 << 20) / whole ? 4 : 1;
    int times = 1;
    a.lanes = kBlock / V;
    while (a.lanes < 1024 && a.lanes * want < whole) a.lanes *= 2;
    while (times <= 8 && a.lanes * times < whole) times *= 2;
    const int threads = std::max(256, a.lanes), each = threads / a.lanes;
    const int64_t step = (int64_t)(UINT32_MAX / threads) * each, all = a.rows;
    for (int64_t r = 0; r < all; r += step) {
        NormArgs p = a;
        p.rows = std::min(step, all - r);
        p.X = (const T *)a.X + r * a.x_stride;
        p.residual = a.residual ? (const T *)a.residual + r * a.residual_stride : nullptr;
        p.sum = a.sum ? (T *)a.sum + r * a.sum_stride : nullptr;
        if constexpr (std::is_same_v<Y, F8Out>) p.Y = (uint8_t *)a.Y + r * a.blocks * kBlock;
        else p.Y = (Y *)a.Y + r * a.y_stride;
        p.scales = a.scales + r * a.pitch;
        const dim3 grid((unsigned)((p.rows + each - 1) / each)), block((unsigned)threads);
        auto launch = [&](auto stream, auto tail) {
            switch (times) {
            case 1: hipLaunchKernelGGL((rms_norm_kernel<T, Y, 1, stream.value, tail.value>), grid, block, 0, st, p); break;
            case 2: hipLaunchKernelGGL((rms_norm_kernel<T, Y, 2, stream.value, tail.value>), grid, block, 0, st, p); break;
            case 4: hipLaunchKernelGGL((rms_norm_kernel<T, Y, 4, stream.value, tail.value>), grid, block, 0, st, p); break;
            case 8: hipLaunchKernelGGL((rms_norm_kernel<T, Y, 8, stream.value, tail.value>), grid, block, 0, st, p); break;
            default: hipLaunchKernelGGL((rms_norm_kernel<T, Y, 0, false, tail.value>), grid, block, 0, st, p); break;
            }
        };
        const bool stream = past_caches(all * a.K * (int64_t)sizeof(T));
        if (a.K % V) stream ? launch(std::true_type{}, std::true_type{}) : launch(std::false_type{}, std::true_type{});
        else stream ? launch(std::true_type{}, std::false_type{}) : launch(std::false_type{}, std::false_type{});
        MX_HIP_TRY(hipGetLastError());
    }
    return CL_OK;
}

}  // namespace f8
}  // namespace cl

using namespace cl;
using namespace cl::f8;

static int32_t check_operand(const char *name, const void *p, int32_t type, int64_t stride, int64_t rows, int32_t K)
{
    if (!p) return fail(CL_EINVAL, "null pointer: %s", name);
    if (rows > 1 && stride < K) return fail(CL_EINVAL, "%s: rows of %d elements overlap at a stride of %lld", name, (int)K, (long long)stride);
    if (!aligned(p, type_bytes(type))) return fail(CL_EINVAL, "%s: elements are not aligned", name);
    return CL_OK;
}

// What is written over what is read has to have its elements where those are.
static int32_t check_in_place(const char *name, const void *to, int32_t to_type, int64_t to_stride, const void *from, const cl_norm_call &c, int64_t from_stride)
{
    if (to == from && (to_type != c.type || (c.rows > 1 && to_stride != from_stride))) return fail(CL_EINVAL, "%s: in place, but of another type or stride", name);
    return CL_OK;
}

extern "C" int32_t cl_rms_norm(const cl_norm_call *call, void *stream)
{
    if (!call) return fail(CL_EINVAL, "null pointer");
    const cl_norm_call &c = *call;
    if (!known_type(c.type)) return fail(CL_EINVAL, "unknown element type %d", (int)c.type);
    if (!known_type(c.y_type) && c.y_type != CL_F8) return fail(CL_EINVAL, "unknown element type %d", (int)c.y_type);
    if (c.rows < 0 || c.K < 1) return fail(CL_EINVAL, "bad matrix: %lld rows of %d", (long long)c.rows, (int)c.K);
    if (c.K > CL_F8_MAX_K) return fail(CL_EUNSUPPORTED, "rows of more than %d elements", (int)CL_F8_MAX_K);
    if (!(c.eps >= 0.0f) || c.eps > 3.0e38f) return fail(CL_EINVAL, "eps must be a finite number of at least 0");
    if (c.rows == 0) return CL_OK;
    if (int32_t rc = check_operand("X", c.d_X, c.type, c.x_stride, c.rows, c.K)) return rc;
    if (c.d_residual) {
        if (int32_t rc = check_operand("residual", c.d_residual, c.type, c.residual_stride, c.rows, c.K)) return rc;
        if (int32_t rc = check_operand("sum", c.d_sum, c.type, c.sum_stride, c.rows, c.K)) return rc;
        if (c.d_sum == c.d_Y) return fail(CL_EINVAL, "the sum and the output are one");
        if (int32_t rc = check_in_place("sum", c.d_sum, c.type, c.sum_stride, c.d_X, c, c.x_stride)) return rc;
        if (int32_t rc = check_in_place("sum", c.d_sum, c.type, c.sum_stride, c.d_residual, c, c.residual_stride)) return rc;
        if (int32_t rc = check_in_place("Y", c.d_Y, c.y_type, c.y_stride, c.d_residual, c, c.residual_stride)) return rc;
    }
    if (int32_t rc = check_in_place("Y", c.d_Y, c.y_type, c.y_stride, c.d_X, c, c.x_stride)) return rc;
    if (c.d_gain) {
        if (c.gain_type != CL_F32 && c.gain_type != c.type) return fail(CL_EINVAL, "a gain is of type CL_F32 or of X's own, got %d", (int)c.gain_type);
        if (!aligned(c.d_gain, type_bytes(c.gain_type))) return fail(CL_EINVAL, "gain: elements are not aligned");
    }
    if (c.y_type == CL_F8) {
        if (!c.d_Y || !c.d_y_scales) return fail(CL_EINVAL, "null pointer");
        if (!aligned(c.d_Y, 16) || !aligned(c.d_y_scales, 16)) return fail(CL_EINVAL, "values and scales must be 16-byte aligned");
    } else if (int32_t rc = check_operand("Y", c.d_Y, c.y_type, c.y_stride, c.rows, c.K)) {
        return rc;
    }
    const NormArgs a{c.d_X, c.d_residual, c.d_gain, c.d_sum, c.d_Y, c.d_y_scales, c.x_stride, c.residual_stride, c.sum_stride, c.y_stride, c.rows,
                     c.K, 0, blocks_of(c.K), scales_of(c.K), 0, c.gain_type == CL_F32, c.eps};
    const int32_t rc = with_type(c.type, [&](auto t) -> int32_t {
        using T = decltype(t);
        if (c.y_type == CL_F8) return launch_norm<T, F8Out>(a, (hipStream_t)stream);
        return with_type(c.y_type, [&](auto y) -> int32_t { return launch_norm<T, decltype(y)>(a, (hipStream_t)stream); });
    });
    if (rc) return rc;
    clear_error();
    return CL_OK;
}
