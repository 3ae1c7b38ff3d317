// The product for few rows of X: one launch, which quantises X itself.  Part of product.hip's translation unit, inside
// namespace cl::f8.
#pragma once

// A workgroup of up to sixteen wavefronts makes 16 outputs (blockIdx.x) of up to 16 rows of X (blockIdx.y: which).  The wavefronts share out the row's blocks: a block of
// 16 rows of W - GATED: of gates and of values - is one matrix instruction; their sums meet in LDS and are added in the order of the wavefronts.  No operand of W is
// shared, so that nothing but the quantisation of X, which is done while the first weights are on their way, waits for a barrier until the end.
// X in numbers: every workgroup quantises all of its rows into LDS, which for so few costs less than a launch of its own; X in 8 bits comes from the caches.
// What bounds it are a launch and one trip to memory: one fp32 row of 4096 x 9216, 38 MB, 9.3 us with the launch, 4.1 TB/s (a large copy 5.1); 8 bf16 rows of
// 2 x 4096 x 4096 gated 10.7.
constexpr int kFewWaves = 16, kFewColumns = 16, kFewAhead = 3;
constexpr size_t kFewLds = 72 << 10;

struct F8In {};

struct FewArgs {
    ProductArgs p;
    const void *X;
    int64_t x_stride;
    Div per_row;                                             // eights of a row's values
    int K;
    int columns;                                             // most of a workgroup
    int waves;                                               // wavefronts that multiply; the others only quantise
};

// A row of X in LDS: its values, with 64 bytes behind that keep rows in different banks; the scales of all rows are behind the last.
__host__ __device__ inline size_t few_row(int blocks) { return (size_t)blocks * kBlock + 64; }
__host__ __device__ inline size_t few_lds(int blocks, int columns) { return columns * (few_row(blocks) + (size_t)(blocks + 3) / 4 * 16); }

template <class X, class T, bool GATED, bool WIDE> __global__ __launch_bounds__(kFewWaves * 64) void f8_few_kernel(FewArgs a)
{
    constexpr int F = GATED ? 2 : 1;
    constexpr bool kNumbers = !std::is_same_v<X, F8In>;
    extern __shared__ __align__(16) uint8_t lds[];
    const ProductArgs &p = a.p;
    const int waves = a.waves, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int o0 = (int)blockIdx.x * 16;
    const int64_t c0 = (int64_t)blockIdx.y * kFewColumns;
    const int columns = (int)min((int64_t)a.columns, p.rows - c0);
    const int64_t row_bytes = (int64_t)p.blocks * kBlock;
    uint8_t *codes = lds;
    float *scales = (float *)(lds + a.columns * few_row(p.blocks));
    f32x4 *sums = (f32x4 *)(lds + (kNumbers ? few_lds(p.blocks, a.columns) : 0));        // [waves][F][64]

    // the values of this thread's first units, then the weights of the wavefront's first blocks, then the other units: what is
    // asked for first arrives first
    constexpr int kBatch = 2;
    float n[kBatch][8];
    [[maybe_unused]] const int units = columns * (int)a.per_row.d, threads = (int)blockDim.x;
    [[maybe_unused]] auto load = [&](int u0) {
        if constexpr (kNumbers) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int u = u0 + i * threads, row = (int)a.per_row.quotient((uint32_t)u), k0 = (u - row * (int)a.per_row.d) * 8;
                if (u < units) load_unit<8>((const X *)a.X + (c0 + row) * a.x_stride + k0, a.K - k0, n[i]);
            }
        }
    };
    [[maybe_unused]] auto quantise = [&](int u0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int u = u0 + i * threads;
            if (u >= units) continue;                        // (a row has whole blocks: the lanes of one are beyond the end together)
            const Scale s = scale_of(top_of_lanes<16>(top_bits<8>(n[i])));
            const int row = (int)a.per_row.quotient((uint32_t)u), in = u - row * (int)a.per_row.d;
            *(u32x2 *)(codes + row * few_row(p.blocks) + in * 8) = u32x2{to_f8(n[i], s.inverse), to_f8(n[i] + 4, s.inverse)};
            if (in % 16 == 0) scales[row * p.blocks + in / 16] = s.scale;
        }
    };
    load((int)threadIdx.x);

    const uint8_t *w[F];
    const float *ws[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        w[f] = p.w + ((int64_t)f * p.width + min(o0 + r, p.width - 1)) * row_bytes + g * 16;
        ws[f] = p.w_scales + (int64_t)(f * p.value_tall + o0 / kBlock) * p.pitch_scales;
    }
    struct Block { i32x8 w[F]; float s[F]; };
    auto load_block = [&](Block &b, int at) {
        if (at >= p.blocks) return;                          // (a block too many for each wavefront costs 0.75 us)
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const uint8_t *q = w[f] + (int64_t)at * kBlock;
            b.w[f] = both(*(const i32x4 *)q, *(const i32x4 *)(q + 64));
            b.s[f] = ws[f][at];
        }
    };
    Block ring[kFewAhead];
    const bool multiplies = wave < waves;
    if (multiplies) {
#pragma unroll
        for (int i = 0; i < kFewAhead; ++i) load_block(ring[i], wave + i * waves);
    }
    const int64_t column = c0 + min(r, columns - 1);
    const uint8_t *xg = p.x + column * row_bytes + g * 16;
    const float *xsg = p.x_scales + column * p.pitch_scales;
    if constexpr (kNumbers) {
        quantise((int)threadIdx.x);
        for (int u = (int)threadIdx.x + kBatch * threads; u < units; u += kBatch * threads) {
            load(u);
            quantise(u);
        }
        __syncthreads();
    }
    f32x4 acc[F] = {};
    auto multiply = [&](const Block &b, int at) {
        const uint8_t *q = kNumbers ? codes + min(r, columns - 1) * few_row(p.blocks) + at * kBlock + g * 16 : xg + (int64_t)at * kBlock;
        const Operand<WIDE> x = operand<WIDE>(both(*(const i32x4 *)q, *(const i32x4 *)(q + 64)));
        const float sx = kNumbers ? scales[min(r, columns - 1) * p.blocks + at] : xsg[at];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const f32x4 v = mfma_f8<WIDE>(operand<WIDE>(b.w[f]), x);
            const float s = sx * b.s[f];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[f][i] = fmaf(v[i], s, acc[f][i]);
        }
    };
    if (multiplies) {
        for (int b = wave; b < p.blocks; b += kFewAhead * waves) {
#pragma unroll
            for (int i = 0; i < kFewAhead; ++i) {
                const int at = b + i * waves;
                if (at >= p.blocks) break;
                multiply(ring[i], at);
                load_block(ring[i], at + kFewAhead * waves);
            }
        }
#pragma unroll
        for (int f = 0; f < F; ++f) sums[(wave * F + f) * 64 + lane] = acc[f];
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int64_t row = c0 + r;
    if (r >= columns) return;
    f32x4 v[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        v[f] = sums[f * 64 + lane];
        for (int i = 1; i < waves; ++i) v[f] += sums[(i * F + f) * 64 + lane];
    }
    const int o = o0 + 4 * g;
    if (p.part) {
#pragma unroll
        for (int f = 0; f < F; ++f) store_part(p, 0, row, o, v[f], f * p.value_at);
    } else {
        store_outputs<T>(p, row, o, activated<T, GATED>(p, o, v[0], v[F - 1]));
    }
}
