// The product for very few rows of X: one launch, which quantises X itself.  Part of product.hip's translation unit, inside
// namespace cl::mx.
#pragma once

// A workgroup of up to sixteen wavefronts makes the sums of 16 F rows of matrices and a few rows of X.  It quantises those into
// LDS - every workgroup all of them, which for so few costs less than a launch of its own - while its first weights are on
// their way; then the wavefronts share out the runs of 16 blocks as in mx_rows_kernel, and their sums meet in LDS.
//
// One matrix: 16 consecutive rows of it, up to kFewColumns rows of X (blockIdx.y: which).  (Microseconds, bf16, here and in two
// launches: 4096 x 4096, one row 4.5 and 6.1, eight 7.1 and 7.2, sixteen 10.2 and 7.6; 4096 x 1024, sixteen 5.3 and 5.7, 32 6.5 and
// 6.2, 64 10.2 and 8.1; 1000 x 256, 256 rows 5.4 and 7.5; one row of 4096 x 9216 7.0 and 8.4 - 21 MB, which a large copy moves in
// 4.1.  A launch less is some 4 us of the host's time besides.)  What bounds it is waiting, for weights that eight or nine wavefronts of a compute
// unit have asked for, and the quantisation: counters show a wavefront waiting for its accesses 73 % of its time with one bf16 token of eight experts of
// 1024 x 4096, 52 % - and 32 % for its turn to issue - with one fp32 row of 4096 x 9216; vector instructions have 21 and 23 % of the cycles.
// Experts: one token (blockIdx.y), `rows_each` rows of each of its k experts' matrices, which are rows of one matrix instruction
// like any others, so that a token's weighted sum needs no second launch either.  (One token, 64 experts of 1024 x 4096, eight
// chosen, 17.8 MB: 8.4 us, in three launches 16.1; 73 tokens, 4 of 14 of 336 x 217: 8.3 and 13.8; 60, 3 of 4 of 3060 x 1697,
// whose matrices every token would read: 113 and 16.)
constexpr int kUnit = 8, kBatch = 4;                         // values that a lane quantises; how often before it asks for more
constexpr int kFewColumns = 16, kFewWaves = kRowsWaves;
constexpr size_t kFewLds = 64 << 10;

struct FewArgs {
    ProductArgs p;
    const void *X;
    int64_t x_stride;
    int K, columns;
    const int32_t *experts_of;
    const float *weights;
    int k, rows_each, x_per_pair;
    int waves;                                               // wavefronts that multiply; the others only quantise
};

__host__ __device__ inline size_t few_lds(int blocks, int columns) { return ((size_t)columns * blocks * 17 + 15) / 16 * 16; }

template <class X, class T, bool EXPERTS> __global__ __launch_bounds__(kFewWaves * 64) void mx_few_kernel(FewArgs a)
{
    constexpr int kFewF = EXPERTS ? 2 : 1;
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ float sums[kFewF * 16];
    const ProductArgs &p = a.p;
    const int waves = a.waves, wave = threadIdx.x / 64, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t token = EXPERTS ? blockIdx.y : 0, column0 = EXPERTS ? 0 : (int64_t)blockIdx.y * kFewColumns;
    const int columns = EXPERTS ? a.columns : min(kFewColumns, p.rows - (int)column0);
    const int m0 = (int)blockIdx.x * (EXPERTS ? a.rows_each : 16 * kFewF);
    uint8_t *codes = lds, *scales = lds + (size_t)a.columns * p.blocks * 16;
    f32x4 *part = (f32x4 *)(lds + few_lds(p.blocks, a.columns));         // [waves][kFewF][64]

    // the values of this thread's first units, then the weights of the wavefront's first two runs, then the other units: what is
    // asked for first arrives first
    const int per_row = p.blocks * 4, units = columns * per_row, threads = (int)blockDim.x;
    float x[kBatch][kUnit];
    auto load = [&](int u0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int u = u0 + i * threads, row = u / per_row, k0 = (u - row * per_row) * kUnit;
            if (u < units) load_unit<kUnit>((const X *)a.X + (EXPERTS ? token * (a.x_per_pair ? a.k : 1) + row : column0 + row) * a.x_stride + k0, a.K - k0, x[i]);
        }
    };
    auto quantise = [&](int u0) {                            // (a row has whole blocks: a quad's lanes stay together)
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int u = u0 + i * threads;
            if (u >= units) continue;
            uint32_t byte;
            ((uint32_t *)codes)[u] = quantise_unit<kUnit>(x[i], byte);
            if ((u & 3) == 0) scales[u >> 2] = (uint8_t)byte;
        }
    };
    load((int)threadIdx.x);

    const uint8_t *w_codes[kFewF], *w_scales[kFewF];
#pragma unroll
    for (int f = 0; f < kFewF; ++f) {
        const int q = f * 16 + r;
        int64_t row;
        if (EXPERTS) {
            const int j = min(q / a.rows_each, a.k - 1), e = a.experts_of[token * a.k + j];
            row = (int64_t)(e >= 0 && e < p.experts ? e : 0) * p.M + min(m0 + q % a.rows_each, p.M - 1);
        } else {
            row = min(m0 + q, p.M - 1);
        }
        w_codes[f] = p.w_codes + row * p.blocks * 16;
        w_scales[f] = p.w_scales + row * p.blocks;
    }
    struct Run {
        i32x4 w[kFewF][4];
        int scales[kFewF];
    };
    auto load_run = [&](Run &run, int b) {
        const bool in = b < p.blocks;                        // (four blocks are in or out together)
#pragma unroll
        for (int f = 0; f < kFewF; ++f) {
#pragma unroll
            for (int s = 0; s < 4; ++s) run.w[f][s] = in ? ((const i32x4 *)(w_codes[f] + (int64_t)b * 16))[s] : i32x4{};
            run.scales[f] = in ? *(const int *)(w_scales[f] + b) : 0;
        }
    };
    const int b0 = wave < waves ? wave * 16 + g * 4 : p.blocks + g * 4, stride = waves * 16;
    constexpr bool kTwo = !EXPERTS;                          // (two runs of two rows' fragments do not fit the registers)
    Run even, odd;
    load_run(even, b0);
    if (kTwo) load_run(odd, b0 + stride);

    quantise((int)threadIdx.x);
    for (int u = (int)threadIdx.x + kBatch * threads; u < units; u += kBatch * threads) {
        load(u);
        quantise(u);
    }
    __syncthreads();

    f32x4 acc[kFewF] = {};
    const int column = min(r, columns - 1);
    const uint8_t *xc = codes + (size_t)column * p.blocks * 16, *xs = scales + (size_t)column * p.blocks;
    auto multiply = [&](const Run &run, int b) {
        const bool in = b < p.blocks;
        i32x4 x[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] = in ? ((const i32x4 *)(xc + (size_t)b * 16))[s] : i32x4{};
        const int sx = in ? *(const int *)(xs + b) : 0;
#pragma unroll
        for (int f = 0; f < kFewF; ++f) {
            acc[f] = mfma_fp4<0>(run.w[f][0], x[0], acc[f], run.scales[f], sx);
            acc[f] = mfma_fp4<1>(run.w[f][1], x[1], acc[f], run.scales[f], sx);
            acc[f] = mfma_fp4<2>(run.w[f][2], x[2], acc[f], run.scales[f], sx);
            acc[f] = mfma_fp4<3>(run.w[f][3], x[3], acc[f], run.scales[f], sx);
        }
    };
    for (int b = b0; b - g * 4 < p.blocks; b += stride) {
        multiply(even, b);
        if (kTwo) {
            load_run(even, b + 2 * stride);
            b += stride;
            if (b - g * 4 >= p.blocks) break;
            multiply(odd, b);
            load_run(odd, b + 2 * stride);
        } else {
            load_run(even, b + stride);
        }
    }
#pragma unroll
    for (int f = 0; f < kFewF; ++f)
        if (wave < waves) part[(wave * kFewF + f) * 64 + lane] = acc[f];
    __syncthreads();
    for (int at = threadIdx.x; at < kFewF * 64; at += (int)blockDim.x) {
        const int f = at / 64, l = at & 63;
        f32x4 v = part[at];
        for (int i = 1; i < waves; ++i) v += part[i * kFewF * 64 + at];
        if (!EXPERTS) {
            if ((l & 15) < columns) store_outputs<T, false>(p, column0 + (l & 15), m0 + f * 16 + 4 * (l >> 4), v, bias_of(p, 0, m0 + f * 16 + 4 * (l >> 4)), 1.0f);
        } else {
            // every column has the token's row, or column j the row of its j-th pair
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int q = f * 16 + 4 * (l >> 4) + i;
                if ((l & 15) == (a.x_per_pair ? q / a.rows_each : 0)) sums[q] = v[i];
            }
        }
    }
    if (!EXPERTS) return;
    __syncthreads();
    // row j rows_each + i is output m0 + i of the token's j-th expert
    const int step = p.act == CL_ACT_GATED ? 2 : 1, i = (int)threadIdx.x * step, m = m0 + i;
    if (i >= a.rows_each || m + step > p.M) return;
    float total = 0.0f;
    for (int j = 0; j < a.k; ++j) {
        const int64_t pair = token * a.k + j;
        const int e = a.experts_of[pair];
        const bool routed = e >= 0 && e < p.experts;
        float v = 0.0f;
        if (routed) {
            v = sums[j * a.rows_each + i];
            if (p.bias) v += p.bias[(int64_t)e * p.M + m];
            if (p.act == CL_ACT_GATED) {
                float u = sums[j * a.rows_each + i + 1];
                if (p.bias) u += p.bias[(int64_t)e * p.M + m + 1];
                v = v / (1.0f + expf(-v)) * u;
            } else if (p.act == CL_ACT_RELU) {
                v = v < 0.0f ? 0.0f : v;
            }
        }
        if (!a.weights) ((T *)p.Y)[pair * p.out_width + m / step] = (T)v;
        else if (routed) total = fmaf(a.weights[pair], v, total);
    }
    if (a.weights) ((T *)p.Y)[token * p.out_width + m / step] = (T)total;
}
