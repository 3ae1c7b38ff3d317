// The product for some columns: smaller tiles of the output.  Part of product.hip's translation unit, inside namespace cl::f8.
#pragma once

// As f8_tile_kernel, one tile to a workgroup, for tiles whose steps are so short that what counts are not multiplies but how often, and for how long, wavefronts wait: for
// LDS, and for each other.  They meet once a step.  What a step multiplies has been read from LDS during the step before: a piece's rows when the registers had been used
// there, columns at its beginning, into a second set.  So nothing waits for LDS where the wavefronts meet; a buffer is asked for again one step after it was read.
//
// WIDE: columns are taken to bf16 when their step begins, and then replaced in their one set.
//
// 256 rows of X, 4096 x 9216, fp32 outputs, WIDE: 128 x 128 in four shares of k 33 us with the sum of the shares (a compute unit has one workgroup, of 18 steps), 64 x 64 in
// two 35, in three 38; 333 rows of 2 x 2900 x 1100 gated, fp16: 128 x 128 8.2 us.
template <int BM, int BN, int WM, int WN> struct SmallTile {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int TI = BM / WM / 16, TJ = BN / WN / 16;
    static constexpr int kRun = TI * 8;                      // rows under one scale: half of a wavefront's
    static constexpr int kLoads = (BM + BN) / 8 / kWaves;    // of a wavefront and step
    static constexpr int kScaleLoads = BN / 64 + 1;          // of the workgroup and four steps: columns, then the wavefronts' rows
    static constexpr int kScaleShare = (kScaleLoads + kWaves - 1) / kWaves;      // (wavefronts beyond that number repeat the last)
    static constexpr int kBuffer = (BM + BN) * kBlock, kSteps = 4;       // of a step, and how many LDS holds
    static constexpr int kScales = kSteps * kBuffer;         // where the scales start: two buffers of four steps
    static constexpr int kScaleBuffer = (BN + 64) * 16;
    static constexpr int kLds = kScales + 2 * kScaleBuffer, kTops = WM * BN * 4;
    static constexpr int share(int n, int of, int i) { return n * i / of; }
    static constexpr int kColumnPieces = TI > 2 ? TI / 2 : 1;          // pieces at whose beginning columns of the next step are read
    static_assert(TI % 2 == 0 && TI > 0 && TJ > 0 && 128 % kRun == 0, "");
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && kRun % 8 == 0 && BN % 64 == 0 && 2 * WM <= 64, "");
    static_assert((kSteps - 1) * kLoads + 2 * kScaleShare < 64, "");             // (the count that a wait names)
};

template <int BM, int BN, int WM, int WN, class T, bool GATED, bool WIDE>
__global__ __launch_bounds__(WM * WN * 64, 2) void f8_small_tile_kernel(ProductArgs a, int row_tiles)
{
    using C = SmallTile<BM, BN, WM, WN>;
    constexpr int TI = C::TI, TJ = C::TJ, kSteps = C::kSteps, kSets = WIDE ? 1 : 2;
    extern __shared__ __align__(128) uint8_t lds[];
    typedef __attribute__((address_space(3))) void *lds_ptr;
    typedef const __attribute__((address_space(1))) void *global_ptr;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)(threadIdx.x & 63), r = lane & 15, g = lane >> 4;
    constexpr int kOutputs = GATED ? BM / 2 : BM;            // of the tile

    // Workgroups go to the eight dies in turn.  Each die takes a run of tiles, four columns of tiles at a time, so that what it has in flight shares rows of W and of X in its
    // cache.
    const int columns = (a.rows + BN - 1) / BN, tiles = columns * row_tiles, die = (int)blockIdx.x % 8, nth = (int)blockIdx.x / 8;
    if (nth >= tiles / 8 + (die < tiles % 8)) return;
    const int tile = die * (tiles / 8) + min(die, tiles % 8) + nth, band = (int)a.band_tiles.quotient((uint32_t)tile) * 4;
    const int in = tile - band * row_tiles, across = min(4, columns - band), down = across == 1 ? in : across == 2 ? in / 2 : across == 3 ? in / 3 : in / 4;
    const int o0 = down * kOutputs, c0 = (band + in - down * across) * BN, count = min(BN, a.rows - c0);
    const int split = (int)blockIdx.y;
    const int t_first = 4 * (split * a.split_fours + min(split, a.split_more));
    const int steps = min(4 * (a.split_fours + (split < a.split_more)), a.blocks - t_first), last = steps - 1;

    const int wm = wave / WN, wn = wave % WN;
    const uint32_t row_bytes = (uint32_t)a.blocks * kBlock;
    // where run n of the tile's rows begins - the first output that it has, and whether it has values -, for runs of kRun rows, two to a wavefront
    auto run_output = [&](int n) { return o0 + (GATED ? n / 2 : n) * C::kRun; };
    auto run_value = [&](int n) { return GATED ? n % 2 : 0; };
    // what each load of a wavefront reads: eight rows (those beyond the last repeat it; a tile's have less than 4 GB)
    const uint8_t *base[C::kLoads];
    uint32_t offset[C::kLoads];
    const uint32_t unit = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
    for (int k = 0; k < C::kLoads; ++k) {
        const int row = (k * C::kWaves + wave) * 8;
        if (k < BM / 8 / C::kWaves) {
            const int run = row / C::kRun, o = min(run_output(run) + row % C::kRun, a.width - 1);
            base[k] = a.w + ((int64_t)run_value(run) * a.width + o) * row_bytes + (int64_t)t_first * kBlock;
            offset[k] = (uint32_t)min(lane >> 3, a.width - 1 - o) * row_bytes + unit;
        } else {
            const int n = min(row - BM, count - 1);
            base[k] = a.x + (int64_t)(c0 + n) * row_bytes + (int64_t)t_first * kBlock;
            offset[k] = (uint32_t)min(lane >> 3, count - 1 - n) * row_bytes + unit;
        }
    }
    const float *scale_at[C::kScaleShare];
#pragma unroll
    for (int k = 0; k < C::kScaleShare; ++k) {
        const int load = min(k * C::kWaves + wave, C::kScaleLoads - 1), n = load * 64 + lane;
        if (n < BN) {
            scale_at[k] = a.x_scales + (int64_t)(c0 + min(n, count - 1)) * a.pitch_scales + t_first;
        } else {
            const int run = min(n - BN, 2 * WM - 1), tall = min(run_output(run), a.width - 1) / kBlock + run_value(run) * a.value_tall;
            scale_at[k] = a.w_scales + (int64_t)tall * a.pitch_scales + t_first;
        }
    }
    auto request = [&](int t, uint8_t *buf, int k) {
        const uint8_t *at = base[k] + (uint32_t)t * kBlock;
        asm("" : "+s"(at));                                  // (the same for all lanes, and added up there: half the registers)
        __builtin_amdgcn_global_load_lds((global_ptr)(at + offset[k]), (lds_ptr)(buf + (k * C::kWaves + wave) * 1024), 16, 0, 0);
    };
    auto scales = [&](int q) { return lds + C::kScales + q % 2 * C::kScaleBuffer; };
    auto request_scales = [&](int q, uint8_t *__restrict__ buf) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < C::kScaleShare; ++k)
            __builtin_amdgcn_global_load_lds((global_ptr)(scale_at[k] + (int64_t)q * 4), (lds_ptr)(buf + min(k * C::kWaves + wave, C::kScaleLoads - 1) * 1024), 16, 0, 0);
    };

    const int wi = wm * TI * 16 + r, wj = BM + wn * TJ * 16 + r;        // the lane's rows of the buffer
    const int lo = (g ^ (r & 7)) * 16, hi = ((g + 4) ^ (r & 7)) * 16;
    auto read_piece = [&](const uint8_t *buf, int row) { return both(*(const i32x4 *)(buf + row * kBlock + lo), *(const i32x4 *)(buf + row * kBlock + hi)); };
    auto scale_of_column = [&](const uint8_t *buf, int j) { return *(const float *)(buf + (wn * TJ * 16 + j * 16 + r) * 16); };
    auto scale_of_run = [&](const uint8_t *buf, int h) { return *(const float *)(buf + (BN + wm * 2 + h) * 16); };

    f32x4 acc[TI][TJ], p[TJ];
    i32x8 w[TI], x[kSets][TJ];
    Operand<WIDE> xw[TJ];                                    // (narrow: not used)
    float sx[TJ], sw[2], by[TJ];
#pragma unroll
    for (auto &v : acc)
#pragma unroll
        for (auto &y : v) y = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < TJ; ++j) p[j] = f32x4{0, 0, 0, 0}, by[j] = 0.0f;

    auto loads_left = [](int n) constexpr { return 0xf70 | (n & 15) | (n >> 4) << 14; };     // s_waitcnt: n loads left
    auto meet = [&](auto LEFT) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        constexpr int left = loads_left(decltype(LEFT)::value);
        __builtin_amdgcn_s_waitcnt(left);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto join = [&](int i, int j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[j][e], by[j], acc[i][j][e]);
        asm volatile("" : "+v"(acc[i][j]));                  // (here, not where the sum is needed next: p would have to be kept)
    };
    // Piece row i of a step of parity P; `next` has the step after, `to` receives step `ask`, scales_next is at the word of the next step.
    auto piece = [&](auto I, auto P, const uint8_t *__restrict__ next, const uint8_t *__restrict__ scales_next, uint8_t *__restrict__ to, int ask) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value, now = WIDE ? 0 : decltype(P)::value, then = WIDE ? 0 : 1 - now;
        if (WIDE && i == 0) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) xw[j] = operand<WIDE>(x[0][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (i < C::kColumnPieces) {
#pragma unroll
            for (int j = C::share(TJ, C::kColumnPieces, i); j < C::share(TJ, C::kColumnPieces, i + 1); ++j) x[then][j] = read_piece(next, wj + j * 16);
            __builtin_amdgcn_sched_barrier(0);
        }
        const Operand<WIDE> row = operand<WIDE>(w[i]);
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            join((i + TI - 1) % TI, j);
            if constexpr (WIDE) p[j] = mfma_f8<WIDE>(row, xw[j]);
            else p[j] = mfma_f8<WIDE>(row, x[now][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        w[i] = read_piece(next, wi + i * 16);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = C::share(C::kLoads, TI, i); k < C::share(C::kLoads, TI, i + 1); ++k) request(ask, to, k);
        if (i == 0 || i == TI / 2) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) by[j] = sx[j] * sw[i == 0 ? 0 : 1];
        }
        if (i == TI / 2) {                                   // (the next step's)
#pragma unroll
            for (int j = 0; j < TJ; ++j) sx[j] = scale_of_column(scales_next, j);
            sw[0] = scale_of_run(scales_next, 0);
            sw[1] = scale_of_run(scales_next, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // (requests beyond the last step repeat it, so that a wait always counts the same; nothing uses what they bring, nor what is read of a step beyond the last)
    int to = kSteps - 1;                                     // the buffer that is asked for: that of the step before
    auto step = [&](auto P, int t) __attribute__((always_inline)) {
        // every wavefront's loads of step t + 1 have arrived - those of t + 2 may be on their way -, and what it read of step t - 1 it has multiplied
        meet(std::integral_constant<int, C::kLoads>{});
        const int ask = min(t + kSteps - 1, last);
        if ((t + kSteps - 1) % 4 == 0) request_scales(ask / 4, scales((t + kSteps - 1) / 4));
        const uint8_t *next = lds + (to + 2 < kSteps ? to + 2 : to + 2 - kSteps) * C::kBuffer, *scales_next = scales((t + 1) / 4) + (t + 1) % 4 * 4;
        each<0, TI>([&](auto I) __attribute__((always_inline)) { piece(I, P, next, scales_next, lds + to * C::kBuffer, ask); });
        to = to + 1 < kSteps ? to + 1 : 0;
    };

    request_scales(0, scales(0));
#pragma unroll
    for (int t = 0; t < kSteps - 1; ++t) {
#pragma unroll
        for (int k = 0; k < C::kLoads; ++k) request(min(t, last), lds + t * C::kBuffer, k);
    }
    meet(std::integral_constant<int, (kSteps - 2) * C::kLoads>{});
#pragma unroll
    for (int j = 0; j < TJ; ++j) x[0][j] = read_piece(lds, wj + j * 16), sx[j] = scale_of_column(scales(0), j);
    sw[0] = scale_of_run(scales(0), 0);
    sw[1] = scale_of_run(scales(0), 1);
#pragma unroll
    for (int i = 0; i < TI; ++i) w[i] = read_piece(lds, wi + i * 16);
    for (int t = 0; t < steps; t += 2) {
        step(std::integral_constant<int, 0>{}, t);
        if (t + 1 < steps) step(std::integral_constant<int, 1>{}, t + 1);
    }
#pragma unroll
    for (int j = 0; j < TJ; ++j) join(TI - 1, j);
    store_tile<TI, TJ, WM, BN, T, GATED>(a, split, o0 + wm * (GATED ? TI * 8 : TI * 16), c0, wm, wn, lane, acc, (float *)(lds + C::kLds));
    // (what is still on its way into LDS has to be there before that is another workgroup's)
    constexpr int none = loads_left(0);
    __builtin_amdgcn_s_waitcnt(none);
}
