// The product for many columns: tiles of the output, operands through LDS.  Part of product.hip's translation unit, inside
// namespace cl::f8.
#pragma once

// A workgroup of WM x WN wavefronts makes BM rows of W of BN columns (rows of X), a wavefront TI x TJ pieces of 16 x 16.  GATED: half of a wavefront's rows are
// gates, the other half their values, so that a lane has both of an output.  A step is one block of 128 k.
//
// LDS holds D steps.  The loads themselves write it.  A wavefront's rows go through registers R pieces at a time, its columns, which a whole step uses, stay
// there.  When it has read the step's last rows, R pieces before the step ends, it waits for the next step's loads and for the other wavefronts: from there on the next step
// may be read, and the buffer of this one is asked for again; what is left of the step's multiplies hides both.  Columns are replaced one by one behind their last
// use.  A piece's sum (it starts at zero in each step) is multiplied by the scales when its register is needed for the piece after it.
//
// In LDS a row's eight units of 16 bytes are 128 consecutive bytes, unit c of row r in place c ^ (r % 8).  A read of 16 bytes a lane is served sixteen lanes at a time,
// of which eight are from one half of a half-wave and eight from the other's; those have units of either parity, and touch each of the 64 banks once.
template <int BM, int BN, int WM, int WN, int D> struct Tile {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int TI = BM / WM / 16, TJ = BN / WN / 16, R = 2;
    static constexpr int kRun = TI * 8;                      // rows under one scale: half of a wavefront's
    static constexpr int kLoads = (BM + BN) / 8 / kWaves;    // of a wavefront and step
    static constexpr int kScaleLoads = BN / 64 + 1;          // of the workgroup and four steps: columns, then the wavefronts' rows
    static constexpr int kScaleShare = (kScaleLoads + kWaves - 1) / kWaves;      // (wavefronts beyond that number repeat the last)
    static constexpr int kBuffer = (BM + BN) * kBlock;
    static constexpr int kScales = D * kBuffer;              // where the scales start: two buffers of four steps
    static constexpr int kScaleBuffer = (BN + 64) * 16;
    static constexpr int kLds = kScales + 2 * kScaleBuffer;
    static_assert(TI % R == 0 && TI % 2 == 0 && TI > 0 && TJ > 0 && 128 % kRun == 0, "");
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && kRun % 8 == 0 && BN % 64 == 0 && 2 * WM <= 64, "");
    static_assert(D >= 2 && D <= 4 && 4 % D == 0, "");
    // loads of a wavefront that may be on their way when step t + 1 has to be there, t % 4 = s: those of the steps t + 2 .. t + D - 1
    static constexpr int on_their_way(int s)
    {
        int n = 0;
        for (int j = s + 2; j <= s + D - 1; ++j) n += kLoads + (j % 4 == 0 ? kScaleShare : 0);
        return n;
    }
    static_assert((D - 2) * kLoads + kScaleShare < 64, "");  // (the count that a wait names)
};

// f(I), ..., f(N - 1), numbers that are known when it is compiled.
template <int I, int N, class F> __device__ __forceinline__ void each(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<I + 1, N>(f);
    }
}

template <int BM, int BN, int WM, int WN, int D, class T, bool GATED, bool WIDE>
__global__ __launch_bounds__(WM * WN * 64, 2) void f8_tile_kernel(ProductArgs a, int row_tiles)
{
    using C = Tile<BM, BN, WM, WN, D>;
    constexpr int TI = C::TI, TJ = C::TJ, R = C::R;
    extern __shared__ __align__(128) uint8_t lds[];
    typedef __attribute__((address_space(3))) void *lds_ptr;
    typedef const __attribute__((address_space(1))) void *global_ptr;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)(threadIdx.x & 63), r = lane & 15, g = lane >> 4;
    constexpr int kOutputs = GATED ? BM / 2 : BM;            // of the tile

    // Workgroups go to the eight dies in turn.  Each die takes a run of tiles, of large ones four columns of tiles at a time, so that what it has in flight shares rows
    // of W and of X in its cache.
    int column, o0;
    const int columns = (a.rows + BN - 1) / BN, tiles = columns * row_tiles;
    if (BM * BN >= 128 * 128) {
        const int per = tiles / 8, more = tiles % 8, die = (int)blockIdx.x % 8, i = (int)blockIdx.x / 8;
        if (i >= per + (die < more)) return;
        const int tile = die * per + min(die, more) + i;
        const int first = (int)a.band_tiles.quotient((uint32_t)tile) * 4, in = tile - first * row_tiles, across = min(4, columns - first);
        const int down = across == 1 ? in : across == 2 ? in / 2 : across == 3 ? in / 3 : in / 4;
        column = first + in - down * across;
        o0 = down * kOutputs;
    } else {
        if ((int)blockIdx.x >= tiles) return;
        column = (int)a.row_tiles.quotient(blockIdx.x);
        o0 = ((int)blockIdx.x - column * row_tiles) * kOutputs;
    }
    const int c0 = column * BN, count = min(BN, a.rows - c0);
    const int split = (int)blockIdx.y;
    const int t_first = 4 * (split * a.split_fours + min(split, a.split_more));
    const int steps = min(4 * (a.split_fours + (split < a.split_more)), a.blocks - t_first), last = steps - 1;

    const int wm = wave / WN, wn = wave % WN;
    const uint32_t row_bytes = (uint32_t)a.blocks * kBlock;
    // Where run n of a tile's rows begins - the first output that it has, and whether it has values -, for runs of kRun rows, two to a wavefront's.
    auto run_output = [&](int n) { return o0 + (GATED ? n / 2 : n) * C::kRun; };
    auto run_value = [&](int n) { return GATED ? n % 2 : 0; };

    // What each load of a wavefront reads: eight rows.  (Rows beyond the last repeat it; a tile's have less than 4 GB.)
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
        __builtin_amdgcn_global_load_lds((global_ptr)(base[k] + (uint32_t)t * kBlock + offset[k]), (lds_ptr)(buf + (k * C::kWaves + wave) * 1024), 16, 0, 0);
    };
    auto request_scales = [&](int q, uint8_t *buf, int k) {
        __builtin_amdgcn_global_load_lds((global_ptr)(scale_at[k] + (int64_t)q * 4), (lds_ptr)(buf + min(k * C::kWaves + wave, C::kScaleLoads - 1) * 1024), 16, 0, 0);
    };

    const bool idle = wn * TJ * 16 >= count;                 // no columns: the wavefront loads, and multiplies nothing
    const int wi = wm * TI * 16 + r, wj = BM + wn * TJ * 16 + r;        // the lane's rows of the buffer
    const int lo = (g ^ (r & 7)) * 16, hi = ((g + 4) ^ (r & 7)) * 16;
    auto read_piece = [&](const uint8_t *buf, int row) { return both(*(const i32x4 *)(buf + row * kBlock + lo), *(const i32x4 *)(buf + row * kBlock + hi)); };
    auto scale_of_column = [&](const uint8_t *buf, int s, int j) { return *(const float *)(buf + (wn * TJ * 16 + j * 16 + r) * 16 + s * 4); };
    auto scale_of_run = [&](const uint8_t *buf, int s, int h) { return *(const float *)(buf + (BN + wm * 2 + h) * 16 + s * 4); };

    f32x4 acc[TI][TJ], p[TJ];
#pragma unroll
    for (auto &x : acc)
#pragma unroll
        for (auto &y : x) y = f32x4{0, 0, 0, 0};
#pragma unroll
    for (auto &x : p) x = f32x4{0, 0, 0, 0};
    Operand<WIDE> x[TJ];
    i32x8 w[R];
    float sx[TJ], sw[2], by[TJ];
#pragma unroll
    for (auto &s : by) s = 0.0f;

    constexpr int kWaitLds = 0xc07f;                         // s_waitcnt: no LDS access left
    auto loads_left = [](int n) constexpr { return 0xf70 | (n & 15) | (n >> 4) << 14; };     // n loads left
    auto barrier = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto join = [&](int i, int j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[j][e], by[j], acc[i][j][e]);
    };
    // Piece row i of a step.  What is read behind it, into the registers that it leaves: rows from `rows`, and, of the last one, columns from `cols`.
    auto piece = [&](auto I, auto S, const uint8_t *__restrict__ rows, const uint8_t *__restrict__ cols, const uint8_t *__restrict__ scales) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value, s = decltype(S)::value;
        const Operand<WIDE> wi_ = operand<WIDE>(w[i % R]);
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            join((i + TI - 1) % TI, j);
            p[j] = mfma_f8<WIDE>(wi_, x[j]);
            __builtin_amdgcn_sched_barrier(0);
            if (i == TI - 1) {
                x[j] = operand<WIDE>(read_piece(cols, wj + j * 16));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        w[i % R] = read_piece(rows, wi + (i + R) % TI * 16);
        if (i == 0 || i == TI / 2) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) by[j] = sx[j] * sw[i == 0 ? 0 : 1];
        }
        if (i == TI - 1) {                                   // (the next step's)
#pragma unroll
            for (int j = 0; j < TJ; ++j) sx[j] = scale_of_column(scales, (s + 1) % 4, j);
            sw[0] = scale_of_run(scales, (s + 1) % 4, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Step t, t % 4 = S: `now` has it, `next` the one after, `to` (the same as now) receives step `ask`.
    auto step = [&](auto S, const uint8_t *now, const uint8_t *next, const uint8_t *scales, const uint8_t *scales_next, uint8_t *to, uint8_t *scales_to, int ask, int ask_scales)
                    __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value;
        auto first = [&](const uint8_t *__restrict__ now, const uint8_t *__restrict__ scales) __attribute__((always_inline)) {
            sw[1] = scale_of_run(scales, s, 1);
            each<0, TI - R>([&](auto I) __attribute__((always_inline)) { piece(I, S, now, now, scales); });
        };
        auto second = [&](const uint8_t *__restrict__ next, const uint8_t *__restrict__ scales_next, uint8_t *__restrict__ to, uint8_t *__restrict__ scales_to) __attribute__((always_inline)) {
            if ((s + D) % 4 == 0) {
#pragma unroll
                for (int k = 0; k < C::kScaleShare; ++k) request_scales(ask_scales, scales_to, k);
            }
#pragma unroll
            for (int k = 0; k < C::kLoads; ++k) request(ask, to, k);
            if (idle) return;
            __builtin_amdgcn_sched_barrier(0);
            each<TI - R, TI>([&](auto I) __attribute__((always_inline)) { piece(I, S, next, next, scales_next); });
        };
        if (!idle) first(now, scales);
        // every wavefront's loads of step t + 1 have arrived, and all reads of this step's buffer are done
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        constexpr int left = loads_left(C::on_their_way(s));
        __builtin_amdgcn_s_waitcnt(left);
        barrier();
        second(next, scales_next, to, scales_to);
    };

    auto buffer = [&](int t) { return lds + t % D * C::kBuffer; };
    auto scales = [&](int q) { return lds + C::kScales + q % 2 * C::kScaleBuffer; };
    // (requests beyond the last step repeat it, so that a wait always counts the same; nothing uses what they bring)
#pragma unroll
    for (int k = 0; k < C::kScaleShare; ++k) request_scales(0, scales(0), k);
#pragma unroll
    for (int t = 0; t < D; ++t) {
        if (t > 0 && t % 4 == 0) {
#pragma unroll
            for (int k = 0; k < C::kScaleShare; ++k) request_scales(min(t, last) / 4, scales(t / 4), k);
        }
#pragma unroll
        for (int k = 0; k < C::kLoads; ++k) request(min(t, last), buffer(t), k);
    }
    constexpr int all_but_first = loads_left((D - 1) * C::kLoads);
    __builtin_amdgcn_s_waitcnt(all_but_first);
    barrier();
    if (!idle) {
#pragma unroll
        for (int j = 0; j < TJ; ++j) x[j] = operand<WIDE>(read_piece(lds, wj + j * 16)), sx[j] = scale_of_column(scales(0), 0, j);
        sw[0] = scale_of_run(scales(0), 0, 0);
#pragma unroll
        for (int i = 0; i < R; ++i) w[i] = read_piece(lds, wi + i * 16);
    }
    auto at = [&](auto S, int q) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value;
        const int t = 4 * q + s, ask = min(t + D, last);
        step(S, lds + s % D * C::kBuffer, lds + (s + 1) % D * C::kBuffer, scales(q), scales(q + (s + 1) / 4), lds + s % D * C::kBuffer, scales(q + 1), ask, ask / 4);
    };
    int q = 0;
    for (; 4 * q + 4 <= steps; ++q) {
        at(std::integral_constant<int, 0>{}, q);
        at(std::integral_constant<int, 1>{}, q);
        at(std::integral_constant<int, 2>{}, q);
        at(std::integral_constant<int, 3>{}, q);
    }
    if (4 * q < steps) at(std::integral_constant<int, 0>{}, q);
    if (4 * q + 1 < steps) at(std::integral_constant<int, 1>{}, q);
    if (4 * q + 2 < steps) at(std::integral_constant<int, 2>{}, q);
#pragma unroll
    for (int j = 0; j < TJ; ++j) join(TI - 1, j);
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    constexpr int none = loads_left(0);
    __builtin_amdgcn_s_waitcnt(none);
    barrier();
    if (idle) return;

    // A wavefront's outputs go through LDS, sixteen columns at a time, so that what it stores of a row of Y is consecutive.
    constexpr int kWide = GATED ? TI * 8 : TI * 16, kPitch = kWide + 4, kLanes = kWide / 4;
    static_assert(C::kWaves * 16 * kPitch * 4 <= C::kLds && 64 % kLanes == 0, "");
    float *mine = (float *)lds + wave * 16 * kPitch;
    const int first = o0 + wm * kWide, o = first + lane % kLanes * 4;
#pragma unroll
    for (int j = 0; j < TJ; ++j) {
        // (parts of a gated product: gates, then values)
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
            if (GATED && h == 1 && !a.part) break;
            lanes_exchange();
#pragma unroll
            for (int i = 0; i < kWide / 16; ++i) {
                f32x4 v = acc[h * (TI / 2) + i][j];
                if (!a.part) v = activated<GATED>(a, first + i * 16 + 4 * g, v, acc[GATED ? TI / 2 + i : i][j]);
                *(f32x4 *)(mine + r * kPitch + i * 16 + 4 * g) = v;
            }
            lanes_exchange();
            for (int n = lane / kLanes; n < 16; n += 64 / kLanes) {
                const int c = wn * TJ * 16 + j * 16 + n;
                if (c >= count) continue;
                const f32x4 v = *(const f32x4 *)(mine + n * kPitch + lane % kLanes * 4);
                if (a.part) store_part(a, split, c0 + c, o, v, h * a.value_at);
                else store_outputs<T>(a, c0 + c, o, v);
            }
        }
    }
}
