// The product for many columns: tiles of the output, operands through LDS.  Part of product.hip's translation unit, inside
// namespace cl::f8.
#pragma once

// A workgroup of WM x WN wavefronts makes BM rows of W of BN columns (rows of X), a wavefront TI x TJ pieces of 16 x 16.  GATED: half of a wavefront's rows are
// gates, the other half their values, so that a lane has both of an output.  A step is one block of 128 k.
//
// LDS holds two steps.  The loads themselves write it.  A wavefront's rows go through registers R pieces at a time, its columns, which a whole step uses, stay
// there, replaced one by one behind their last use.  A piece's sum (it starts at zero in each step) is multiplied by the scales when its register is needed for the piece
// after it.
//
// What bounds it are loads: all workgroups of a die want the same lines at about the same time, and wait for the first of them to come from beyond its cache.  So a
// buffer is asked for again in two parts, each as soon as it has been read: the columns and each wavefront's first half of rows halfway through the step, the
// second halves at its end; and either part is waited for when it is to be read, one and a half steps (of two) later.  At both points the wavefronts wait for each
// other.  (4096 x 4096 x 25088, 256 x 256: without loads 222 us; all of a buffer asked for at once behind the step 343, in four bunches 336; 2.5 PFLOP/s, where
// the library's product with one scale to a matrix comes to 2.76, and the card's power holds its clock at 1.9 GHz.)
// WIDE, 256 x 128 (the columns in bf16, and a 256 x 256 tile's sums beside them, do not fit the registers): 4096 x 2 x 9216 x 4096 gated with 8-bit outputs 531-550 us, 1.12-1.16
// PFLOP/s, matrix units busy 48 % of the time and vector units, which take operands to bf16, multiply by scales and make the gates, 45 % (at 2.4 GHz); when it took 540, without loads 523,
// without taking operands to bf16 500.  4096 x 4096 x 9216, fp32 outputs: 278 us, 1.11 PFLOP/s, 46 % and 39 %.
//
// In LDS a row's eight units of 16 bytes are 128 consecutive bytes, unit c of row r in place c ^ (r % 8).  A read of 16 bytes a lane is served sixteen lanes at a time,
// of which eight are from one half of a half-wave and eight from the other's; those have units of either parity, and touch each of the 64 banks once.
template <int BM, int BN, int WM, int WN> struct Tile {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int TI = BM / WM / 16, TJ = BN / WN / 16, R = 2;
    static constexpr int kRun = TI * 8;                      // rows under one scale: half of a wavefront's
    static constexpr int kLoads = (BM + BN) / 8 / kWaves;    // of a wavefront and step
    static constexpr int kLate = BM / 16 / kWaves, kEarly = kLoads - kLate;       // second halves of rows; all others
    // Where the wavefronts wait for each other: before piece row kFree the second halves have to be there, and what is early may be asked for again; before kNext
    // the next step's early part has to be there, and the second halves may be asked for again.
    static constexpr int kNext = TI - R, kFree = TI / 2 - R;
    // loads behind piece row i: the early ones from early(i) to early(i + 1), the late ones likewise
    static constexpr int share(int n, int of, int i) { return n * (i < 0 ? 0 : i < of ? i : of) / of; }
    static constexpr int early(int i) { return share(kEarly, TI / 2, i - kFree); }
    static constexpr int late(int i) { return share(kLate, R, i - kNext); }
    static constexpr int kScaleLoads = BN / 64 + 1;          // of the workgroup and four steps: columns, then the wavefronts' rows
    static constexpr int kScaleShare = (kScaleLoads + kWaves - 1) / kWaves;      // (wavefronts beyond that number repeat the last)
    static constexpr int kBuffer = (BM + BN) * kBlock, kSteps = 2;       // of a step, and how many LDS holds
    static constexpr int kScales = kSteps * kBuffer;         // where the scales start: as many buffers of four steps
    static constexpr int kScaleBuffer = (BN + 64) * 16;
    static constexpr int kLds = kScales + kSteps * kScaleBuffer, kTops = WM * BN * 4;     // (8-bit outputs: the largest of each column, of each wavefront)
    static_assert(TI % (2 * R) == 0 && TI > 0 && TJ > 0 && 128 % kRun == 0, "");
    static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && kRun % 8 == 0 && BN % 64 == 0 && 2 * WM <= 64, "");
    static_assert(BM / 16 % kWaves == 0, "");
    // Loads of a wavefront that may be on their way, at the least those asked for after the next step's early part, or after this one's second halves.  (Those of scales
    // not counted: there may be one or two more.)
    static constexpr int kInFlight = (kSteps - 1) * kLoads;
    static_assert(kInFlight + kLate < 64, "");             // (the count that a wait names)
};

// f(I), ..., f(N - 1), numbers that are known when it is compiled.
template <int I, int N, class F> __device__ __forceinline__ void each(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<I + 1, N>(f);
    }
}

// Sixteen 16-bit outputs of a lane's column, of two neighbouring pieces, so that a lane has eight consecutive ones: even sixteens of lanes of the first piece, odd ones of the
// second; lo, hi: four outputs of each as they come from the matrix instructions.
__device__ __forceinline__ u32x4 eight_outputs(u32x2 first, u32x2 second)
{
    const auto a = __builtin_amdgcn_permlane16_swap(first[0], second[0], false, false), b = __builtin_amdgcn_permlane16_swap(first[1], second[1], false, false);
    return u32x4{(uint32_t)a[0], (uint32_t)b[0], (uint32_t)a[1], (uint32_t)b[1]};
}

// The same for 8-bit outputs.
__device__ __forceinline__ u32x2 eight_outputs(uint32_t first, uint32_t second)
{
    const auto a = __builtin_amdgcn_permlane16_swap(first, second, false, false);
    return u32x2{(uint32_t)a[0], (uint32_t)a[1]};
}

// And of four pieces, so that a lane has sixteen consecutive ones, lanes of sixteen n those of piece n.
__device__ __forceinline__ u32x4 sixteen_outputs(const uint32_t *q)
{
    const auto a = __builtin_amdgcn_permlane16_swap(q[0], q[1], false, false), b = __builtin_amdgcn_permlane16_swap(q[2], q[3], false, false);
    const auto c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
    return u32x4{(uint32_t)c[0], (uint32_t)d[0], (uint32_t)c[1], (uint32_t)d[1]};
}

// What a wavefront has of a tile - outputs from `first` on, columns of X from c0 - to memory, straight from the registers: of a row it stores 64 consecutive bytes at a time, and
// loads that are on their way into LDS need not be waited for.  tops: room for WM BN numbers, [wm][column] (8-bit outputs).
template <int TI, int TJ, int WM, int BN, class T, bool GATED>
__device__ __forceinline__ void store_tile(const ProductArgs &a, int split, int first, int c0, int wm, int wn, int lane, f32x4 (&acc)[TI][TJ], float *tops)
{
    constexpr int kWide = GATED ? TI * 8 : TI * 16, kPieces = kWide / 16;
    const int r = lane & 15, g = lane >> 4, c_first = c0 + wn * TJ * 16 + r;
    if (a.part) {
#pragma unroll
        for (int i = 0; i < TI; ++i) {
            const int h = GATED && i >= kPieces, o = first + (i - h * kPieces) * 16 + 4 * g;
#pragma unroll
            for (int j = 0; j < TJ; ++j)
                if (c_first + j * 16 < a.rows) store_part(a, split, c_first + j * 16, o, acc[i][j], h * a.value_at);
        }
    } else if constexpr (std::is_same_v<T, F8Out>) {
        // A block of 128 outputs belongs to kShare wavefronts that have the same columns.
        constexpr int kShare = kBlock / kWide;
        static_assert(kWide * kShare == kBlock && kShare > 1 && WM % kShare == 0, "");
        uint32_t top[TJ];
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int o = first + i * 16 + 4 * g;
                f32x4 v = activated<T, GATED>(a, o, acc[i][j], acc[GATED ? kPieces + i : i][j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = o + e < a.width ? v[e] : 0.0f;
                    top[j] = max(top[j], __float_as_uint(v[e]) & 0x7fffffffu);
                }
                acc[i][j] = v;
            }
            top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 16));
            top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 32));
            if (g == 0) tops[wm * BN + wn * TJ * 16 + j * 16 + r] = __uint_as_float(top[j]);
        }
        // (before these are written again come the barriers of the next tile's steps)
        __builtin_amdgcn_s_waitcnt(0xc07f);                  // (no LDS access left)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int n = 0; n < kShare; ++n)
#pragma unroll
            for (int j = 0; j < TJ; ++j) top[j] = max(top[j], __float_as_uint(tops[(wm / kShare * kShare + n) * BN + wn * TJ * 16 + j * 16 + r]));
        const int y_blocks = (a.width + kBlock - 1) / kBlock, y_pitch = (y_blocks + 3) / 4 * 4;
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const int64_t c = c_first + j * 16;
            const Scale s = scale_of(top[j]);
            uint32_t q[kPieces];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                q[i] = to_f8(v, s.inverse);
            }
            const int o = first + (kPieces == 4 ? g * 16 : (g & 1) * 16 + g / 2 * 8);
            uint8_t *y = (uint8_t *)a.Y + c * y_blocks * kBlock + o;
            if constexpr (kPieces == 4) {
                const u32x4 sixteen = sixteen_outputs(q);
                if (c < a.rows && o < y_blocks * kBlock) *(u32x4 *)y = sixteen;
            } else {
                const u32x2 eight = eight_outputs(q[0], q[1]);
                if (c < a.rows && o < y_blocks * kBlock) *(u32x2 *)y = eight;
            }
            if (c < a.rows && g == 0 && wm % kShare == 0 && first < a.width) {
                const int b = first / kBlock;
                float *to = a.y_scales + c * y_pitch;
                to[b] = s.scale;
                if (b == y_blocks - 1)
                    for (int i = y_blocks; i < y_pitch; ++i) to[i] = 0.0f;
            }
        }
    } else if constexpr (sizeof(T) == 2 && kPieces % 2 == 0) {
#pragma unroll
        for (int i = 0; i < kPieces; i += 2) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                const f32x4 v = activated<T, GATED>(a, first + i * 16 + 4 * g, acc[i][j], acc[GATED ? kPieces + i : i][j]);
                const f32x4 u = activated<T, GATED>(a, first + i * 16 + 16 + 4 * g, acc[i + 1][j], acc[GATED ? kPieces + i + 1 : i + 1][j]);
                const T four[2][4] = {{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}, {(T)u[0], (T)u[1], (T)u[2], (T)u[3]}};
                u32x2 lo, hi;
                __builtin_memcpy(&lo, four[0], 8);
                __builtin_memcpy(&hi, four[1], 8);
                const u32x4 eight = eight_outputs(lo, hi);
                const int o = first + (i + (g & 1)) * 16 + g / 2 * 8;
                if (c_first + j * 16 >= a.rows || o >= a.width) continue;
                T *y = (T *)a.Y + (int64_t)(c_first + j * 16) * a.width + o;
                if (o + 8 <= a.width) {
                    __builtin_memcpy(y, &eight, 16);
                } else {
                    T out[8];
                    __builtin_memcpy(out, &eight, 16);
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (o + e < a.width) y[e] = out[e];
                }
            }
        }
    } else if constexpr (!std::is_same_v<T, F8Out>) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int o = first + i * 16 + 4 * g;
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                const f32x4 v = activated<T, GATED>(a, o, acc[i][j], acc[GATED ? kPieces + i : i][j]);
                if (c_first + j * 16 < a.rows) store_outputs<T>(a, c_first + j * 16, o, v);
            }
        }
    }
}

template <int BM, int BN, int WM, int WN, class T, bool GATED, bool WIDE>
__global__ __launch_bounds__(WM * WN * 64, 2) void f8_tile_kernel(ProductArgs a, int row_tiles)
{
    using C = Tile<BM, BN, WM, WN>;
    constexpr int TI = C::TI, TJ = C::TJ, R = C::R, kSteps = C::kSteps;
    extern __shared__ __align__(128) uint8_t lds[];
    typedef __attribute__((address_space(3))) void *lds_ptr;
    typedef const __attribute__((address_space(1))) void *global_ptr;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)(threadIdx.x & 63), r = lane & 15, g = lane >> 4;
    constexpr int kOutputs = GATED ? BM / 2 : BM;            // of the tile

    // Workgroups go to the eight dies in turn.  Each die takes a run of tiles, four columns of tiles at a time, so that what it has in flight shares rows
    // of W and of X in its cache.  A workgroup takes every gridDim.x / 8-th tile of its die's run, and asks for its next tile's first steps while it multiplies the
    // last of the one before.
    const int columns = (a.rows + BN - 1) / BN, tiles = columns * row_tiles, die = (int)blockIdx.x % 8, dies_run = tiles / 8 + (die < tiles % 8);
    const int run_first = die * (tiles / 8) + min(die, tiles % 8), stride = (int)gridDim.x / 8;
    int nth = (int)blockIdx.x / 8;
    if (nth >= dies_run) return;
    const int split = (int)blockIdx.y;
    const int t_first = 4 * (split * a.split_fours + min(split, a.split_more));
    const int steps = min(4 * (a.split_fours + (split < a.split_more)), a.blocks - t_first);

    const int wm = wave / WN, wn = wave % WN;
    const uint32_t row_bytes = (uint32_t)a.blocks * kBlock;
    // which of the buffer's rows load k of the wavefront writes: columns, then first halves of rows, then second halves
    auto load_row = [&](int k) {
        constexpr int kColumns = BN / 8 / C::kWaves;
        if (k < kColumns) return BM + (k * C::kWaves + wave) * 8;
        const int n = (k - kColumns) % C::kLate * C::kWaves + wave, half = (k - kColumns) / C::kLate;
        return n / TI * (TI * 16) + half * C::kRun + n % TI * 8;
    };
    struct Place { int o, c; };                              // a tile's first output and column
    auto place = [&](int nth) {
        const int tile = run_first + nth, band = (int)a.band_tiles.quotient((uint32_t)tile) * 4, in = tile - band * row_tiles, across = min(4, columns - band);
        const int down = across == 1 ? in : across == 2 ? in / 2 : across == 3 ? in / 3 : in / 4;
        return Place{down * kOutputs, (band + in - down * across) * BN};
    };
    // The tile that is asked for: what each load of a wavefront reads, eight rows (those beyond the last repeat it; a tile's have less than 4 GB).
    const uint8_t *base[C::kLoads];
    uint32_t offset[C::kLoads];
    const float *scale_at[C::kScaleShare];
    auto take = [&](int nth) __attribute__((always_inline)) {
        const Place at = place(nth);
        const int o0 = at.o, c0 = at.c, count = min(BN, a.rows - c0);
        // where run n of a tile's rows begins - the first output that it has, and whether it has values -, for runs of kRun rows, two to a wavefront
        auto run_output = [&](int n) { return o0 + (GATED ? n / 2 : n) * C::kRun; };
        auto run_value = [&](int n) { return GATED ? n % 2 : 0; };
        const uint32_t unit = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
        for (int k = 0; k < C::kLoads; ++k) {
            const int row = load_row(k);
            if (k >= BN / 8 / C::kWaves) {
                const int run = row / C::kRun, o = min(run_output(run) + row % C::kRun, a.width - 1);
                base[k] = a.w + ((int64_t)run_value(run) * a.width + o) * row_bytes + (int64_t)t_first * kBlock;
                offset[k] = (uint32_t)min(lane >> 3, a.width - 1 - o) * row_bytes + unit;
            } else {
                const int n = min(row - BM, count - 1);
                base[k] = a.x + (int64_t)(c0 + n) * row_bytes + (int64_t)t_first * kBlock;
                offset[k] = (uint32_t)min(lane >> 3, count - 1 - n) * row_bytes + unit;
            }
        }
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
    };
    auto request = [&](int t, uint8_t *buf, int k) {
        const uint8_t *at = base[k] + (uint32_t)t * kBlock;
        asm("" : "+s"(at));                                  // (the same for all lanes, and added up there: half the registers)
        __builtin_amdgcn_global_load_lds((global_ptr)(at + offset[k]), (lds_ptr)(buf + load_row(k) * kBlock), 16, 0, 0);
    };
    auto request_scales = [&](int q, uint8_t *buf, int k) {
        __builtin_amdgcn_global_load_lds((global_ptr)(scale_at[k] + (int64_t)q * 4), (lds_ptr)(buf + min(k * C::kWaves + wave, C::kScaleLoads - 1) * 1024), 16, 0, 0);
    };

    const int wi = wm * TI * 16 + r, wj = BM + wn * TJ * 16 + r;        // the lane's rows of the buffer
    const int lo = (g ^ (r & 7)) * 16, hi = ((g + 4) ^ (r & 7)) * 16;
    auto read_piece = [&](const uint8_t *buf, int row) { return both(*(const i32x4 *)(buf + row * kBlock + lo), *(const i32x4 *)(buf + row * kBlock + hi)); };
    auto scale_of_column = [&](const uint8_t *buf, int j) { return *(const float *)(buf + (wn * TJ * 16 + j * 16 + r) * 16); };
    auto scale_of_run = [&](const uint8_t *buf, int h) { return *(const float *)(buf + (BN + wm * 2 + h) * 16); };

    f32x4 acc[TI][TJ], p[TJ];
    Operand<WIDE> x[TJ];
    i32x8 w[R];
    float sx[TJ], sw[2], by[TJ];

    constexpr int kWaitLds = 0xc07f;                         // s_waitcnt: no LDS access left
    auto loads_left = [](int n) constexpr { return 0xf70 | (n & 15) | (n >> 4) << 14; };     // n loads left
    auto join = [&](int i, int j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[j][e], by[j], acc[i][j][e]);
        asm volatile("" : "+v"(acc[i][j]));                  // (here, not where the sum is needed next: p would have to be kept)
    };
    // What is asked for: step `ask` of the tile that was taken, and the scales of four into their buffers in turn.  (Behind the last step of the last tile that one again, so
    // that a wait always counts the same; nothing uses what it brings.)
    int ask = 0, scales_asked = 0;
    auto scales = [&](int n) { return lds + C::kScales + n % kSteps * C::kScaleBuffer; };
    auto ask_scales = [&](uint8_t *__restrict__ to) __attribute__((always_inline)) {
        if (ask % 4) return;
#pragma unroll
        for (int k = 0; k < C::kScaleShare; ++k) request_scales(ask / 4, to, k);
        ++scales_asked;
    };
    auto asked = [&]() __attribute__((always_inline)) {
        if (++ask < steps) return;
        ask = steps - 1;
        if (nth + stride >= dies_run) return;
        nth += stride;
        take(nth);
        ask = 0;
    };
    // Piece row i of a step.  What is read behind it, into the registers that it leaves: rows from `rows`, and, of the last one, columns from `cols`.
    auto piece = [&](auto I, const uint8_t *__restrict__ rows, const uint8_t *__restrict__ cols, const uint8_t *__restrict__ scales, uint8_t *__restrict__ to) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value;
        const Operand<WIDE> row = operand<WIDE>(w[i % R]);
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            join((i + TI - 1) % TI, j);
            p[j] = mfma_f8<WIDE>(row, x[j]);
            __builtin_amdgcn_sched_barrier(0);
            if (i == TI - 1) {
                x[j] = operand<WIDE>(read_piece(cols, wj + j * 16));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        w[i % R] = read_piece(rows, wi + (i + R) % TI * 16);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = C::early(i); k < C::early(i + 1); ++k) request(ask, to, k);
#pragma unroll
        for (int k = C::late(i); k < C::late(i + 1); ++k) request(ask, to, C::kEarly + k);
        if (i == 0 || i == TI / 2) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) by[j] = sx[j] * sw[i == 0 ? 0 : 1];
        }
        if (i == TI - 1) {                                   // (the next step's)
#pragma unroll
            for (int j = 0; j < TJ; ++j) sx[j] = scale_of_column(scales, j);
            sw[0] = scale_of_run(scales, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto meet = [&](auto LEFT) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        constexpr int left = loads_left(decltype(LEFT)::value);
        __builtin_amdgcn_s_waitcnt(left);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // A step.  `now` has it, `next` the one after; `to`, which is `now`, receives step `ask`.  `scales_now` and `scales_next` are at the word of their step.
    auto step = [&](const uint8_t *now, const uint8_t *next, uint8_t *to, const uint8_t *scales_now, const uint8_t *scales_next) __attribute__((always_inline)) {
        sw[1] = scale_of_run(scales_now, 1);
        each<0, C::kFree>([&](auto I) __attribute__((always_inline)) { piece(I, now, now, scales_now, to); });
        meet(std::integral_constant<int, C::kInFlight>{});
        ask_scales(scales(scales_asked));
        each<C::kFree, C::kNext>([&](auto I) __attribute__((always_inline)) { piece(I, now, now, scales_now, to); });
        meet(std::integral_constant<int, C::kInFlight>{});
        each<C::kNext, TI>([&](auto I) __attribute__((always_inline)) { piece(I, next, next, scales_next, to); });
    };

    const int nth0 = nth;
    take(nth);
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
        ask_scales(scales(scales_asked));
#pragma unroll
        for (int k = 0; k < C::kLoads; ++k) request(ask, lds + t * C::kBuffer, k);
        asked();
    }
    meet(std::integral_constant<int, C::kInFlight + C::kLate>{});
#pragma unroll
    for (int j = 0; j < TJ; ++j) x[j] = operand<WIDE>(read_piece(lds, wj + j * 16)), sx[j] = scale_of_column(scales(0), j);
    sw[0] = scale_of_run(scales(0), 0);
#pragma unroll
    for (int i = 0; i < R; ++i) w[i] = read_piece(lds, wi + i * 16);

    int buffer = 0, fours = 0;                               // of the step that is multiplied
    for (int mth = nth0; mth < dies_run; mth += stride) {
#pragma unroll
        for (auto &v : acc)
#pragma unroll
            for (auto &y : v) y = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < TJ; ++j) p[j] = f32x4{0, 0, 0, 0}, by[j] = 0.0f;
        for (int t = 0; t < steps; ++t) {
            uint8_t *now = lds + buffer * C::kBuffer;
            buffer = (buffer + 1) % kSteps;
            const int in = t % 4, in_next = t + 1 < steps ? (t + 1) % 4 : 0;
            const uint8_t *scales_now = scales(fours) + in * 4;
            fours += in_next == 0;
            step(now, lds + buffer * C::kBuffer, now, scales_now, scales(fours) + in_next * 4);
            asked();
        }
#pragma unroll
        for (int j = 0; j < TJ; ++j) join(TI - 1, j);

        const Place at = place(mth);
        store_tile<TI, TJ, WM, BN, T, GATED>(a, split, at.o + wm * (GATED ? TI * 8 : TI * 16), at.c, wm, wn, lane, acc, (float *)(lds + C::kLds));
    }
    // (what is still on its way into LDS has to be there before that is another workgroup's)
    constexpr int none = loads_left(0);
    __builtin_amdgcn_s_waitcnt(none);
}
