// The product for many columns: tiles of the output, operands through LDS.  Part of product.hip's translation unit, inside
// namespace cl::mx.
#pragma once

// A workgroup of WM x WN wavefronts makes BM outputs (rows of W) of BN columns (rows of X), a wavefront TI x TJ pieces of
// 16 x 16.  A step is one matrix instruction deep: 128 k, four blocks, 64 bytes and one word of scales of each row.
//
// LDS holds D steps.  Step t is multiplied while t + 1 lies there and t + 2 .. t + D - 1 are on their way, written by the
// loads themselves.  Its fragments are read from LDS between the multiplies: a row's fragment up to four pieces before its use, the
// columns' fragments, which a whole step uses, during the step before (a second set of registers).  Requests, reads and
// multiplies stay in program order (scheduling barriers): in a bunch behind the step's barrier they would fill their queues
// and the multiplies would wait behind them.
//
// What bounds it.  256 x 256 (eight wavefronts, one workgroup to a compute unit): 4096 x 4096 x 25088 204 us, 4.1 PFLOP/s, of which
// the loads into LDS cost 25 (measured without them) and start and stores 8; the rest are multiplies with the reads that feed
// them, at the rate that power leaves.  With experts, stores of 32-bit rows of pairs: 32768 pairs of 2048 outputs, 268 MB, are 54 of 251
// us.  64 x 64 (four wavefronts): 256 x 4096 x 9216 18.3 us - 2 to the first step, 0.18 a step, 1.3 to store -; a step takes as
// long with its loads alone and with its multiplies alone, and with two steps to a barrier.  128 x 128: eight wavefronts, two to a
// SIMD, which take over from each other: 3000 x 3000 x 300 17.3 us, on four 20.0.  More (256 x 256 on sixteen) do not fit the registers.
//
// In LDS a row's four blocks are 64 consecutive bytes, block c of row r in place c ^ (r / 2 % 4).  A read of 16 bytes a lane is
// served sixteen lanes at a time, of which eight are from one half of a half-wave and eight from the other's; those then touch each of
// the 64 banks once.  (Otherwise - in order, or with r or r / 4 - reads take twice as long, but are not what a step waits for.)
template <int BM, int BN, int WM, int WN, int D> struct Tile {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int TI = BM / WM / 16, TJ = BN / WN / 16;
    static constexpr int kAhead = TI <= 4 ? TI : 4;          // how many pieces before its use a row fragment is read
    static constexpr int kRing = TI <= 4 ? 2 * TI : TI;      // row fragments in registers
    static constexpr int slot(int f, int p) { return f % TI + (kRing > TI && ((f / TI + p) & 1) ? TI : 0); }    // of piece f, a step of parity p
    static constexpr int kCodeLoads = (BM + BN) / 16 / kWaves;    // of a wavefront and step
    static constexpr int kScaleLoads = (BM + BN) / 64;       // of the workgroup and four steps; wavefronts beyond that number repeat the last
    static constexpr int kScaleShare = (kScaleLoads + kWaves - 1) / kWaves;
    static constexpr int kBuffer = (BM + BN) * 64;
    static constexpr int kScales = D * kBuffer;              // where the scales start: three buffers of four steps
    static constexpr int kScaleBuffer = (BM + BN) * 16;
    static constexpr int kLds = kScales + 3 * kScaleBuffer;
    static_assert(BM % (WM * 16) == 0 && BN % (WN * 16) == 0 && TI >= TJ, "");
    static_assert((BM + BN) / 16 % kWaves == 0 && BM % 64 == 0 && BN % 64 == 0, "");
    // loads of a wavefront that may be on their way when step s (of four) begins: those asked for in the D - 3 steps before
    static constexpr int on_their_way(int s)
    {
        int n = 0;
        for (int i = 1; i <= D - 3; ++i) n += kCodeLoads + ((s + 8 - i) % 4 == 0 ? kScaleShare : 0);
        return n;
    }
    // (scales are asked for six steps before they have to be there: D - 3 less than that)
    static_assert(BM + BN <= kThreads && D >= 3 && D <= 8 && (D - 3) * kCodeLoads + (D + 3) / 4 * kScaleShare < 64 && (D - 2) * kCodeLoads < 64, "");       // (the count that a wait names)
};

// WEIGHTED: outputs times a weight of their row of Y.
template <int BM, int BN, int WM, int WN, int D, class T, bool WEIGHTED>
__global__ __launch_bounds__(WM * WN * 64, 2) void mx_tile_kernel(ProductArgs a, int row_tiles)
{
    using C = Tile<BM, BN, WM, WN, D>;
    constexpr int TI = C::TI, TJ = C::TJ;
    extern __shared__ __align__(128) uint8_t lds[];
    typedef __attribute__((address_space(3))) void *lds_ptr;
    typedef const __attribute__((address_space(1))) void *global_ptr;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = (int)(threadIdx.x & 63), r = lane & 15, g = lane >> 4;

    // Workgroups go to the eight dies in turn.  Each die takes a run of tiles - with one matrix and large tiles four columns of
    // tiles at a time - so that what it has in flight shares rows of W and of X in its cache.  (4096 x 8192 x 4096: 121 us, tiles in
    // order 125; 15 experts of 561 x 3661, 4784 pairs, 64 x 64: 25 us, in order 31.  With one matrix and small tiles the order as
    // it is is 2 % faster; so it is, by 8 %, with experts and the largest, few to a die, which the fuller experts' die then
    // waits for.)
    int column, m0;
    const int columns = a.order ? *a.tile_count : (a.rows + BN - 1) / BN, tiles = columns * row_tiles;
    if (a.order ? BM * BN <= 128 * 128 : BM * BN >= 128 * 128) {
        const int per = tiles / 8, more = tiles % 8, die = (int)blockIdx.x % 8, i = (int)blockIdx.x / 8;
        if (i >= per + (die < more)) return;
        const int tile = die * per + min(die, more) + i, band = a.order ? 1 : 4;
        const int first = (int)a.band_tiles.quotient((uint32_t)tile) * band, in = tile - first * row_tiles, across = min(band, columns - first);
        const int down = across == 1 ? in : across == 2 ? in / 2 : across == 3 ? in / 3 : in / 4;
        column = first + in - down * across;
        m0 = down * BM;
    } else {
        if ((int)blockIdx.x >= tiles) return;
        column = (int)a.row_tiles.quotient(blockIdx.x);
        m0 = ((int)blockIdx.x - column * row_tiles) * BM;
    }
    Columns c;
    if (!columns_of<BN>(a, column, c)) return;
    const bool routed = !a.order || c.expert < a.experts;
    const int split = (int)blockIdx.y, all_steps = a.blocks / 4;
    const int t_first = split * a.split_steps + min(split, a.split_more);
    const int steps = routed ? a.split_steps + (split < a.split_more) : 0;

    // Which rows and columns the wavefront has.  A SIMD gets wavefronts s and s + 4: those have different columns, so that a tile
    // that is not full leaves every SIMD some.
    const int wm = wave / WN, wn = (wave + wave / 4 * (WN / 2)) % WN;
    // The rows of X of what the wavefront loads, and the row of Y of its column `lane`: all asked for before the first is used.  (2194
    // tokens, 8 of 55 experts of 2238 x 1965: 149.7 us in all, one after the other 152.1.)  Columns beyond the last repeat it.
    auto place = [&](int n) { return c.first + min(max(n, 0), c.count - 1); };
    auto load_row = [&](int i) { return (i * C::kWaves + wave) * 16 + (lane >> 2); };
    auto scale_load = [&](int i) { return min(i * C::kWaves + wave, C::kScaleLoads - 1); };
    int x_code[C::kCodeLoads], x_scale[C::kScaleShare], y_row = place(wn * TJ * 16 + lane);
#pragma unroll
    for (int i = 0; i < C::kCodeLoads; ++i) x_code[i] = place(load_row(i) - BM);
#pragma unroll
    for (int i = 0; i < C::kScaleShare; ++i) x_scale[i] = place(scale_load(i) * 64 + lane - BM);
    static_assert(TJ * 16 <= 64, "");
    if (a.order) {
#pragma unroll
        for (int i = 0; i < C::kCodeLoads; ++i) x_code[i] = a.order[x_code[i]];
#pragma unroll
        for (int i = 0; i < C::kScaleShare; ++i) x_scale[i] = a.order[x_scale[i]];
        y_row = a.order[y_row];
        if (a.x_div.d > 1) {
#pragma unroll
            for (int i = 0; i < C::kCodeLoads; ++i) x_code[i] = (int)a.x_div.quotient((uint32_t)x_code[i]);
#pragma unroll
            for (int i = 0; i < C::kScaleShare; ++i) x_scale[i] = (int)a.x_div.quotient((uint32_t)x_scale[i]);
        }
    }
    float weight = 1.0f;
    if (WEIGHTED) weight = routed ? a.weights[y_row] : 0.0f;

    // where each load of a wavefront reads: rows of W beyond the last repeat it (a tile's rows have less than 4 GB)
    const uint32_t row_bytes = (uint32_t)a.blocks * 16;
    const int64_t w_first = (routed ? (int64_t)c.expert * a.M : 0) + m0;
    const uint8_t *w_tile = a.w_codes + w_first * row_bytes, *w_tile_scales = a.w_scales + w_first * a.blocks;
    auto w_row = [&](int row) { return (uint32_t)min(row, a.M - 1 - m0); };
    const uint8_t *code_at[C::kCodeLoads], *scale_at[C::kScaleShare];
#pragma unroll
    for (int i = 0; i < C::kCodeLoads; ++i) {
        const int chunk = (lane & 3) ^ (lane >> 3 & 3);
        code_at[i] = (i * C::kWaves + wave < BM / 16 ? w_tile + w_row(load_row(i)) * row_bytes : a.x_codes + (uint64_t)(uint32_t)x_code[i] * row_bytes) + chunk * 16;
    }
#pragma unroll
    for (int i = 0; i < C::kScaleShare; ++i) {
        const int row = scale_load(i) * 64 + lane;
        // (a row of fewer than four steps is read below, and what these loads bring is not used)
        scale_at[i] = all_steps < 4 ? a.w_codes : row < BM ? w_tile_scales + w_row(row) * (uint32_t)a.blocks : a.x_scales + (uint64_t)(uint32_t)x_scale[i] * (uint32_t)a.blocks;
    }
    // code load k of step t into its buffer
    auto request_code = [&](int t, uint8_t *buf, int k) {
        __builtin_amdgcn_global_load_lds((global_ptr)(code_at[k] + (int64_t)(t_first + t) * 64), (lds_ptr)(buf + (k * C::kWaves + wave) * 1024), 16, 0, 0);
    };
    // scale load k of steps 4 q .. 4 q + 3.  (One word a step and row would be a load of 64 cache lines each time.)  Where fewer
    // than four steps are left in the row, its last four are loaded: shift(q) words in front of what is wanted.
    auto request_scales = [&](int q, uint8_t *buf, int k) {
        const int at = max(0, min(t_first + 4 * q, all_steps - 4));
        __builtin_amdgcn_global_load_lds((global_ptr)(scale_at[k] + (int64_t)at * 4), (lds_ptr)(buf + scale_load(k) * 1024), 16, 0, 0);
    };
    auto shift = [&](int q) { return all_steps < 4 ? 0 : t_first + 4 * q - min(t_first + 4 * q, all_steps - 4); };

    // its first output of each row of Y, and the bias from there on
    constexpr int kWide = TI * 16, kLanes = kWide / 4;
    const int m = m0 + wm * kWide + lane % kLanes * 4;
    const f32x4 bias = bias_of(a, c.expert, m);
    const bool idle = wn * TJ * 16 >= c.count;      // no columns: the wavefront loads, and multiplies nothing
    const int wi = wm * TI * 16 + r, wj = BM + wn * TJ * 16 + r;        // the lane's rows of the buffer
    const int at_code = (g ^ (r >> 1 & 3)) * 16;
    auto read_code = [&](const uint8_t *buf, int row) { return *(const i32x4 *)(buf + row * 64 + at_code); };
    // The scales of a row's four steps, by step when they arrive, are turned in place (a thread per row) so that the word of
    // block g has its bytes of the four steps: one read for four multiplies, which pick their byte.  (Reading a byte a
    // step, the LDS reads of scales took a third of the time: 4096 x 4096 x 25088 240 us, now 204.)
    auto turned = [&](u32x4 v, int late) {
        const uint32_t ab01 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400), ab23 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602);
        const uint32_t cd01 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400), cd23 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602);
        return u32x4{__builtin_amdgcn_perm(cd01, ab01, 0x05040100) >> late, __builtin_amdgcn_perm(cd01, ab01, 0x07060302) >> late,
                     __builtin_amdgcn_perm(cd23, ab23, 0x05040100) >> late, __builtin_amdgcn_perm(cd23, ab23, 0x07060302) >> late};
    };
    auto turn_scales = [&](uint8_t *buf, int q) {
        if (threadIdx.x >= BM + BN) return;
        u32x4 *at = (u32x4 *)(buf + threadIdx.x * 16);
        *at = turned(*at, 8 * shift(q));
    };
    // (apart from the above: a load into registers there would have every turn wait for all loads on their way)
    auto short_scales = [&](uint8_t *buf) {
        if (threadIdx.x >= BM + BN) return;
        const int row = (int)threadIdx.x;
        const int at = place(row - BM), x = a.order ? (int)a.x_div.quotient((uint32_t)a.order[at]) : at;
        const uint8_t *from = row < BM ? w_tile_scales + w_row(row) * (uint32_t)a.blocks : a.x_scales + (uint64_t)(uint32_t)x * (uint32_t)a.blocks;
        u32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < all_steps) v[i] = ((const uint32_t *)from)[i];
        *(u32x4 *)(buf + row * 16) = turned(v, 0);
    };
    auto read_scales = [&](const uint8_t *buf, int row) { return *(const int *)(buf + row * 16 + g * 4); };

    f32x4 acc[TI][TJ];
#pragma unroll
    for (auto &x : acc)
#pragma unroll
        for (auto &y : x) y = f32x4{0, 0, 0, 0};
    i32x4 w[C::kRing], x[2][TJ];
    int sw[TI], sx[TJ], sx_next[TJ];

    constexpr int kWaitLds = 0xc07f;                         // s_waitcnt: no LDS access left
    auto loads_left = [](int n) constexpr { return 0xf70 | (n & 15) | (n >> 4) << 14; };     // n loads left
    auto barrier = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Step t = 4 q + S: `now` and `next` hold its codes and those of the step after, `to` receives those of step `ask`.  Step 4 q
    // asks for the scales of the eighth to eleventh step after it, step 4 q + 2 turns those of the next four, and step 4 q + 3
    // reads them.
    auto step = [&](auto S, const uint8_t *__restrict__ now, const uint8_t *__restrict__ next, uint8_t *__restrict__ to, uint8_t *__restrict__ scales_next,
                    uint8_t *__restrict__ scales_to, int q, int ask, int ask_scales) __attribute__((always_inline)) {
        constexpr int s = decltype(S)::value, p = s & 1;
        // every wavefront's loads of step t + 1 have arrived, and all reads of the buffers that are asked for next are done
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        constexpr int left = loads_left(C::on_their_way(s));
        __builtin_amdgcn_s_waitcnt(left);
        barrier();
        if (s == 2) turn_scales(scales_next, q + 1);
        if (idle) {
#pragma unroll
            for (int k = 0; k < C::kCodeLoads; ++k) request_code(ask, to, k);
            if (s == 0) {
#pragma unroll
                for (int k = 0; k < C::kScaleShare; ++k) request_scales(ask_scales, scales_to, k);
            }
            return;
        }
        if (s == 0) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) sx[j] = sx_next[j];
        }
#pragma unroll
        for (int i = 0; i < TI; ++i) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                if (j == 0) {
                    const int f = i + C::kAhead;
                    w[C::slot(f, p)] = read_code(f < TI ? now : next, wi + f % TI * 16);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (j == TJ / 2 && i >= TI - TJ) {
                    const int f = i - (TI - TJ);
                    x[1 - p][f] = read_code(next, wj + f * 16);
                    if (s == 3) sx_next[f] = read_scales(scales_next, wj + f * 16);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (j == TJ - 1) {
#pragma unroll
                    for (int k = i; k < C::kCodeLoads; k += TI) request_code(ask, to, k);
                    if (s == 0 && i == TI - 1) {
#pragma unroll
                        for (int k = 0; k < C::kScaleShare; ++k) request_scales(ask_scales, scales_to, k);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                acc[i][j] = mfma_fp4<s>(w[C::slot(i, p)], x[p][j], acc[i][j], sw[i], sx[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (s == 3) {
                sw[i] = read_scales(scales_next, wi + i * 16);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    if (steps > 0) {
        auto buffer = [&](int t) { return lds + t % D * C::kBuffer; };
        auto scales = [&](int q) { return lds + C::kScales + q % 3 * C::kScaleBuffer; };
        const int last = steps - 1;
        auto at = [&](auto S, int t) __attribute__((always_inline)) {
            const int q = t / 4;
            step(S, buffer(t), buffer(t + 1), buffer(t + D - 1), scales(q + 1), scales(q + 2), q, min(t + D - 1, last), min(q + 2, last / 4));
        };
        // (requests beyond the last step repeat it, so that a wait always counts the same; nothing reads what they bring.  The first
        // ones are in the order that steps 1 - D .. -1 would ask in, of which step -4 asks for scales: step 0 counts them so)
        auto request_first_scales = [&](int q) {
#pragma unroll
            for (int k = 0; k < C::kScaleShare; ++k) request_scales(min(q, last / 4), scales(q), k);
        };
        request_first_scales(0);
        if (D < 5) request_first_scales(1);
#pragma unroll
        for (int t = 0; t < D - 1; ++t) {
#pragma unroll
            for (int k = 0; k < C::kCodeLoads; ++k) request_code(min(t, last), buffer(t), k);
            if (t == D - 5) request_first_scales(1);
        }
        constexpr int all_but_first = loads_left((D - 2) * C::kCodeLoads + (D < 5 ? 0 : C::kScaleShare));
        __builtin_amdgcn_s_waitcnt(all_but_first);
        barrier();
        if (all_steps < 4) short_scales(scales(0));
        else turn_scales(scales(0), 0);
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        barrier();
#pragma unroll
        for (int j = 0; j < TJ; ++j) x[0][j] = read_code(lds, wj + j * 16), sx_next[j] = read_scales(scales(0), wj + j * 16);
#pragma unroll
        for (int i = 0; i < TI; ++i) sw[i] = read_scales(scales(0), wi + i * 16);
#pragma unroll
        for (int i = 0; i < C::kAhead; ++i) w[i] = read_code(lds, wi + i * 16);
        int t = 0;
        for (; t + 4 <= steps; t += 4) {
            at(std::integral_constant<int, 0>{}, t);
            at(std::integral_constant<int, 1>{}, t + 1);
            at(std::integral_constant<int, 2>{}, t + 2);
            at(std::integral_constant<int, 3>{}, t + 3);
        }
        if (t < steps) at(std::integral_constant<int, 0>{}, t);
        if (t + 1 < steps) at(std::integral_constant<int, 1>{}, t + 1);
        if (t + 2 < steps) at(std::integral_constant<int, 2>{}, t + 2);
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        constexpr int none = loads_left(0);
        __builtin_amdgcn_s_waitcnt(none);
        barrier();
    }

    // A wavefront's outputs go through LDS, sixteen columns at a time, so that what it stores of a row of Y is consecutive.
    constexpr int kPitch = kWide + 4;
    static_assert(C::kWaves * 16 * kPitch * 4 <= C::kLds, "");
    float *mine = (float *)lds + wave * 16 * kPitch;
#pragma unroll
    for (int j = 0; j < TJ; ++j) {
#pragma unroll
        for (int i = 0; i < TI; ++i) *(f32x4 *)(mine + r * kPitch + i * 16 + 4 * g) = acc[i][j];
        lanes_exchange();
        const int first = wn * TJ * 16 + j * 16;
        for (int n = lane / kLanes; n < 16; n += 64 / kLanes) {
            const f32x4 v = *(const f32x4 *)(mine + n * kPitch + lane % kLanes * 4);
            const int row = __shfl(y_row, j * 16 + n);
            const float scale = WEIGHTED ? __shfl(weight, j * 16 + n) : 1.0f;
            if (first + n >= c.count) continue;
            if (a.part) store_part(a, split, row, m, v);
            else store_outputs<T, WEIGHTED>(a, row, m, v, bias, scale);
        }
        lanes_exchange();
    }
}
