// The choice of experts for tokens, and the lists of tokens that each expert is given.
#include <algorithm>

#include "quantize_kernel.hpp"

namespace cl {
namespace mx {

// ------------------------------------------------------------------------- //
// the choice
// ------------------------------------------------------------------------- //
struct RouteArgs {
    const void *logits;
    int64_t stride;
    const float *bias;
    int32_t *experts_out;
    float *weights_out;
    int tokens, experts, k, groups, kept, top2, sigmoid, renormalize;
    float scale;
};

template <int L, class F> __device__ __forceinline__ float over_lanes(float v, F f)
{
#pragma unroll
    for (int d = 1; d < L; d *= 2) v = f(v, __shfl_xor(v, d));
    return v;
}

// Chosen experts whose scores come to less than this together take their weights from their logits instead, as exp(x_j - largest): some scores
// may be below what fp32 holds, and their ratios are not.  (Softmax: the common denominator cancels.  Logistic function: it is exp(x)
// there, to one part in 2^60.)
constexpr float kSmallScores = 0x1p-60f;

// L lanes to a token, C consecutive experts to a lane, so that the lower of two lanes has the lower experts.  k rounds: the
// largest key of the lanes' own largest, the lowest lane that has it, which then leaves its expert out.
template <class T, int L, int C> __global__ __launch_bounds__(256) void route_kernel(RouteArgs a)
{
    __shared__ float s_key[256 * C];                         // keys of the groups' scores
    __shared__ float s_group[256 / L][CL_ROUTE_MAX_GROUPS];
    const int sub = threadIdx.x % L, local = threadIdx.x / L;
    const int token = (int)blockIdx.x * (256 / L) + local;
    const bool live = token < a.tokens;
    const float lowest = sizeof(T) == 4 ? -3.402823466e38f : std::is_same<T, f16_t>::value ? -65504.0f : -3.38953138925e38f;
    const T *x = (const T *)a.logits + (int64_t)(live ? token : 0) * a.stride;
    float key[C], score[C];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int e = sub * C + j;
        const float v = live && e < a.experts ? to_float(x[e]) : -INFINITY;
        key[j] = v > lowest ? v : -INFINITY;                 // (NaN too)
        top = fmaxf(top, key[j]);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int j = 0; j < C; ++j) score[j] = 1.0f / (1.0f + expf(-key[j]));
    } else {
        top = over_lanes<L>(top, [](float p, float q) { return fmaxf(p, q); });
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            // (equal to the largest: 1 also where that is infinite; masked: 0 also where all are)
            score[j] = key[j] == -INFINITY ? 0.0f : key[j] == top ? 1.0f : expf(key[j] - top);
            sum += score[j];
        }
        sum = over_lanes<L>(sum, [](float p, float q) { return p + q; });
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) score[j] *= inv;
    }
    if (a.bias || a.groups > 1) {
        float biased[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int e = sub * C + j;
            const float b = a.bias && e < a.experts ? score[j] + a.bias[e] : score[j];
            biased[j] = key[j] == -INFINITY || !(b == b) ? -INFINITY : b;
            if (a.bias) key[j] = biased[j];
        }
        if (a.groups > 1) {
            const int size = a.experts / a.groups;
            float *mine = s_key + local * (L * C);
#pragma unroll
            for (int j = 0; j < C; ++j) mine[sub * C + j] = biased[j];
            __syncthreads();
            for (int g = sub; g < a.groups; g += L) {
                float best = -INFINITY, second = -INFINITY;
                for (int i = 0; i < size; ++i) {
                    const float v = mine[g * size + i];
                    second = fmaxf(second, fminf(best, v));
                    best = fmaxf(best, v);
                }
                s_group[local][g] = a.top2 && second != -INFINITY ? best + second : best;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int e = sub * C + j;
                if (e >= a.experts) continue;
                const int g = e / size;
                const float v = s_group[local][g];
                int before = 0;
                for (int o = 0; o < a.groups; ++o) before += s_group[local][o] > v || (s_group[local][o] == v && o < g);
                if (before >= a.kept) key[j] = -INFINITY;
            }
        }
    }
    // lane i of the token keeps what round i chose
    int chosen = -1;
    float weight = 0.0f;
    const int lane = threadIdx.x & 63, base = lane - sub;
    for (int i = 0; i < a.k; ++i) {
        float best = key[0], s = score[0];
        int at = 0;
#pragma unroll
        for (int j = 1; j < C; ++j)
            if (key[j] > best) best = key[j], s = score[j], at = j;
        const float most = over_lanes<L>(best, [](float p, float q) { return fmaxf(p, q); });
        const uint64_t has = __ballot(best == most) >> base & (L == 64 ? ~0ull : (1ull << L) - 1);
        const int winner = __ffsll((unsigned long long)has) - 1;
        const int e = __shfl(sub * C + at, base + winner);
        const float w = __shfl(s, base + winner);
        if (sub == i && most != -INFINITY) chosen = e, weight = w;
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (sub == winner && j == at) key[j] = -INFINITY;
    }
    if (a.renormalize) {
        float sum = over_lanes<L>(weight, [](float p, float q) { return p + q; });
        if (sum < kSmallScores) {                            // (the same for all lanes of a token)
            const float logit = live && chosen >= 0 ? to_float(x[chosen]) : -INFINITY;
            const float most = over_lanes<L>(logit, [](float p, float q) { return fmaxf(p, q); });
            // (beside an infinite logit the others' scores are 0)
            weight = logit == -INFINITY || (!a.sigmoid && top == INFINITY) ? 0.0f : expf(logit - most);
            sum = over_lanes<L>(weight, [](float p, float q) { return p + q; });
        }
        weight = sum > 0.0f ? weight / sum : 0.0f;
    }
    if (live && sub < a.k) {
        a.experts_out[(int64_t)token * a.k + sub] = chosen;
        a.weights_out[(int64_t)token * a.k + sub] = weight * a.scale;
    }
}

// exp(x) from the hardware's 2^x: what rounding leaves of x log2(e), and log2(e) itself, goes in as a factor, so that the error stays
// near one unit in the last place where |x| is large.
__device__ __forceinline__ float exp_of(float x)
{
    const float log2e = 1.44269504f, rest = 1.92596299e-8f, ln2 = 0.693147181f;
    const float p = x * log2e, r = fmaf(x, log2e, -p) + x * rest, e = __builtin_amdgcn_exp2f(p);
    return fmaf(e, r * ln2, e);
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true); }
template <int CTRL> __device__ __forceinline__ float dpp(float x) { return __uint_as_float(dpp<CTRL>(__float_as_uint(x))); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140, kRotate = 0x120;

// f over the sixteen lanes of a row, in every lane.  (Mirrors stand in for the exchanges over 4 and 8, as what they exchange is the
// same in all lanes of a quad and of a half.)
template <class V, class F> __device__ __forceinline__ V over_row(V v, F f)
{
    v = f(v, dpp<kXor1>(v));
    v = f(v, dpp<kXor2>(v));
    v = f(v, dpp<kHalfMirror>(v));
    return f(v, dpp<kMirror>(v));
}

// Numbers in the order of floats, the two zeros equal; 0 is below all of them.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x == -INFINITY ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Groups (of `lanes` lanes each) that come before this lane's: a larger score, or an equal one and lower experts.
template <int R> __device__ __forceinline__ void groups_before(float v, int g, int row_lane, int lanes, int &before)
{
    if constexpr (R < 16) {
        if (R % lanes == 0) {
            const float o = dpp<kRotate + R>(v);
            const int og = ((row_lane - R) & 15) / lanes;
            before += o > v || (o == v && og < g);
        }
        groups_before<R + 1>(v, g, row_lane, lanes, before);
    }
}

// The same for up to sixteen choices among up to 16 C experts: sixteen lanes - a row, within which lanes exchange registers without the LDS -
// to a token, C experts to a lane, four tokens to a wavefront.  A lane keeps its three largest keys and looks for the next
// three only when all are taken (8 of 256 experts in half of eight groups: one round of eight, over a wavefront's four tokens).
// What bounds it is instructions, which have 61 % of the vector units' cycles (counters), and rounds that wait for each other: 16381 tokens
// of 256 experts, logistic scores, a bias, groups, 8 chosen, 17 us - of 16.8 MB, which take 3.5 - where sixty-four lanes to a token, four
// experts each, and exchanges through LDS took 30.
// group_lanes: lanes of a group, a power of two; 0: groups do not end with a lane (16381 tokens, 12 groups of 20 experts: 16 us, 33).
template <class T, int C> __global__ __launch_bounds__(256) void route_rows_kernel(RouteArgs a, int group_lanes)
{
    __shared__ float s_score[16][16 * C];
    __shared__ int32_t s_chosen[16][16];
    const int sub = threadIdx.x & 15, local = threadIdx.x / 16, lane = threadIdx.x & 63;
    const int token = (int)blockIdx.x * 16 + local;
    const bool live = token < a.tokens;
    const float lowest = sizeof(T) == 4 ? -3.402823466e38f : std::is_same<T, f16_t>::value ? -65504.0f : -3.38953138925e38f;
    const T *x = (const T *)a.logits + (int64_t)(live ? token : 0) * a.stride + sub * C;
    const int mine = live ? a.experts - sub * C : 0;         // experts of this lane, or more
    float logit[C], score[C];
    float top = -INFINITY;
    if (mine >= C) {
        T v[C];
        load_values<C>(x, v);
#pragma unroll
        for (int j = 0; j < C; ++j) logit[j] = to_float(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) logit[j] = j < mine ? to_float(x[j]) : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        logit[j] = logit[j] > lowest ? logit[j] : -INFINITY;         // (NaN too)
        top = fmaxf(top, logit[j]);
    }
    // (values first, choices after: a choice between a value and its computation would be a branch each)
    if (a.sigmoid) {
        // (below -88, where exp(-x) would leave the range: 0; the reciprocal's error is one unit in the last place)
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const float s = __builtin_amdgcn_rcpf(1.0f + exp_of(__builtin_amdgcn_fmed3f(-logit[j], -100.0f, 88.0f)));
            score[j] = logit[j] < -88.0f ? 0.0f : s;
        }
    } else {
        top = over_row(top, [](float p, float q) { return fmaxf(p, q); });
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            // (equal to the largest: 1 also where that is infinite; masked: 0 also where all are)
            const float e = exp_of(fmaxf(logit[j] - top, -200.0f)), s = logit[j] == top ? 1.0f : e;
            score[j] = logit[j] == -INFINITY ? 0.0f : s;
            sum += score[j];
        }
        sum = over_row(sum, [](float p, float q) { return p + q; });
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) score[j] *= inv;
    }
    uint32_t key[C];
    bool open = true;
    if (a.bias || a.groups > 1) {
        float biased[C];
#pragma unroll
        for (int j = 0; j < C; ++j) biased[j] = score[j];
        if (a.bias) {
            float bias[C];
            if (mine >= C) {
                load_values<C>(a.bias + sub * C, bias);
            } else {
#pragma unroll
                for (int j = 0; j < C; ++j) bias[j] = a.bias[min(sub * C + j, a.experts - 1)];
            }
#pragma unroll
            for (int j = 0; j < C; ++j) biased[j] += bias[j];
        }
        float best = -INFINITY, second = -INFINITY;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            biased[j] = logit[j] == -INFINITY || !(biased[j] == biased[j]) ? -INFINITY : biased[j];
            key[j] = ordered(a.bias ? biased[j] : logit[j]);
            second = fmaxf(second, fminf(best, biased[j]));
            best = fmaxf(best, biased[j]);
        }
        if (a.groups > 1 && group_lanes > 0) {
            auto merge = [&](float b, float s) {
                second = fmaxf(fmaxf(second, s), fminf(best, b));
                best = fmaxf(best, b);
            };
            if (group_lanes > 1) merge(dpp<kXor1>(best), dpp<kXor1>(second));
            if (group_lanes > 2) merge(dpp<kXor2>(best), dpp<kXor2>(second));
            if (group_lanes > 4) merge(dpp<kHalfMirror>(best), dpp<kHalfMirror>(second));
            const float v = a.top2 && second != -INFINITY ? best + second : best;
            int before = 0;
            groups_before<1>(v, sub / group_lanes, sub, group_lanes, before);
            open = before < a.kept;
        } else if (a.groups > 1) {
            // groups that do not end with a lane: lane g looks group g over in LDS
            const int size = a.experts / a.groups;
#pragma unroll
            for (int j = 0; j < C; ++j) s_score[local][sub * C + j] = biased[j];
            lanes_exchange();
            best = second = -INFINITY;
            if (sub < a.groups)
                for (int i = 0; i < size; ++i) {
                    const float v = s_score[local][sub * size + i];
                    second = fmaxf(second, fminf(best, v));
                    best = fmaxf(best, v);
                }
            lanes_exchange();
            const float v = a.top2 && second != -INFINITY ? best + second : best;
            int before = 0;
            groups_before<1>(v, sub, sub, 1, before);
            const uint32_t kept = (uint32_t)(__ballot(sub < a.groups && before < a.kept) >> (lane & 48)) & 0xffffu;
            int g = sub * C / size, left = (g + 1) * size - sub * C;         // the group of expert j, and how many it has from there on
#pragma unroll
            for (int j = 0; j < C; ++j) {
                key[j] = g < 16 && kept >> g & 1 ? key[j] : 0u;
                if (--left == 0) ++g, left = size;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) key[j] = ordered(logit[j]);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) s_score[local][sub * C + j] = score[j];
    // the three largest keys of the lane that are not taken, the lower expert first where they are equal
    uint32_t best = 0, second = 0, third = 0, taken = 0;
    int best_at = 0, second_at = 0, third_at = 0;
    auto look = [&] {
        best = second = third = 0;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const uint32_t k = taken >> j & 1 ? 0u : key[j];
            const bool before_best = k > best, before_second = k > second, before_third = k > third;
            third_at = before_second ? second_at : before_third ? j : third_at;
            second_at = before_best ? best_at : before_second ? j : second_at;
            best_at = before_best ? j : best_at;
            third = max(third, min(second, k));
            second = max(second, min(best, k));
            best = max(best, k);
        }
    };
    if (open) look();
    for (int i = 0; i < a.k; ++i) {
        const uint32_t most = over_row(best, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
        const uint32_t has = (uint32_t)(__ballot(best == most) >> (lane & 48)) & 0xffffu;
        const bool winner = (has & (0u - has)) == 1u << sub;
        if (winner) {
            s_chosen[local][i] = most ? sub * C + best_at : -1;
            taken |= 1u << best_at;
            best = second;
            best_at = second_at;
            second = third;
            second_at = third_at;
            third = 0;
            if (best == 0 && most != 0 && i + 1 < a.k) look();
        }
    }
    lanes_exchange();                                        // (a token's lanes are one wavefront's: its LDS accesses are in order)
    int chosen = -1;
    float weight = 0.0f;
    if (sub < a.k) {
        chosen = s_chosen[local][sub];
        weight = chosen >= 0 ? s_score[local][chosen] : 0.0f;
    }
    if (a.renormalize) {
        float sum = over_row(weight, [](float p, float q) { return p + q; });
        if (sum < kSmallScores) {                            // (the same for all lanes of a token)
            const float l = live && chosen >= 0 ? to_float(x[chosen - sub * C]) : -INFINITY;
            const float most = over_row(l, [](float p, float q) { return fmaxf(p, q); });
            // (beside an infinite logit the others' scores are 0)
            weight = l == -INFINITY || (!a.sigmoid && top == INFINITY) ? 0.0f : exp_of(fmaxf(l - most, -200.0f));
            sum = over_row(weight, [](float p, float q) { return p + q; });
        }
        weight = sum > 0.0f ? weight / sum : 0.0f;
    }
    if (live && sub < a.k) {
        a.experts_out[(int64_t)token * a.k + sub] = chosen;
        a.weights_out[(int64_t)token * a.k + sub] = weight * a.scale;
    }
}

// launch(arguments, workgroups) over the tokens, `per` of them to a workgroup of 256, in pieces whose threads number less than 2^32.
template <class T, class F> static int32_t in_pieces(RouteArgs a, int per, F launch)
{
    const int64_t tokens = a.tokens, step = (int64_t)per << 23;
    for (int64_t t0 = 0; t0 < tokens; t0 += step) {
        a.tokens = (int)std::min(step, tokens - t0);
        launch(a, dim3((unsigned)(((int64_t)a.tokens + per - 1) / per)));
        MX_HIP_TRY(hipGetLastError());
        a.logits = (const T *)a.logits + step * a.stride;
        a.experts_out += step * a.k;
        a.weights_out += step * a.k;
    }
    return CL_OK;
}

template <class T, int C> static int32_t launch_route_rows(const RouteArgs &a, int group_lanes, hipStream_t st)
{
    return in_pieces<T>(a, 16, [&](const RouteArgs &p, dim3 grid) { hipLaunchKernelGGL((route_rows_kernel<T, C>), grid, dim3(256), 0, st, p, group_lanes); });
}

template <class T, int L, int C> static int32_t launch_route(const RouteArgs &a, hipStream_t st)
{
    return in_pieces<T>(a, 256 / L, [&](const RouteArgs &p, dim3 grid) { hipLaunchKernelGGL((route_kernel<T, L, C>), grid, dim3(256), 0, st, p); });
}

// ------------------------------------------------------------------------- //
// the lists: a stable counting sort of the pairs (token, j) by their expert, pairs without one last
// ------------------------------------------------------------------------- //
// Pairs of one workgroup: a multiple of 4096 that makes at most 256 workgroups, each of which adds the others' counts up.
constexpr int kListThreads = 1024, kListWaves = kListThreads / 64;
// Up to this many pairs, each workgroup counts all of them itself, and the counts need no launch of their own: with the
// quantisation beside, 22971 pairs of 11 experts take 13.7 us, in two launches 20.4; 32768 pairs of 64 take 6 us less.
constexpr int kListAll = 32768;
static int64_t list_chunk(int64_t pairs) { return std::max<int64_t>(1, (pairs + 4096 * 256 - 1) / (4096 * 256)) * 4096; }

ExpertLists expert_lists_at(void *base, int32_t tokens, int32_t k, int32_t experts)
{
    ExpertLists L;
    const int64_t pairs = (int64_t)tokens * k, chunks = std::min<int64_t>(256, (pairs + 4095) / 4096);       // (not fewer than there are, and not fewer for more pairs)
    size_t at = 0;
    auto take = [&](size_t bytes) { char *p = (char *)base + at; at += round_up(bytes, 256); return p; };
    L.offsets = (int32_t *)take(((size_t)experts + 2) * 4);
    L.tile_count = (int32_t *)take(kTileWidths * 4);
    L.order = (int32_t *)take((size_t)pairs * 4);
    for (int w = 0; w < kTileWidths; ++w) {
        L.max_tiles[w] = pairs / kTileWidth[w] + std::min<int64_t>(pairs, (int64_t)experts + 1);
        L.tiles[w] = (int2 *)take((size_t)L.max_tiles[w] * sizeof(int2));
    }
    L.chunk_counts = (int32_t *)take(pairs > kListAll ? (size_t)chunks * ((size_t)experts + 1) * 4 : 0);
    L.bytes = at;
    return L;
}

__device__ __forceinline__ int bucket_of(int e, int experts) { return e >= 0 && e < experts ? e : experts; }

struct ListArgs {
    ExpertLists L;
    const int32_t *experts_of;
    int pairs, chunk, chunks, experts;
};

__device__ __forceinline__ void lists_count(const ListArgs &a)
{
    extern __shared__ int32_t list_lds[];
    const int32_t *experts_of = a.experts_of;
    const int pairs = a.pairs, chunk = a.chunk, experts = a.experts;
    int32_t *counts = a.L.chunk_counts, *n = list_lds;
    for (int b = threadIdx.x; b <= experts; b += kListThreads) n[b] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * chunk, p1 = min((int64_t)pairs, p0 + chunk);
    for (int64_t p = p0 + threadIdx.x; p < p1; p += kListThreads) atomicAdd(&n[bucket_of(experts_of[p], experts)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b <= experts; b += kListThreads) counts[(int64_t)blockIdx.x * (experts + 1) + b] = n[b];
}

// Every workgroup finds where its own pairs of each expert go (the first: also the tiles), and puts them there.  Wavefront w has the
// w-th sixteenth of the chunk.
__device__ __forceinline__ void lists_place(const ListArgs &a)
{
    extern __shared__ int32_t list_lds[];
    const ExpertLists &L = a.L;
    const int32_t *experts_of = a.experts_of;
    const int pairs = a.pairs, chunk = a.chunk, chunks = a.chunks, experts = a.experts;
    const int buckets = experts + 1, wave = (int)threadIdx.x / 64, lane = (int)threadIdx.x & 63;
    int32_t *at = list_lds;                                  // [wavefront][bucket]: how many, then where the next goes
    int32_t *starts = at + kListWaves * buckets;             // [1 + kTileWidths][bucket + 1]: first pair, first tile of each width
    int32_t *others = starts + (1 + kTileWidths) * (buckets + 1);        // [earlier, later chunks][bucket]: how many, where they are counted here
    const bool count_all = chunks > 1 && pairs <= kListAll;
    __shared__ int32_t wave_sum[kListWaves][1 + kTileWidths];
    for (int i = threadIdx.x; i < kListWaves * buckets; i += kListThreads) at[i] = 0;
    for (int i = threadIdx.x; i < 2 * buckets; i += kListThreads) others[i] = 0;
    __syncthreads();
    if (count_all) {
        // kListAll / kListThreads of each thread, half of them asked for together
        const int p0 = (int)blockIdx.x * chunk, p1 = p0 + chunk;
        constexpr int kEach = kListAll / kListThreads / 2;
        for (int base = 0; base < pairs; base += kEach * kListThreads) {
            int e[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) e[i] = experts_of[min(base + i * kListThreads + (int)threadIdx.x, pairs - 1)];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int p = base + i * kListThreads + (int)threadIdx.x;
                if (p < pairs && (p < p0 || p >= p1)) atomicAdd(&others[(p < p0 ? 0 : buckets) + bucket_of(e[i], experts)], 1);
            }
        }
    }
    const int64_t first = (int64_t)blockIdx.x * chunk + (int64_t)wave * (chunk / kListWaves);
    const int64_t end = min((int64_t)pairs, first + chunk / kListWaves);
    // the buckets of four times 64 pairs from p0 on, -1 beyond the end; asked for together
    auto buckets_of = [&](int64_t p0, int *b) {
        int e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = experts_of[min(p0 + i * 64 + lane, (int64_t)pairs - 1)];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = p0 + i * 64 + lane < end ? bucket_of(e[i], experts) : -1;
    };
    int b[4];
    for (int64_t p0 = first; p0 < end; p0 += 256) {
        buckets_of(p0, b);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (b[i] >= 0) atomicAdd(&at[wave * buckets + b[i]], 1);
    }
    __syncthreads();
    // a thread has two buckets: all pairs of each, and those of earlier chunks
    const int b0 = 2 * (int)threadIdx.x;
    int all[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int bucket = b0 + i;
        if (bucket >= buckets) continue;
        if (chunks > 1 && !count_all) {
#pragma unroll 8
            for (int c = 0; c < chunks; ++c) {
                const int n = L.chunk_counts[(int64_t)c * buckets + bucket];
                all[i] += n;
                before[i] += c < (int)blockIdx.x ? n : 0;
            }
        } else {
#pragma unroll
            for (int w = 0; w < kListWaves; ++w) all[i] += at[w * buckets + bucket];
            before[i] = others[bucket];
            all[i] += others[bucket] + others[buckets + bucket];
        }
    }
    // exclusive sums over the buckets of the pairs and of the tiles of each width, by the wavefronts that have buckets
    const int scanning = buckets / 128 + 1;                  // (one more than the last bucket: the end)
    int sum[1 + kTileWidths] = {}, mine[1 + kTileWidths] = {};
    if (wave < scanning) {
#pragma unroll
        for (int v = 0; v <= kTileWidths; ++v) {
            const int width = v ? kTileWidth[v ? v - 1 : 0] : 1;
            mine[v] = sum[v] = (all[0] + width - 1) / width + (all[1] + width - 1) / width;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            int o[1 + kTileWidths];
#pragma unroll
            for (int v = 0; v <= kTileWidths; ++v) o[v] = __shfl_up(sum[v], d);
#pragma unroll
            for (int v = 0; v <= kTileWidths; ++v) sum[v] += lane >= d ? o[v] : 0;
        }
        if (lane == 63) {
#pragma unroll
            for (int v = 0; v <= kTileWidths; ++v) wave_sum[wave][v] = sum[v];
        }
    }
    __syncthreads();
    if (wave < scanning) {
#pragma unroll
        for (int v = 0; v <= kTileWidths; ++v) {
            const int width = v ? kTileWidth[v ? v - 1 : 0] : 1;
            int start = sum[v] - mine[v];
            for (int w = 0; w < wave; ++w) start += wave_sum[w][v];
            if (b0 <= buckets) starts[v * (buckets + 1) + b0] = start;
            if (b0 + 1 <= buckets) starts[v * (buckets + 1) + b0 + 1] = start + (all[0] + width - 1) / width;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int bucket = b0 + i;
        if (bucket >= buckets) continue;
        int n[kListWaves], to = starts[bucket] + before[i];
#pragma unroll
        for (int w = 0; w < kListWaves; ++w) n[w] = at[w * buckets + bucket];
#pragma unroll
        for (int w = 0; w < kListWaves; ++w) {
            at[w * buckets + bucket] = to;
            to += n[w];
        }
    }
    if (blockIdx.x == 0) {
        for (int b = threadIdx.x; b <= buckets; b += kListThreads) L.offsets[b] = starts[b];
        if (threadIdx.x < kTileWidths) L.tile_count[threadIdx.x] = starts[(threadIdx.x + 1) * (buckets + 1) + buckets];
        for (int b = wave; b < buckets; b += kListWaves)
#pragma unroll
            for (int v = 1; v <= kTileWidths; ++v) {
                const int t0 = starts[v * (buckets + 1) + b], t1 = starts[v * (buckets + 1) + b + 1];
                for (int t = t0 + lane; t < t1; t += 64) {
                    const int first = starts[b] + (t - t0) * kTileWidth[v - 1];
                    L.tiles[v - 1][t] = make_int2(b << 16 | min(kTileWidth[v - 1], starts[b + 1] - first), first);
                }
            }
    }
    __syncthreads();
    const int bits = 32 - __clz(experts);                    // (experts is the bucket of the pairs without one)
    for (int64_t p0 = first; p0 < end; p0 += 256) {
        if (p0 > first || chunk > 256 * kListWaves) buckets_of(p0, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // the lanes with the same expert, by its bits
            uint64_t same = __ballot(b[i] >= 0);
            for (int bit = 0; bit < bits; ++bit) {
                const uint64_t set = __ballot(b[i] >> bit & 1);
                same &= b[i] >> bit & 1 ? set : ~set;
            }
            if (b[i] >= 0) L.order[at[wave * buckets + b[i]] + __popcll(same & ((1ull << lane) - 1))] = (int32_t)(p0 + i * 64 + lane);
            lanes_exchange();
            if (b[i] >= 0 && (same >> lane) == 1) at[wave * buckets + b[i]] += __popcll(same);        // the highest of them
            lanes_exchange();
        }
    }
}

__global__ __launch_bounds__(kListThreads) void lists_count_kernel(ListArgs a) { lists_count(a); }
__global__ __launch_bounds__(kListThreads) void lists_place_kernel(ListArgs a) { lists_place(a); }

// The first launch of the lists (COUNT: of two) and the quantisation of the rows that are multiplied next, which do not need each
// other, in one: the first `chunks` workgroups have the lists.
template <class T, bool STREAM, bool COUNT> __global__ __launch_bounds__(kListThreads) void mx_prepare_kernel(ListArgs a, QuantiseArgs q)
{
    if ((int)blockIdx.x >= a.chunks) quantise_units<T, STREAM>(blockIdx.x - (uint32_t)a.chunks, q);
    else if (COUNT) lists_count(a);
    else lists_place(a);
}

static size_t list_lds_bytes(int experts) { return ((size_t)kListWaves * (experts + 1) + (1 + kTileWidths) * ((size_t)experts + 2) + 2 * ((size_t)experts + 1)) * 4; }

static int32_t launch_place(const ListArgs &a, hipStream_t st)
{
    const size_t lds = list_lds_bytes(a.experts);
    static LdsLimit seen;
    if (lds > 32768)
        if (int32_t rc = allow_lds((const void *)lists_place_kernel, list_lds_bytes(CL_ROUTE_MAX_EXPERTS), seen)) return rc;
    hipLaunchKernelGGL(lists_place_kernel, dim3((unsigned)a.chunks), dim3(kListThreads), lds, st, a);
    MX_HIP_TRY(hipGetLastError());
    return CL_OK;
}

int32_t launch_expert_lists(const int32_t *experts_of, int32_t tokens, int32_t k, int32_t experts, const ExpertLists &L, const QuantiseRows *rows, hipStream_t st)
{
    const int pairs = tokens * k, chunk = (int)list_chunk(pairs), chunks = std::max(1, (int)(((int64_t)pairs + chunk - 1) / chunk));
    const bool count = pairs > kListAll;                     // in a launch of its own
    const ListArgs a{L, experts_of, pairs, chunk, chunks, experts};
    const size_t lds = list_lds_bytes(experts);
    const uint32_t per_row = rows ? (uint32_t)(row_blocks(rows->K) * (rows->type == CL_F32 ? 8 : 4)) : 0;
    if (rows && (lds > 32768 || rows->rows * per_row > 1 << 30)) {       // (more LDS would keep the quantising workgroups few)
        if (int32_t rc = launch_quantize(rows->X, rows->type, rows->stride, rows->rows, rows->K, rows->codes, rows->scales, st)) return rc;
        rows = nullptr;
    }
    if (rows) {
        const QuantiseArgs q{rows->X, rows->codes, rows->scales, rows->stride, make_div(per_row), (uint32_t)(rows->rows * per_row), rows->K};
        const unsigned wgs = (q.units + kListThreads * kUnits - 1) / (kListThreads * kUnits);
        const bool stream = past_caches(rows->rows * rows->K * (int64_t)type_bytes(rows->type));
        const int32_t rc = with_type(rows->type, [&](auto t) -> int32_t {
            using T = decltype(t);
            auto kernel = count ? (stream ? mx_prepare_kernel<T, true, true> : mx_prepare_kernel<T, false, true>)
                                     : (stream ? mx_prepare_kernel<T, true, false> : mx_prepare_kernel<T, false, false>);
            hipLaunchKernelGGL(kernel, dim3((unsigned)chunks + wgs), dim3(kListThreads), lds, st, a, q);
            MX_HIP_TRY(hipGetLastError());
            return CL_OK;
        });
        if (rc) return rc;
    } else if (count) {
        hipLaunchKernelGGL(lists_count_kernel, dim3((unsigned)chunks), dim3(kListThreads), ((size_t)experts + 1) * 4, st, a);
        MX_HIP_TRY(hipGetLastError());
    }
    return rows && !count ? (int32_t)CL_OK : launch_place(a, st);
}

}  // namespace mx
}  // namespace cl

using namespace cl;
using namespace cl::mx;

extern "C" int32_t cl_route_experts(const void *d_logits, int32_t type, int64_t x_stride, const float *d_bias, int32_t tokens, const cl_route_desc *desc,
                                    int32_t *d_experts, float *d_weights, void *stream)
{
    if (!desc) return fail(CL_EINVAL, "null pointer");
    const cl_route_desc &d = *desc;
    if (!known_type(type)) return fail(CL_EINVAL, "unknown element type %d", (int)type);
    if (tokens < 0 || d.experts < 1) return fail(CL_EINVAL, "bad logits: %d tokens, %d experts", (int)tokens, (int)d.experts);
    if (d.experts > CL_ROUTE_MAX_EXPERTS) return fail(CL_EUNSUPPORTED, "%d experts: at most %d", (int)d.experts, CL_ROUTE_MAX_EXPERTS);
    if (d.score != CL_SCORE_SOFTMAX && d.score != CL_SCORE_SIGMOID) return fail(CL_EINVAL, "unknown score %d", (int)d.score);
    if (d.group_score != CL_GROUP_MAX && d.group_score != CL_GROUP_TOP2) return fail(CL_EINVAL, "unknown group score %d", (int)d.group_score);
    if (d.groups < 1 || d.experts % d.groups) return fail(CL_EINVAL, "%d groups do not divide %d experts", (int)d.groups, (int)d.experts);
    if (d.groups > CL_ROUTE_MAX_GROUPS) return fail(CL_EUNSUPPORTED, "%d groups: at most %d", (int)d.groups, CL_ROUTE_MAX_GROUPS);
    if (d.groups_kept < 1 || d.groups_kept > d.groups) return fail(CL_EINVAL, "%d of %d groups kept", (int)d.groups_kept, (int)d.groups);
    if (d.k < 1 || d.k > d.experts / d.groups * d.groups_kept) return fail(CL_EINVAL, "%d of the %d experts of the kept groups", (int)d.k, (int)(d.experts / d.groups * d.groups_kept));
    if (d.k > CL_ROUTE_MAX_K) return fail(CL_EUNSUPPORTED, "%d experts for a token: at most %d", (int)d.k, CL_ROUTE_MAX_K);
    if (tokens == 0) return CL_OK;
    if (!d_logits || !d_experts || !d_weights) return fail(CL_EINVAL, "null pointer");
    if (tokens > 1 && x_stride < d.experts) return fail(CL_EINVAL, "rows of %d logits overlap at a stride of %lld", (int)d.experts, (long long)x_stride);
    RouteArgs a{d_logits, x_stride, d_bias, d_experts, d_weights, tokens, d.experts, d.k, d.groups, d.groups_kept, d.group_score == CL_GROUP_TOP2,
                d.score == CL_SCORE_SIGMOID, d.renormalize, d.scale};
    const int32_t rc = with_type(type, [&](auto t) -> int32_t {
        using T = decltype(t);
        hipStream_t st = (hipStream_t)stream;
        // sixteen lanes to a token while experts, choices and groups are few enough for them
        if (d.experts <= 512 && d.k <= 16 && d.groups <= 16) {
            const int C = d.experts <= 64 ? 4 : d.experts <= 128 ? 8 : d.experts <= 256 ? 16 : 32, size = d.experts / d.groups;
            const int lanes = size % C == 0 && (size / C & (size / C - 1)) == 0 ? size / C : 0;
            if (C == 4) return launch_route_rows<T, 4>(a, lanes, st);
            if (C == 8) return launch_route_rows<T, 8>(a, lanes, st);
            if (C == 16) return launch_route_rows<T, 16>(a, lanes, st);
            return launch_route_rows<T, 32>(a, lanes, st);
        }
        if (d.experts <= 256) return launch_route<T, 64, 4>(a, st);
        return launch_route<T, 64, 16>(a, st);
    });
    if (rc) return rc;
    clear_error();
    return CL_OK;
}

static int32_t check_lists(int32_t tokens, int32_t k, int32_t experts)
{
    if (tokens < 0 || k < 1 || experts < 1) return fail(CL_EINVAL, "bad lists: %d tokens, %d of %d experts", (int)tokens, (int)k, (int)experts);
    if (experts > CL_ROUTE_MAX_EXPERTS) return fail(CL_EUNSUPPORTED, "%d experts: at most %d", (int)experts, CL_ROUTE_MAX_EXPERTS);
    if ((int64_t)tokens * k > CL_EXPERTS_MAX_PAIRS) return fail(CL_EUNSUPPORTED, "more than 2^30 pairs of token and expert");
    return CL_OK;
}

extern "C" int32_t cl_expert_lists_bytes(int32_t tokens, int32_t k, int32_t experts, size_t *out)
{
    if (!out) return fail(CL_EINVAL, "null pointer");
    if (int32_t rc = check_lists(tokens, k, experts)) return rc;
    *out = expert_lists_at(nullptr, tokens, k, experts).bytes;
    clear_error();
    return CL_OK;
}

extern "C" int32_t cl_expert_lists(const int32_t *d_experts, int32_t tokens, int32_t k, int32_t experts, void *d_lists, size_t lists_bytes, void *stream)
{
    if (int32_t rc = check_lists(tokens, k, experts)) return rc;
    const ExpertLists L = expert_lists_at(d_lists, tokens, k, experts);
    if (!d_lists || (tokens && !d_experts)) return fail(CL_EINVAL, "null pointer");
    if (!aligned(d_lists, 256)) return fail(CL_EINVAL, "lists must be 256-byte aligned");
    if (lists_bytes < L.bytes) return fail(CL_EINVAL, "lists need %zu bytes, got %zu", L.bytes, lists_bytes);
    if (int32_t rc = launch_expert_lists(d_experts, tokens, k, experts, L, nullptr, (hipStream_t)stream)) return rc;
    clear_error();
    return CL_OK;
}
