// The choice of experts for tokens, and the lists of tokens that each expert is given.
#include <algorithm>

#include "mx_common.hpp"

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
        const float sum = over_lanes<L>(weight, [](float p, float q) { return p + q; });
        weight = sum > 0.0f ? weight / sum : 0.0f;
    }
    if (live && sub < a.k) {
        a.experts_out[(int64_t)token * a.k + sub] = chosen;
        a.weights_out[(int64_t)token * a.k + sub] = weight * a.scale;
    }
}

template <class T, int L, int C> static int32_t launch_route(const RouteArgs &a, hipStream_t st)
{
    const int per = 256 / L;
    hipLaunchKernelGGL((route_kernel<T, L, C>), dim3((unsigned)((a.tokens + per - 1) / per)), dim3(256), 0, st, a);
    MX_HIP_TRY(hipGetLastError());
    return CL_OK;
}

// ------------------------------------------------------------------------- //
// the lists: a stable counting sort of the pairs (token, j) by their expert, pairs without one last
// ------------------------------------------------------------------------- //
// Pairs of one workgroup: a multiple of 4096 that makes at most 256 workgroups, each of which adds the others' counts up.
constexpr int kListThreads = 1024, kListWaves = kListThreads / 64;
static int64_t list_chunk(int64_t pairs) { return std::max<int64_t>(1, (pairs + 4096 * 256 - 1) / (4096 * 256)) * 4096; }

ExpertLists expert_lists_at(void *base, int32_t tokens, int32_t k, int32_t experts)
{
    ExpertLists L;
    const int64_t pairs = (int64_t)tokens * k, chunk = list_chunk(pairs), chunks = (pairs + chunk - 1) / chunk;
    size_t at = 0;
    auto take = [&](size_t bytes) { char *p = (char *)base + at; at += round_up(bytes, 256); return p; };
    L.offsets = (int32_t *)take(((size_t)experts + 2) * 4);
    L.tile_count = (int32_t *)take(kTileWidths * 4);
    L.order = (int32_t *)take((size_t)pairs * 4);
    for (int w = 0; w < kTileWidths; ++w) {
        L.max_tiles[w] = pairs / kTileWidth[w] + std::min<int64_t>(pairs, (int64_t)experts + 1);
        L.tiles[w] = (int2 *)take((size_t)L.max_tiles[w] * sizeof(int2));
    }
    L.chunk_counts = (int32_t *)take(chunks > 1 ? (size_t)chunks * ((size_t)experts + 1) * 4 : 0);
    L.bytes = at;
    return L;
}

__device__ __forceinline__ int bucket_of(int e, int experts) { return e >= 0 && e < experts ? e : experts; }

__global__ __launch_bounds__(kListThreads) void lists_count_kernel(const int32_t *__restrict__ experts_of, int pairs, int chunk, int experts, int32_t *counts)
{
    __shared__ int32_t n[CL_ROUTE_MAX_EXPERTS + 1];
    for (int b = threadIdx.x; b <= experts; b += kListThreads) n[b] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * chunk, p1 = min((int64_t)pairs, p0 + chunk);
    for (int64_t p = p0 + threadIdx.x; p < p1; p += kListThreads) atomicAdd(&n[bucket_of(experts_of[p], experts)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b <= experts; b += kListThreads) counts[(int64_t)blockIdx.x * (experts + 1) + b] = n[b];
}

// Every workgroup finds where its own pairs of each expert go (the first: also the tiles), and puts them there.  Wavefront w has the
// w-th sixteenth of the chunk.
__global__ __launch_bounds__(kListThreads) void lists_place_kernel(ExpertLists L, const int32_t *__restrict__ experts_of, int pairs, int chunk, int chunks, int experts)
{
    extern __shared__ int32_t list_lds[];
    const int buckets = experts + 1, wave = (int)threadIdx.x / 64, lane = (int)threadIdx.x & 63;
    int32_t *at = list_lds;                                  // [wavefront][bucket]: how many, then where the next goes
    int32_t *starts = at + kListWaves * buckets;             // [1 + kTileWidths][bucket + 1]: first pair, first tile of each width
    __shared__ int32_t wave_sum[kListWaves][1 + kTileWidths];
    for (int i = threadIdx.x; i < kListWaves * buckets; i += kListThreads) at[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * chunk + (int64_t)wave * (chunk / kListWaves);
    const int64_t end = min((int64_t)pairs, first + chunk / kListWaves);
    for (int64_t p = first + lane; p < end; p += 64) atomicAdd(&at[wave * buckets + bucket_of(experts_of[p], experts)], 1);
    __syncthreads();
    // a thread has two buckets: all pairs of each, and those of earlier chunks
    const int b0 = 2 * (int)threadIdx.x;
    int all[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int b = b0 + i;
        if (b >= buckets) continue;
        if (chunks > 1) {
            for (int c = 0; c < chunks; ++c) {
                const int n = L.chunk_counts[(int64_t)c * buckets + b];
                all[i] += n;
                before[i] += c < (int)blockIdx.x ? n : 0;
            }
        } else {
            for (int w = 0; w < kListWaves; ++w) all[i] += at[w * buckets + b];
        }
    }
    // exclusive sums over the buckets of the pairs and of the tiles of each width
    int sum[1 + kTileWidths], mine[1 + kTileWidths];
#pragma unroll
    for (int v = 0; v <= kTileWidths; ++v) {
        const int width = v ? kTileWidth[v ? v - 1 : 0] : 1;
        mine[v] = (all[0] + width - 1) / width + (all[1] + width - 1) / width;
        sum[v] = mine[v];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(sum[v], d);
            sum[v] += lane >= d ? o : 0;
        }
        if (lane == 63) wave_sum[wave][v] = sum[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v <= kTileWidths; ++v) {
        const int width = v ? kTileWidth[v ? v - 1 : 0] : 1;
        int start = sum[v] - mine[v];
        for (int w = 0; w < wave; ++w) start += wave_sum[w][v];
        if (b0 <= buckets) starts[v * (buckets + 1) + b0] = start;
        if (b0 + 1 <= buckets) starts[v * (buckets + 1) + b0 + 1] = start + (all[0] + width - 1) / width;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int b = b0 + i;
        if (b >= buckets) continue;
        int to = starts[b] + before[i];
        for (int w = 0; w < kListWaves; ++w) {
            const int n = at[w * buckets + b];
            at[w * buckets + b] = to;
            to += n;
        }
    }
    if (blockIdx.x == 0) {
        for (int b = threadIdx.x; b <= buckets; b += kListThreads) L.offsets[b] = starts[b];
        if (threadIdx.x < kTileWidths) L.tile_count[threadIdx.x] = starts[(threadIdx.x + 1) * (buckets + 1) + buckets];
        for (int b = wave; b < buckets; b += kListWaves)
#pragma unroll
            for (int v = 1; v <= kTileWidths; ++v) {
                const int t0 = starts[v * (buckets + 1) + b], t1 = starts[v * (buckets + 1) + b + 1];
                for (int t = t0 + lane; t < t1; t += 64) L.tiles[v - 1][t] = make_int2(b, starts[b] + (t - t0) * kTileWidth[v - 1]);
            }
    }
    __syncthreads();
    for (int64_t p0 = first; p0 < end; p0 += 64) {
        const int64_t p = p0 + lane;
        const int b = p < end ? bucket_of(experts_of[p], experts) : -1;
        // the lanes with the same expert, by its bits
        uint64_t same = __ballot(b >= 0);
        for (int bit = 0; bit < 11; ++bit) {
            const uint64_t set = __ballot(b >> bit & 1);
            same &= b >> bit & 1 ? set : ~set;
        }
        if (b >= 0) L.order[at[wave * buckets + b] + __popcll(same & ((1ull << lane) - 1))] = (int32_t)p;
        __builtin_amdgcn_wave_barrier();
        if (b >= 0 && (same >> lane) == 1) at[wave * buckets + b] += __popcll(same);      // the highest of them
        __builtin_amdgcn_wave_barrier();
    }
}

int32_t launch_expert_lists(const int32_t *experts_of, int32_t tokens, int32_t k, int32_t experts, const ExpertLists &L, hipStream_t st)
{
    const int pairs = tokens * k, chunk = (int)list_chunk(pairs), chunks = std::max(1, (int)(((int64_t)pairs + chunk - 1) / chunk));
    if (chunks > 1) {
        hipLaunchKernelGGL(lists_count_kernel, dim3((unsigned)chunks), dim3(kListThreads), 0, st, experts_of, pairs, chunk, experts, L.chunk_counts);
        MX_HIP_TRY(hipGetLastError());
    }
    const size_t lds = ((size_t)kListWaves * (experts + 1) + (1 + kTileWidths) * ((size_t)experts + 2)) * 4;
    static LdsLimit seen;
    if (lds > 32768)
        if (int32_t rc = allow_lds((const void *)lists_place_kernel, ((size_t)kListWaves * (CL_ROUTE_MAX_EXPERTS + 1) + (1 + kTileWidths) * (CL_ROUTE_MAX_EXPERTS + 2)) * 4, seen)) return rc;
    hipLaunchKernelGGL(lists_place_kernel, dim3((unsigned)chunks), dim3(kListThreads), lds, st, L, experts_of, pairs, chunk, chunks, experts);
    MX_HIP_TRY(hipGetLastError());
    return CL_OK;
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
        if (d.experts <= 64 && d.k <= 16) return launch_route<T, 16, 4>(a, st);
        if (d.experts <= 128) return launch_route<T, 32, 4>(a, st);
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
    if (int32_t rc = launch_expert_lists(d_experts, tokens, k, experts, L, (hipStream_t)stream)) return rc;
    clear_error();
    return CL_OK;
}
