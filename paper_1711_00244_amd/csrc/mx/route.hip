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
ExpertLists expert_lists_at(void *base, int32_t tokens, int32_t k, int32_t experts)
{
    ExpertLists L;
    const int64_t pairs = (int64_t)tokens * k, chunks = (pairs + kListChunk - 1) / kListChunk;
    size_t at = 0;
    auto take = [&](size_t bytes) { char *p = (char *)base + at; at += round_up(bytes, 256); return p; };
    L.offsets = (int32_t *)take(((size_t)experts + 2) * 4);
    L.tile_count = (int32_t *)take(kTileWidths * 4);
    L.order = (int32_t *)take((size_t)pairs * 4);
    for (int w = 0; w < kTileWidths; ++w) {
        L.max_tiles[w] = pairs / kTileWidth[w] + std::min<int64_t>(pairs, (int64_t)experts + 1);
        L.tiles[w] = (int2 *)take((size_t)L.max_tiles[w] * sizeof(int2));
    }
    L.chunk_counts = (int32_t *)take((size_t)chunks * ((size_t)experts + 1) * 4);
    L.bytes = at;
    return L;
}

__device__ __forceinline__ int bucket_of(int e, int experts) { return e >= 0 && e < experts ? e : experts; }

__global__ __launch_bounds__(256) void lists_count_kernel(const int32_t *__restrict__ experts_of, int pairs, int experts, int32_t *counts)
{
    __shared__ int32_t n[CL_ROUTE_MAX_EXPERTS + 1];
    for (int b = threadIdx.x; b <= experts; b += 256) n[b] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * kListChunk;
    for (int i = threadIdx.x; i < kListChunk; i += 256)
        if (p0 + i < pairs) atomicAdd(&n[bucket_of(experts_of[p0 + i], experts)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b <= experts; b += 256) counts[(int64_t)blockIdx.x * (experts + 1) + b] = n[b];
}

// Exclusive sums of v over 1024 threads, and the total.
__device__ __forceinline__ int exclusive_sum(int v, int *s, int &total)
{
    const int t = threadIdx.x;
    __syncthreads();
    s[t] = v;
    __syncthreads();
    for (int d = 1; d < 1024; d *= 2) {
        const int o = t >= d ? s[t - d] : 0;
        __syncthreads();
        s[t] += o;
        __syncthreads();
    }
    total = s[1023];
    return s[t] - v;
}

// One workgroup: where each expert's pairs start, how many of them the chunks before a chunk have, and the tiles.  A thread
// takes two buckets (experts + 1 <= 2048).
__global__ __launch_bounds__(1024) void lists_scan_kernel(ExpertLists L, int chunks, int experts)
{
    __shared__ int s[1024];
    const int b0 = 2 * (int)threadIdx.x;
    int n[2] = {0, 0};
    for (int i = 0; i < 2; ++i)
        if (b0 + i <= experts)
            for (int c = 0; c < chunks; ++c) {
                int32_t *p = L.chunk_counts + (int64_t)c * (experts + 1) + b0 + i;
                const int v = *p;
                *p = n[i];
                n[i] += v;
            }
    int total;
    int start[2];
    start[0] = exclusive_sum(n[0] + n[1], s, total);
    start[1] = start[0] + n[0];
    for (int i = 0; i < 2; ++i)
        if (b0 + i <= experts) L.offsets[b0 + i] = start[i];
    if (threadIdx.x == 0) L.offsets[experts + 1] = total;
    for (int w = 0; w < kTileWidths; ++w) {
        const int width = kTileWidth[w];
        const int t0 = (n[0] + width - 1) / width, t1 = (n[1] + width - 1) / width;
        int at = exclusive_sum(t0 + t1, s, total);
        if (threadIdx.x == 0) L.tile_count[w] = total;
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < (i ? t1 : t0); ++j) L.tiles[w][at++] = make_int2(b0 + i, start[i] + j * width);
    }
}

__global__ __launch_bounds__(256) void lists_scatter_kernel(ExpertLists L, const int32_t *__restrict__ experts_of, int pairs, int experts)
{
    __shared__ int32_t at[4][CL_ROUTE_MAX_EXPERTS + 1];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    for (int b = threadIdx.x; b < 4 * (CL_ROUTE_MAX_EXPERTS + 1); b += 256) at[0][b] = 0;
    __syncthreads();
    // a wavefront has a quarter of the chunk, 64 pairs at a time
    const int64_t p0 = (int64_t)blockIdx.x * kListChunk + wave * (kListChunk / 4) + lane;
    int bucket[kListChunk / 256];
    for (int i = 0; i < kListChunk / 256; ++i) {
        const int64_t p = p0 + i * 64;
        bucket[i] = p < pairs ? bucket_of(experts_of[p], experts) : -1;
        if (bucket[i] >= 0) atomicAdd(&at[wave][bucket[i]], 1);
    }
    __syncthreads();
    for (int b = threadIdx.x; b <= experts; b += 256) {
        int sum = L.offsets[b] + L.chunk_counts[(int64_t)blockIdx.x * (experts + 1) + b];
        for (int w = 0; w < 4; ++w) {
            const int n = at[w][b];
            at[w][b] = sum;
            sum += n;
        }
    }
    __syncthreads();
    for (int i = 0; i < kListChunk / 256; ++i) {
        const int b = bucket[i];
        // the lanes with the same expert, by its bits
        uint64_t same = __ballot(b >= 0);
        for (int bit = 0; bit < 11; ++bit) {
            const uint64_t set = __ballot(b >> bit & 1);
            same &= b >> bit & 1 ? set : ~set;
        }
        if (b >= 0) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const int to = at[wave][b] + rank;
            L.order[to] = (int32_t)(p0 + i * 64);
        }
        __builtin_amdgcn_wave_barrier();
        if (b >= 0 && (same >> lane) == 1) at[wave][b] += __popcll(same);        // the highest of them
        __builtin_amdgcn_wave_barrier();
    }
}

int32_t launch_expert_lists(const int32_t *experts_of, int32_t tokens, int32_t k, int32_t experts, const ExpertLists &L, hipStream_t st)
{
    const int pairs = tokens * k, chunks = (pairs + kListChunk - 1) / kListChunk;
    if (chunks) {
        hipLaunchKernelGGL(lists_count_kernel, dim3((unsigned)chunks), dim3(256), 0, st, experts_of, pairs, experts, L.chunk_counts);
        MX_HIP_TRY(hipGetLastError());
    }
    hipLaunchKernelGGL(lists_scan_kernel, dim3(1), dim3(1024), 0, st, L, chunks, experts);
    MX_HIP_TRY(hipGetLastError());
    if (chunks) {
        hipLaunchKernelGGL(lists_scatter_kernel, dim3((unsigned)chunks), dim3(256), 0, st, L, experts_of, pairs, experts);
        MX_HIP_TRY(hipGetLastError());
    }
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
    if ((int64_t)tokens * k > (int64_t)INT32_MAX - kListChunk) return fail(CL_EUNSUPPORTED, "more than 2^31 pairs of token and expert");
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
