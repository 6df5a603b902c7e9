// Routing of requests to experts: scores, choice, weights, the order of the experts' rows, and the
// gradient of the weights.
//
//   s = softmax(x) or 1 / (1 + exp(-x));  c = s + bias;  groups of experts by the sum of their best c;
//   the top_k best c of the kept groups;  weight = scale * s / (sum of the chosen s + 1e-20)
//
// A choice is a comparison of floats, so it is made on order-preserving 32-bit keys (key 0: not to
// be chosen) with the lowest index winning among equal keys.  The order of the rows is a counting
// sort by expert in three launches that share one partition of the tokens into runs, one per CTA:
// count (in the routing kernel), prefix sums, place.  No atomics on floats, nothing that depends
// on the order of execution.
#include <type_traits>

#include "operators.cuh"

namespace gs {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr float kLargest = 3.402823466e38f;
constexpr float kSumFloor = 1e-20f;
constexpr int kRouteThreads = 256;

// Order-preserving key of a float that is no NaN; 0 is below all of them.
__device__ __forceinline__ unsigned key_of(float v) {
    const unsigned b = __float_as_uint(v);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

struct RouterParams {
    int n_experts, top_k, n_groups, top_groups, group_top, group_size;
    bool sigmoid, renormalise;
    float scale;
};

RouterParams params_of(const gs_expert_router &r) {
    return {r.n_experts, r.top_k, r.n_groups, r.top_groups, r.group_top, r.n_experts / r.n_groups,
            r.score == GS_SCORE_SIGMOID, r.renormalise != 0, r.scale};
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// A row's logits, expert i * 32 + lane in element i; -infinity where there is none to choose.
template <typename T, int V>
__device__ __forceinline__ bool load_row(const T *__restrict__ row, int n_experts, int lane, float (&x)[V]) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        float v = e < n_experts ? to_float(row[e]) : -INFINITY;
        if (v != v) { nan = true; v = -INFINITY; }
        x[i] = fminf(v, kLargest);
    }
    return nan;
}

// Scores in place of logits; 0 for what cannot be chosen.
template <int V>
__device__ __forceinline__ void scores_of(float (&x)[V], bool sigmoid) {
    if (sigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = x[i] == -INFINITY ? 0.f : 1.f / (1.f + expf(-x[i]));
        return;
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
    top = warp_max(top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) { x[i] = x[i] == -INFINITY ? 0.f : expf(x[i] - top); sum += x[i]; }
    sum = warp_sum(sum);
    const float inv_safe = sum > 0.f ? sum : 1.f;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = x[i] / inv_safe;
}

// Best key of the warp and its lowest expert; removes it from its lane.
template <int V>
__device__ __forceinline__ unsigned take_best(unsigned (&key)[V], int lane, int lo, int hi, int *expert) {
    unsigned best = 0;
    int at = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        if (e >= lo && e < hi && key[i] > best) { best = key[i]; at = e; }
    }
    const unsigned top = __reduce_max_sync(kFull, best);
    const unsigned who = __reduce_min_sync(kFull, best == top ? (unsigned)at : 0x7FFFFFFFu);
    *expert = top ? (int)who : -1;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (top && i * 32 + lane == (int)who) key[i] = 0;
    return top;
}

__device__ __forceinline__ float value_of(unsigned key) {
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// One warp per row, V * 32 experts at most.
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads)
route_rows_kernel(const T *__restrict__ logits, int64_t n_tokens, int64_t ld, const float *__restrict__ bias,
                  RouterParams p, int rows_per_cta, int32_t *__restrict__ out_expert, float *__restrict__ out_weight,
                  int *__restrict__ counts, unsigned *__restrict__ status)
{
    __shared__ int cta_count[GS_MAX_EXPERTS];
    dependent_begin();
    for (int e = threadIdx.x; e < p.n_experts; e += kRouteThreads) cta_count[e] = 0;
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = (int64_t)blockIdx.x * rows_per_cta;
    const int64_t last = min(first + rows_per_cta, n_tokens);
    float b[V];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        b[i] = bias && e < p.n_experts ? fminf(bias[e], kLargest) : 0.f;
        if (b[i] != b[i]) { nan = true; b[i] = -INFINITY; }
    }
    for (int64_t n = first + warp; n < last; n += kRouteThreads / 32) {
        float s[V];
        unsigned key[V];
        nan |= load_row<T, V>(logits + n * ld, p.n_experts, lane, s);
        bool on[V];
#pragma unroll
        for (int i = 0; i < V; ++i) on[i] = s[i] != -INFINITY && b[i] != -INFINITY;
        scores_of<V>(s, p.sigmoid);
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = on[i] ? key_of(s[i] + b[i]) : 0u;
        if (p.n_groups > 1) {
            unsigned mine = 0;                       // lane g: key of group g's score
            for (int g = 0; g < p.n_groups; ++g) {
                unsigned left[V];
#pragma unroll
                for (int i = 0; i < V; ++i) left[i] = key[i];
                int at;
                const int lo = g * p.group_size, hi = lo + p.group_size;
                const unsigned k1 = take_best<V>(left, lane, lo, hi, &at);
                unsigned score = k1;
                if (p.group_top == 2 && k1) {
                    const unsigned k2 = take_best<V>(left, lane, lo, hi, &at);
                    if (k2) score = key_of(value_of(k1) + value_of(k2));
                }
                if (lane == g) mine = score;
            }
            int before = 0;                          // groups that rank before this lane's
            for (int g = 0; g < p.n_groups; ++g) {
                const unsigned other = __shfl_sync(kFull, mine, g);
                before += other > mine || (other == mine && g < lane);
            }
            const unsigned kept = __ballot_sync(kFull, lane < p.n_groups && before < p.top_groups);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = i * 32 + lane;
                if (e < p.n_experts && !((kept >> (e / p.group_size)) & 1)) key[i] = 0;
            }
        }
        int my_expert = -1;                          // lane j: slot j
        float my_score = 0.f;
        for (int j = 0; j < p.top_k; ++j) {
            int e;
            take_best<V>(key, lane, 0, p.n_experts, &e);
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) if (e == i * 32 + lane) v = s[i];
            v = __shfl_sync(kFull, v, e & 31);
            if (lane == j && e >= 0) { my_expert = e; my_score = v; }
        }
        const float total = warp_sum(my_score) + kSumFloor;
        if (lane < p.top_k) {
            const float w = p.renormalise ? p.scale * (my_score / total) : p.scale * my_score;
            out_expert[n * p.top_k + lane] = my_expert;
            out_weight[n * p.top_k + lane] = w;
            if (counts && my_expert >= 0) atomicAdd(&cta_count[my_expert], 1);
        }
    }
    if (nan) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
    if (!counts) return;
    __syncthreads();
    for (int e = threadIdx.x; e < p.n_experts; e += kRouteThreads)
        counts[e * kMaxRouteCtas + blockIdx.x] = cta_count[e];
}

// Per expert (one warp each): counts per CTA become the rows before that CTA's, and their total.
__global__ void __launch_bounds__(kRouteThreads)
route_prefix_kernel(int *__restrict__ counts, int n_experts, int n_ctas)
{
    dependent_begin();
    const int e = blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (e >= n_experts) return;
    int *c = counts + e * kMaxRouteCtas, before = 0;
    for (int base = 0; base < n_ctas; base += 32) {
        const int i = base + lane;
        const int own = i < n_ctas ? c[i] : 0;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFull, sum, o);
            if (lane >= o) sum += up;
        }
        if (i < n_ctas) c[i] = before + sum - own;
        before += __shfl_sync(kFull, sum, 31);
    }
    if (lane == 0) counts[GS_MAX_EXPERTS * kMaxRouteCtas + e] = before;
}

// Places every slot of the CTA's tokens: each warp takes a stretch of them, first counts its
// experts, then (knowing what the warps before it hold) hands out rows in order.
__global__ void __launch_bounds__(kRouteThreads)
route_place_kernel(const int32_t *__restrict__ expert, int64_t n_slots, int top_k, int slots_per_cta, int n_experts,
                   const int *__restrict__ counts, int32_t *__restrict__ offsets, int32_t *__restrict__ row_token,
                   int32_t *__restrict__ token_row)
{
    constexpr int kWarps = kRouteThreads / 32;
    extern __shared__ int place_smem[];
    int *cnt = place_smem;                           // [kWarps][n_experts]
    int *start = place_smem + kWarps * n_experts;    // [n_experts + 1]
    dependent_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int *total = counts + GS_MAX_EXPERTS * kMaxRouteCtas;
    for (int i = threadIdx.x; i < kWarps * n_experts; i += kRouteThreads) cnt[i] = 0;
    if (warp == 0) {
        int before = 0;
        for (int base = 0; base < n_experts; base += 32) {
            const int e = base + lane, own = e < n_experts ? total[e] : 0;
            int sum = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(kFull, sum, o);
                if (lane >= o) sum += up;
            }
            if (e < n_experts) start[e] = before + sum - own;
            before += __shfl_sync(kFull, sum, 31);
        }
        if (lane == 0) start[n_experts] = before;
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= n_experts; e += kRouteThreads) offsets[e] = start[e];
    const int64_t cta_first = (int64_t)blockIdx.x * slots_per_cta, cta_last = min(cta_first + slots_per_cta, n_slots);
    const int per_warp = ((slots_per_cta + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int64_t first = cta_first + (int64_t)warp * per_warp, last = min(first + per_warp, cta_last);
    int *mine = cnt + warp * n_experts;
    for (int64_t i = first + lane; i - lane < last; i += 32) {
        const int e = i < last ? expert[i] : -1;
        const unsigned same = __match_any_sync(kFull, e);
        if (e >= 0 && __ffs(same) - 1 == lane) mine[e] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n_experts; e += kRouteThreads) {
        int row = start[e] + counts[e * kMaxRouteCtas + blockIdx.x];
        for (int w = 0; w < kWarps; ++w) { const int c = cnt[w * n_experts + e]; cnt[w * n_experts + e] = row; row += c; }
    }
    __syncthreads();
    for (int64_t i = first + lane; i - lane < last; i += 32) {
        const int e = i < last ? expert[i] : -1;
        const unsigned same = __match_any_sync(kFull, e);
        int row = -1;
        if (e >= 0) row = mine[e] + __popc(same & ((1u << lane) - 1));
        __syncwarp();
        if (e >= 0 && __ffs(same) - 1 == lane) mine[e] += __popc(same);
        __syncwarp();
        if (i < last) {
            token_row[i] = row;
            if (row >= 0) row_token[row] = (int)((unsigned)i / (unsigned)top_k);
        }
    }
    // rows that no slot took
    const int64_t step = (int64_t)gridDim.x * kRouteThreads;
    for (int64_t i = start[n_experts] + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; i < n_slots; i += step)
        row_token[i] = -1;
}

// Gradient of the weights, one warp per row.  With q the chosen scores, t = sum q + 1e-20:
//   renormalised: dq_j = scale * (dw_j - sum_i dw_i q_i / t) / t;   else dq_j = scale * dw_j
//   sigmoid: dx = dq * s (1 - s);   softmax: dx = s * (dq - sum_j dq_j s_j)
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads)
route_rows_backward_kernel(const T *__restrict__ logits, int64_t n_tokens, int64_t ld, RouterParams p,
                           const int32_t *__restrict__ expert, const float *__restrict__ d_weight,
                           T *__restrict__ d_logits, int64_t ld_d, unsigned *__restrict__ status)
{
    dependent_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    bool bad = false;
    for (int64_t n = (int64_t)blockIdx.x * (kRouteThreads / 32) + warp; n < n_tokens; n += (int64_t)gridDim.x * (kRouteThreads / 32)) {
        float s[V];
        bad |= load_row<T, V>(logits + n * ld, p.n_experts, lane, s);
        scores_of<V>(s, p.sigmoid);
        int e = lane < p.top_k ? expert[n * p.top_k + lane] : -1;
        if (e < -1 || e >= p.n_experts) { bad = true; e = -1; }
        const float dw = e >= 0 ? d_weight[n * p.top_k + lane] : 0.f;
        float q = 0.f;                               // lane j: the score of slot j
        for (int j = 0; j < p.top_k; ++j) {
            const int ej = __shfl_sync(kFull, e, j);
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) if (ej == i * 32 + lane) v = s[i];
            v = __shfl_sync(kFull, v, ej & 31);
            if (lane == j && ej >= 0) q = v;
        }
        float dq = p.scale * dw;
        if (p.renormalise) {
            const float t = warp_sum(q) + kSumFloor;
            const float mean = warp_sum(dw * (q / t));
            dq = e >= 0 ? p.scale * ((dw - mean) / t) : 0.f;
        }
        float ds[V];
#pragma unroll
        for (int i = 0; i < V; ++i) ds[i] = 0.f;
        for (int j = 0; j < p.top_k; ++j) {
            const int ej = __shfl_sync(kFull, e, j);
            const float v = __shfl_sync(kFull, dq, j);
#pragma unroll
            for (int i = 0; i < V; ++i) if (ej == i * 32 + lane) ds[i] += v;
        }
        const float mean = p.sigmoid ? 0.f : warp_sum(dq * q);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int k = i * 32 + lane;
            const float dx = p.sigmoid ? ds[i] * s[i] * (1.f - s[i]) : s[i] * (ds[i] - mean);
            if (k < p.n_experts) d_logits[n * ld_d + k] = from_float<T>(dx);
        }
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename F> cudaError_t by_width(int n_experts, F &&f) {
    if (n_experts <= 32) return f(std::integral_constant<int, 1>());
    if (n_experts <= 64) return f(std::integral_constant<int, 2>());
    if (n_experts <= 128) return f(std::integral_constant<int, 4>());
    if (n_experts <= 256) return f(std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 16>());
}

template <typename T>
cudaError_t route_rows(gs_ctx *ctx, const ExpertRouteArgs &a, int n_ctas, int rows_per_cta, cudaStream_t st) {
    int *counts = a.offsets ? operator_scratch(ctx).expert_counts : nullptr;
    return by_width(a.r.n_experts, [&](auto v) {
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        return launch_dependent(route_rows_kernel<T, decltype(v)::value>, dim3(n_ctas), dim3(kRouteThreads), 0, st,
                                (const T *)a.logits, a.n_tokens, a.ld, a.bias, params_of(a.r), rows_per_cta,
                                a.expert, a.weight, counts, ctx->s.status);
    });
}

template <typename T>
cudaError_t route_rows_backward(gs_ctx *ctx, const ExpertRouteGradArgs &a, cudaStream_t st) {
    const int64_t want = (a.n_tokens + kRouteThreads / 32 - 1) / (kRouteThreads / 32);
    const int n_ctas = (int)(want < 16 * ctx->n_sm ? want : 16 * ctx->n_sm);
    return by_width(a.r.n_experts, [&](auto v) {
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        return launch_dependent(route_rows_backward_kernel<T, decltype(v)::value>, dim3(n_ctas), dim3(kRouteThreads), 0, st,
                                (const T *)a.logits, a.n_tokens, a.ld, params_of(a.r), a.expert, a.d_weight,
                                (T *)a.d_logits, a.ld_d, ctx->s.status);
    });
}

}  // namespace

cudaError_t launch_expert_route(gs_ctx *ctx, const ExpertRouteArgs &a, cudaStream_t st) {
    const int warps = kRouteThreads / 32;
    int64_t want = (a.n_tokens + warps - 1) / warps;
    const int most = ctx->n_sm * 4 < kMaxRouteCtas ? ctx->n_sm * 4 : kMaxRouteCtas;
    const int n_ctas = want < 1 ? 1 : want < most ? (int)want : most;
    const int rows_per_cta = (int)((a.n_tokens + n_ctas - 1) / n_ctas);
    cudaError_t e = a.dtype == GS_F32 ? route_rows<float>(ctx, a, n_ctas, rows_per_cta, st)
                  : a.dtype == GS_BF16 ? route_rows<__nv_bfloat16>(ctx, a, n_ctas, rows_per_cta, st)
                                       : route_rows<__half>(ctx, a, n_ctas, rows_per_cta, st);
    if (e != cudaSuccess || !a.offsets) return e;
    int *counts = operator_scratch(ctx).expert_counts;
    {
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        e = launch_dependent(route_prefix_kernel, dim3((a.r.n_experts + warps - 1) / warps), dim3(kRouteThreads), 0, st,
                             counts, a.r.n_experts, n_ctas);
    }
    if (e != cudaSuccess) return e;
    const size_t smem = sizeof(int) * ((size_t)warps * a.r.n_experts + a.r.n_experts + 1);
    LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
    return launch_dependent(route_place_kernel, dim3(n_ctas), dim3(kRouteThreads), smem, st, a.expert,
                            a.n_tokens * a.r.top_k, a.r.top_k, rows_per_cta * a.r.top_k, a.r.n_experts,
                            counts, a.offsets, a.row_token, a.token_row);
}

cudaError_t launch_expert_route_backward(gs_ctx *ctx, const ExpertRouteGradArgs &a, cudaStream_t st) {
    return a.dtype == GS_F32 ? route_rows_backward<float>(ctx, a, st)
         : a.dtype == GS_BF16 ? route_rows_backward<__nv_bfloat16>(ctx, a, st)
                              : route_rows_backward<__half>(ctx, a, st);
}

}  // namespace gs
