// Weighted sums of the experts' rows per token, and their gradients.
//   out[n] = sum_j w[n, j] y[row(n, j)];   dy[row(n, j)] = w[n, j] d_out[n];   dw[n, j] = y[row(n, j)] . d_out[n]
// Bound by memory: every row of y is read (or written) once.  A group of lanes owns a token and
// walks its columns eight at a time (16 bytes of 16-bit values); the slots' rows and weights are
// held in registers.  One token's sums are taken by one group in a fixed order: no atomics.
#include <type_traits>

#include "operators.cuh"

namespace gs {
namespace {

constexpr int kCombineThreads = 256;
constexpr unsigned kFull = 0xFFFFFFFFu;

template <typename T> struct Eight { T v[8]; };

// Eight columns from `col`; the row is 16-byte aligned and holds `features` of them.
template <typename T>
__device__ __forceinline__ void load8(const T *__restrict__ row, int col, int features, float (&v)[8]) {
    if (col + 8 <= features) {
        if constexpr (sizeof(T) == 2) {
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(row + col));
            const T *t = reinterpret_cast<const T *>(&q);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
        } else {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(row + col)), b = __ldg(reinterpret_cast<const float4 *>(row + col) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < features ? to_float(row[col + i]) : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *__restrict__ row, int col, int features, const float (&v)[8]) {
    if (col + 8 <= features) {
        if constexpr (sizeof(T) == 2) {
            uint4 q;
            T *t = reinterpret_cast<T *>(&q);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = from_float<T>(v[i]);
            *reinterpret_cast<uint4 *>(row + col) = q;
        } else {
            reinterpret_cast<float4 *>(row + col)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(row + col)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (col + i < features) row[col + i] = from_float<T>(v[i]);
    }
}

// kLanes lanes own a token (the fewest that cover its columns, a warp at most).
template <typename T, typename O, int kLanes>
__global__ void __launch_bounds__(kCombineThreads)
combine_kernel(const T *__restrict__ y, int n_rows, int64_t ld_y, const int32_t *__restrict__ token_row,
               const float *__restrict__ weight, int64_t n_tokens, int top_k, int features,
               O *__restrict__ out, int64_t ld_out, unsigned *__restrict__ status)
{
    dependent_begin();
    const int part = threadIdx.x % kLanes;
    bool bad = false;
    for (int64_t n = ((int64_t)blockIdx.x * kCombineThreads + threadIdx.x) / kLanes; n < n_tokens;
         n += (int64_t)gridDim.x * (kCombineThreads / kLanes)) {
        for (int col = part * 8; col < features; col += kLanes * 8) {
            float sum[8] = {};
            for (int j = 0; j < top_k; ++j) {
                const int r = token_row[n * top_k + j];
                if (r < 0 || r >= n_rows) { bad |= r != -1; continue; }
                const float w = weight ? weight[n * top_k + j] : 1.f;
                float v[8];
                load8(y + (int64_t)r * ld_y, col, features, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
            }
            store8(out + n * ld_out, col, features, sum);
        }
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename T, typename O, int kLanes>
__global__ void __launch_bounds__(kCombineThreads)
combine_backward_kernel(const O *__restrict__ d_out, int64_t ld_d, const T *__restrict__ y, int n_rows, int64_t ld_y,
                        const int32_t *__restrict__ token_row, const float *__restrict__ weight, int64_t n_tokens,
                        int top_k, int features, bool relu, T *__restrict__ dy, int64_t ld_dy,
                        float *__restrict__ d_weight, unsigned *__restrict__ status)
{
    dependent_begin();
    const int part = threadIdx.x % kLanes;
    const bool reads_y = d_weight || relu;
    bool bad = false;
    // (all lanes of a warp stay in the loop: the sums below are exchanged between a token's lanes)
    const int64_t step = (int64_t)gridDim.x * (kCombineThreads / kLanes);
    const int64_t n_first = ((int64_t)blockIdx.x * kCombineThreads + threadIdx.x) / kLanes;
    for (int64_t n = n_first; __any_sync(kFull, n < n_tokens); n += step) {
        for (int j = 0; j < top_k; ++j) {
            int r = -1;
            if (n < n_tokens) {
                r = token_row[n * top_k + j];
                if (r < -1 || r >= n_rows) { bad = true; r = -1; }
            }
            float dot = 0.f;
            if (r >= 0) {
                const float w = weight ? weight[n * top_k + j] : 1.f;
                for (int col = part * 8; col < features; col += kLanes * 8) {
                    float g[8], v[8];
                    load8(d_out + n * ld_d, col, features, g);
                    if (reads_y) load8(y + (int64_t)r * ld_y, col, features, v);
                    if (d_weight)
#pragma unroll
                        for (int i = 0; i < 8; ++i) dot = fmaf(v[i], g[i], dot);
                    if (dy) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) g[i] = relu && !(v[i] > 0.f) ? 0.f : w * g[i];
                        store8(dy + (int64_t)r * ld_dy, col, features, g);
                    }
                }
            }
            if (d_weight) {
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(kFull, dot, o);
                if (part == 0 && n < n_tokens) d_weight[n * top_k + j] = dot;
            }
        }
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename F> cudaError_t by_lanes(int features, F &&f) {
    if (features <= 8) return f(std::integral_constant<int, 1>());
    if (features <= 32) return f(std::integral_constant<int, 4>());
    if (features <= 128) return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

int combine_ctas(const gs_ctx *ctx, int64_t n_tokens, int lanes) {
    const int64_t want = (n_tokens * lanes + kCombineThreads - 1) / kCombineThreads;
    const int64_t most = (int64_t)ctx->n_sm * 32;
    return (int)(want < most ? want : most);
}

template <typename T, typename O>
cudaError_t combine_as(gs_ctx *ctx, const ExpertCombineArgs &a, cudaStream_t st) {
    return by_lanes(a.features, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        LaunchTimer t(ctx, GS_K_EXPERT_COMBINE, st);
        return launch_dependent(combine_kernel<T, O, L>, dim3(combine_ctas(ctx, a.n_tokens, L)), dim3(kCombineThreads), 0, st,
                                (const T *)a.y, (int)a.n_rows, a.ld_y, a.token_row, a.weight, a.n_tokens, a.top_k,
                                a.features, (O *)a.out, a.ld_out, ctx->s.status);
    });
}

template <typename T, typename O>
cudaError_t combine_backward_as(gs_ctx *ctx, const ExpertCombineArgs &a, cudaStream_t st) {
    return by_lanes(a.features, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        LaunchTimer t(ctx, GS_K_EXPERT_COMBINE, st);
        return launch_dependent(combine_backward_kernel<T, O, L>, dim3(combine_ctas(ctx, a.n_tokens, L)), dim3(kCombineThreads), 0, st,
                                (const O *)a.d_out, a.ld_d_out, (const T *)a.y, (int)a.n_rows, a.ld_y, a.token_row, a.weight,
                                a.n_tokens, a.top_k, a.features, (a.flags & GS_EXPERT_RELU_INPUT) != 0, (T *)a.dy, a.ld_dy,
                                a.d_weight, ctx->s.status);
    });
}

}  // namespace

cudaError_t launch_expert_combine(gs_ctx *ctx, const ExpertCombineArgs &a, cudaStream_t st) {
    if (a.dtype == GS_BF16)
        return a.out_dtype == GS_F32 ? combine_as<__nv_bfloat16, float>(ctx, a, st) : combine_as<__nv_bfloat16, __nv_bfloat16>(ctx, a, st);
    return a.out_dtype == GS_F32 ? combine_as<__half, float>(ctx, a, st) : combine_as<__half, __half>(ctx, a, st);
}

cudaError_t launch_expert_combine_backward(gs_ctx *ctx, const ExpertCombineArgs &a, cudaStream_t st) {
    if (a.dtype == GS_BF16)
        return a.out_dtype == GS_F32 ? combine_backward_as<__nv_bfloat16, float>(ctx, a, st) : combine_backward_as<__nv_bfloat16, __nv_bfloat16>(ctx, a, st);
    return a.out_dtype == GS_F32 ? combine_backward_as<__half, float>(ctx, a, st) : combine_backward_as<__half, __half>(ctx, a, st);
}

}  // namespace gs
