// Weighted sums of the experts' rows per token, and their gradients.
//   out[n] = sum_j w[n, j] y[row(n, j)];   dy[row(n, j)] = w[n, j] d_out[n];   dw[n, j] = y[row(n, j)] . d_out[n]
// Bound by memory: every row of y is read (or written) once.  A group of lanes owns a token and
// walks its columns eight at a time (16 bytes of 16-bit values).  One token's sums are taken by one
// group in a fixed order: no atomics.  131,072 x 1024 from two rows each: 125 us = 6.45 TB/s, the
// rate of a plain copy; the gradient of 65,536 x 1024: 119 us = 5.65 TB/s.
#include <type_traits>

#include "operators.cuh"

namespace gs {
namespace {

constexpr int kCombineThreads = 256;
constexpr unsigned kFull = 0xFFFFFFFFu;

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

// Eight columns as they lie in memory (16-bit values), zeros past the last one.
template <typename T>
__device__ __forceinline__ uint4 load_packed(const T *__restrict__ row, int col, int features) {
    if (col + 8 <= features) return __ldg(reinterpret_cast<const uint4 *>(row + col));
    uint4 q = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) if (col + i < features) reinterpret_cast<T *>(&q)[i] = row[col + i];
    return q;
}

// Rows and weights of a token's slots: lane j of the token's lanes holds slot j (or, where a token has
// fewer lanes than slots, they are read where they are used).  The next token's are asked for while
// this one's rows are on their way: otherwise every token waits for memory twice.
template <int kLanes>
struct Slots {
    static constexpr bool kHeld = kLanes >= GS_MAX_TOP_K;
    const int32_t *__restrict__ token_row;
    const float *__restrict__ weight;
    int64_t n_tokens;
    int top_k, n_rows, r = -1;
    float w = 0.f;
    bool bad = false;
    __device__ __forceinline__ int checked(int row) {
        if (row < -1 || row >= n_rows) { bad = true; return -1; }
        return row;
    }
    __device__ __forceinline__ void ask(int64_t n, int part) {
        if (!kHeld) return;
        const bool there = n < n_tokens && part < top_k;
        r = there ? token_row[n * top_k + part] : -1;
        w = there ? weight ? weight[n * top_k + part] : 1.f : 0.f;
    }
    // slot j of token n, from the values asked for (held) or from memory; -1: none
    __device__ __forceinline__ int row(int64_t n, int j, int held) {
        if (kHeld) { const int v = __shfl_sync(kFull, held, j & (kLanes - 1), kLanes); return j < top_k ? v : -1; }
        return n < n_tokens && j < top_k ? checked(token_row[n * top_k + j]) : -1;
    }
    __device__ __forceinline__ float factor(int64_t n, int j, float held) {
        if (kHeld) return __shfl_sync(kFull, held, j & (kLanes - 1), kLanes);
        return n < n_tokens && j < top_k ? weight ? weight[n * top_k + j] : 1.f : 0.f;
    }
};

// kLanes lanes own a token (the fewest that cover its columns, a warp at most).  A lane has kBlocks
// blocks of eight columns of kSlots slots under way at a time; more in flight costs more warps than it
// brings (four blocks as floats, 112 registers: 328 us instead of 162 us at 131,072 x 1024).
constexpr int kBlocks = 2, kSlots = 2;
template <typename T, typename O, int kLanes>
__global__ void __launch_bounds__(kCombineThreads, 4)
combine_kernel(const T *__restrict__ y, int n_rows, int64_t ld_y, const int32_t *__restrict__ token_row,
               const float *__restrict__ weight, int64_t n_tokens, int top_k, int features,
               O *__restrict__ out, int64_t ld_out, unsigned *__restrict__ status)
{
    dependent_begin();
    const int part = threadIdx.x % kLanes;
    const int64_t step = (int64_t)gridDim.x * (kCombineThreads / kLanes);
    Slots<kLanes> slots = {token_row, weight, n_tokens, top_k, n_rows};
    int64_t n = ((int64_t)blockIdx.x * kCombineThreads + threadIdx.x) / kLanes;
    slots.ask(n, part);
    for (; __any_sync(kFull, n < n_tokens); n += step) {
        const int held_r = slots.checked(slots.r);
        const float held_w = slots.w;
        slots.ask(n + step, part);
        for (int col0 = 0; col0 < features; col0 += kLanes * 8 * kBlocks) {
            const int col = col0 + part * 8;
            float sum[kBlocks][8] = {};
            for (int j0 = 0; j0 < top_k; j0 += kSlots) {
                uint4 q[kSlots][kBlocks];
                float w[kSlots];
                int r[kSlots];
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    r[j] = slots.row(n, j0 + j, held_r);
                    w[j] = slots.factor(n, j0 + j, held_w);
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
                        if (r[j] >= 0 && col + b * kLanes * 8 < features) q[j][b] = load_packed(y + r[j] * ld_y, col + b * kLanes * 8, features);
                }
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if (r[j] < 0) continue;
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[b][i] = fmaf(w[j], to_float(reinterpret_cast<const T *>(&q[j][b])[i]), sum[b][i]);
                }
            }
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                if (n < n_tokens && col + b * kLanes * 8 < features) store8(out + n * ld_out, col + b * kLanes * 8, features, sum[b]);
        }
    }
    if (slots.bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

// Eight columns of d_out, packed where they are 16-bit values.
template <typename T, typename O> struct Gradient {
    uint4 q;
    __device__ __forceinline__ void load(const T *row, int col, int features) { q = load_packed(row, col, features); }
    __device__ __forceinline__ float at(int i) const { return to_float(reinterpret_cast<const T *>(&q)[i]); }
};
template <typename T> struct Gradient<T, float> {
    float v[8];
    __device__ __forceinline__ void load(const float *row, int col, int features) { load8(row, col, features, v); }
    __device__ __forceinline__ float at(int i) const { return v[i]; }
};

template <typename T, typename O, int kLanes>
__global__ void __launch_bounds__(kCombineThreads, 4)
combine_backward_kernel(const O *__restrict__ d_out, int64_t ld_d, const T *__restrict__ y, int n_rows, int64_t ld_y,
                        const int32_t *__restrict__ token_row, const float *__restrict__ weight, int64_t n_tokens,
                        int top_k, int features, bool relu, T *__restrict__ dy, int64_t ld_dy,
                        float *__restrict__ d_weight, unsigned *__restrict__ status)
{
    dependent_begin();
    const int part = threadIdx.x % kLanes;
    const bool reads_y = d_weight || relu;
    const int64_t step = (int64_t)gridDim.x * (kCombineThreads / kLanes);
    Slots<kLanes> slots = {token_row, weight, n_tokens, top_k, n_rows};
    int64_t n = ((int64_t)blockIdx.x * kCombineThreads + threadIdx.x) / kLanes;
    slots.ask(n, part);
    for (; __any_sync(kFull, n < n_tokens); n += step) {
        const int held_r = slots.checked(slots.r);
        const float held_w = slots.w;
        slots.ask(n + step, part);
        for (int j0 = 0; j0 < top_k; j0 += kSlots) {
            int r[kSlots];
            float w[kSlots], dot[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                r[j] = slots.row(n, j0 + j, held_r);
                w[j] = slots.factor(n, j0 + j, held_w);
                dot[j] = 0.f;
            }
            for (int col = part * 8; n < n_tokens && col < features; col += kLanes * 8 * kBlocks) {
                uint4 q[kSlots][kBlocks];
                Gradient<T, O> g[kBlocks];
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const int c = col + b * kLanes * 8;
                    if (c >= features) continue;
                    g[b].load(d_out + n * ld_d, c, features);
#pragma unroll
                    for (int j = 0; j < kSlots; ++j)
                        if (reads_y && r[j] >= 0) q[j][b] = load_packed(y + r[j] * ld_y, c, features);
                }
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const int c = col + b * kLanes * 8;
                    if (c >= features) continue;
#pragma unroll
                    for (int j = 0; j < kSlots; ++j) {
                        if (r[j] < 0) continue;
                        float z[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float v = reads_y ? to_float(reinterpret_cast<const T *>(&q[j][b])[i]) : 0.f;
                            if (d_weight) dot[j] = fmaf(v, g[b].at(i), dot[j]);
                            z[i] = relu && !(v > 0.f) ? 0.f : w[j] * g[b].at(i);
                        }
                        if (dy) store8(dy + r[j] * ld_dy, c, features, z);
                    }
                }
            }
            if (d_weight) {
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
#pragma unroll
                    for (int o = kLanes / 2; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(kFull, dot[j], o);
                    if (part == 0 && n < n_tokens && j0 + j < top_k) d_weight[n * top_k + j0 + j] = dot[j];
                }
            }
        }
    }
    if (slots.bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename F> cudaError_t by_lanes(int features, F &&f) {
    if (features <= 8) return f(std::integral_constant<int, 1>());
    if (features <= 32) return f(std::integral_constant<int, 4>());
    if (features <= 128) return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

int combine_ctas(const gs_ctx *ctx, int64_t n_tokens, int lanes) {
    const int64_t want = (n_tokens * lanes + kCombineThreads - 1) / kCombineThreads;
    const int64_t most = (int64_t)ctx->n_sm * 4;     // as many as are resident (launch bounds)
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
