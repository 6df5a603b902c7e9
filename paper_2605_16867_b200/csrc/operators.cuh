// Internal declarations of the length predictor's operators (expert routing, the experts'
// products, their combination, gradient clipping; token embeddings, gated recurrence, dropout, dense
// layers).  Nothing here is part of the C ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_internal.cuh"
#include "pairs.cuh"

namespace gs {

constexpr int kMaxRouteCtas = 592;     // CTAs of one expert routing (a few per SM), one count per expert each
constexpr size_t kExpertCountBytes = sizeof(int) * (size_t)GS_MAX_EXPERTS * (kMaxRouteCtas + 1);
constexpr int kMaxClipCtas = 4096;     // partial sums of one global norm

// Device scratch of the operators, owned by a context.
struct OperatorScratch {
    int *expert_counts;                // [GS_MAX_EXPERTS][kMaxRouteCtas] rows per expert and CTA, then [GS_MAX_EXPERTS] totals
    double *clip_partials;             // [kMaxClipCtas] sums of squares
};

struct Context : gs_ctx {
    OperatorScratch ops;
};
inline OperatorScratch &operator_scratch(gs_ctx *ctx) { return static_cast<Context *>(ctx)->ops; }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Eight columns from `col`; the row is 16-byte aligned and holds `features` of them.  (kReadOnly: nothing writes them while
// the kernel runs, not even the kernel itself in place.)
template <typename V, bool kReadOnly> __device__ __forceinline__ V load_as(const void *p) {
    const V *v = reinterpret_cast<const V *>(p);
    return kReadOnly ? __ldg(v) : *v;
}
template <bool kReadOnly = true, typename T>
__device__ __forceinline__ void load8(const T *row, int col, int features, float (&v)[8]) {
    if (col + 8 <= features) {
        if constexpr (sizeof(T) == 2) {
            const uint4 q = load_as<uint4, kReadOnly>(row + col);
            const T *t = reinterpret_cast<const T *>(&q);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_float(t[i]);
        } else {
            const float4 a = load_as<float4, kReadOnly>(row + col), b = load_as<float4, kReadOnly>(row + col + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < features ? to_float(row[col + i]) : 0.f;
    }
}

// (kStream: not read again soon, so that it does not push out of the L2 cache what is)
template <bool kStream = false, typename T>
__device__ __forceinline__ void store8(T *__restrict__ row, int col, int features, const float (&v)[8]) {
    if (col + 8 <= features) {
        if constexpr (sizeof(T) == 2) {
            uint4 q;
            T *t = reinterpret_cast<T *>(&q);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = from_float<T>(v[i]);
            if (kStream) __stcs(reinterpret_cast<uint4 *>(row + col), q);
            else *reinterpret_cast<uint4 *>(row + col) = q;
        } else {
            const float4 a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]);
            if (kStream) {
                __stcs(reinterpret_cast<float4 *>(row + col), a);
                __stcs(reinterpret_cast<float4 *>(row + col) + 1, b);
            } else {
                reinterpret_cast<float4 *>(row + col)[0] = a;
                reinterpret_cast<float4 *>(row + col)[1] = b;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (col + i < features) row[col + i] = from_float<T>(v[i]);
    }
}

// Eight columns as they are kept in memory, asked for now and used later.  (No branch around the load and nothing
// that waits for it: where a load and its conversion share a branch, loads come one at a time.)
template <typename T> struct Eight {
    uint4 q[sizeof(T) / 2];
    template <bool kReadOnly = true> __device__ __forceinline__ void ask(const T *row, int col, int features) {
        if (col + 8 <= features) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = load_as<uint4, kReadOnly>(reinterpret_cast<const uint4 *>(row + col) + i);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) if (col + i < features) reinterpret_cast<T *>(q)[i] = row[col + i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return to_float(reinterpret_cast<const T *>(q)[i]); }
};

// Pairs of the eight columns.
template <typename T> __device__ __forceinline__ float2 two(const Eight<T> &v, int i) {
    if constexpr (sizeof(T) == 4) return make_float2(v[2 * i], v[2 * i + 1]);
    else return unpack2<T>(reinterpret_cast<const uint32_t *>(v.q)[i]);
}

// Two floats rounded to T, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// max(v, 0) of both halves; a NaN stays one.
template <typename T> __device__ __forceinline__ uint32_t relu2(uint32_t v);
template <> __device__ __forceinline__ uint32_t relu2<__nv_bfloat16>(uint32_t v) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0u));
    return r;
}
template <> __device__ __forceinline__ uint32_t relu2<__half>(uint32_t v) {
    uint32_t r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0u));
    return r;
}

// First and last of a kernel launched with launch_dependent: the kernel after this one may be set
// up, and this one waits until everything before it in the stream is done and visible.
__device__ __forceinline__ void dependent_begin() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}
// The same in two parts, for kernels of several CTAs per SM: CTAs of the next kernel that are set
// up early gather on the SMs that have room first, and stay there.  So the next kernel is let in at
// the end.
__device__ __forceinline__ void dependent_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dependent_end() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Launches a kernel once the one before it has ended (no programmatic dependence).
template <typename... KArgs, typename... Args>
inline cudaError_t launch_after(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

struct ExpertRouteArgs {
    const void *logits;
    int dtype;
    int64_t n_tokens, ld;
    const float *bias;
    gs_expert_router r;
    int32_t *expert, *offsets, *row_token, *token_row;
    float *weight;
};
cudaError_t launch_expert_route(gs_ctx *ctx, const ExpertRouteArgs &a, cudaStream_t st);

struct ExpertRouteGradArgs {
    const void *logits;
    int dtype;
    int64_t n_tokens, ld, ld_d;
    gs_expert_router r;
    const int32_t *expert;
    const float *d_weight;
    void *d_logits;
};
cudaError_t launch_expert_route_backward(gs_ctx *ctx, const ExpertRouteGradArgs &a, cudaStream_t st);

struct ExpertLinearArgs {
    int dtype;
    const void *x;              // [n_x_rows, in]
    int64_t n_x_rows, ld_x;
    const int32_t *row_token, *offsets;
    int n_experts;
    int64_t n_rows;
    const void *w;              // [n_experts, out, in]
    int64_t ld_w;
    int in, out;
    unsigned flags;
    // forward
    const float *bias;
    void *y;
    int64_t ld_y;
    // backward
    const void *dz;
    int64_t ld_dz;
    void *dx;
    int64_t ld_dx;
    float *dw;
    int64_t ld_dw;
    float *db;
    void *workspace;
    int timed_as = GS_K_EXPERT_LINEAR;          // the kernel that the launches' time is booked under
};
cudaError_t configure_expert_linear();
cudaError_t launch_expert_linear(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st);
cudaError_t launch_expert_linear_dx(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st);
cudaError_t launch_expert_linear_dw(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st);
int64_t expert_linear_workspace(const gs_ctx *ctx, int n_experts, int64_t n_rows, int in, int out);

struct ExpertCombineArgs {
    int dtype, out_dtype;
    const void *y;
    int64_t n_rows, ld_y;
    const int32_t *token_row;
    const float *weight;
    int64_t n_tokens;
    int top_k, features;
    void *out;
    int64_t ld_out;
    // backward
    const void *d_out;
    int64_t ld_d_out;
    unsigned flags;
    void *dy;
    int64_t ld_dy;
    float *d_weight;
};
cudaError_t launch_expert_combine(gs_ctx *ctx, const ExpertCombineArgs &a, cudaStream_t st);
cudaError_t launch_expert_combine_backward(gs_ctx *ctx, const ExpertCombineArgs &a, cudaStream_t st);

struct EmbeddingArgs {
    int dtype;
    const void *table;          // [vocabulary, features]
    int64_t ld_table;
    const int32_t *ids;
    int64_t n_tokens;
    int vocabulary, features;
    float scale;
    void *out;
    int64_t ld_out;
    // backward
    const void *d_out;
    int64_t ld_d_out;
    float *d_table;
    int64_t ld_d_table;
    void *workspace;
};
cudaError_t configure_embedding();
cudaError_t launch_embedding(gs_ctx *ctx, const EmbeddingArgs &a, cudaStream_t st);
cudaError_t launch_embedding_backward(gs_ctx *ctx, const EmbeddingArgs &a, cudaStream_t st);
int64_t embedding_workspace(const gs_ctx *ctx, int64_t n_tokens, int vocabulary, int features);

struct GatedScanArgs {
    int dtype;
    const void *x, *gate;       // [n_rows, features]
    int64_t ld_x, ld_gate;
    const int32_t *offsets;
    int64_t n_sequences;
    int n_rows, features;
    const float *h0;
    int64_t ld_h0;
    void *out;
    int64_t ld_out;
    float *last;
    int64_t ld_last;
    float *states;              // written by the forward direction, read by the backward one
    int64_t ld_states;
    // backward
    const void *d_out;
    int64_t ld_d_out;
    const float *d_last;
    int64_t ld_d_last;
    void *dx, *d_gate;
    int64_t ld_dx, ld_d_gate;
    float *d_h0;
    int64_t ld_d_h0;
    unsigned *status;
};
cudaError_t configure_gated_scan();
cudaError_t launch_gated_scan(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st);
cudaError_t launch_gated_scan_backward(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st);

struct DropoutArgs {
    int dtype;
    const void *x, *residual;
    int64_t ld_x, ld_residual, n_rows;
    int features;
    const int64_t *rng;
    unsigned cut;               // of 65536 values so many are dropped
    void *out;
    int64_t ld_out;
};
cudaError_t launch_dropout(gs_ctx *ctx, const DropoutArgs &a, cudaStream_t st);

struct LinearArgs {
    int dtype;
    const void *x;              // [n_rows, in]
    int64_t ld_x, n_rows;
    const void *w;              // [out, in]
    int64_t ld_w;
    int in, out, activation;
    const void *add;            // the residual, or what goes around the layer
    int64_t ld_add;
    // forward
    const float *bias;
    void *z, *y;
    int64_t ld_z, ld_y;
    // backward
    const void *dz, *z_below;
    int64_t ld_dz, ld_z_below;
    void *dx, *dz_below;
    int64_t ld_dx, ld_dz_below;
    float *dw, *db;
    int64_t ld_dw;
    void *workspace;
};
bool linear_is_few(const gs_ctx *ctx, const LinearArgs &a);
cudaError_t launch_linear_few(gs_ctx *ctx, const LinearArgs &a, cudaStream_t st);
cudaError_t launch_linear(gs_ctx *ctx, const LinearArgs &a, cudaStream_t st);
cudaError_t launch_linear_dx(gs_ctx *ctx, const LinearArgs &a, cudaStream_t st);
cudaError_t launch_linear_dw(gs_ctx *ctx, const LinearArgs &a, cudaStream_t st);

struct ActivationArgs {
    int dtype, activation;
    const void *d_out, *z;
    int64_t ld_d_out, ld_z, n_rows;
    int features;
    void *dz;
    int64_t ld_dz;
};
cudaError_t launch_activation_backward(gs_ctx *ctx, const ActivationArgs &a, cudaStream_t st);

cudaError_t launch_clip(gs_ctx *ctx, const gs_grad *grads, int n_tensors, float max_norm, bool write,
                        float *out_norm, cudaStream_t st);

}  // namespace gs
