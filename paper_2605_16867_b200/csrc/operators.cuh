// Internal declarations of the length predictor's operators (expert routing, the experts'
// products, their combination, gradient clipping).  Nothing here is part of the C ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_internal.cuh"

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

cudaError_t launch_clip(gs_ctx *ctx, const gs_grad *grads, int n_tensors, float max_norm, bool write,
                        float *out_norm, cudaStream_t st);

}  // namespace gs
