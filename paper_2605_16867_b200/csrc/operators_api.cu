// C-ABI entry points of the length predictor's operators: argument checks and kernel sequencing.
#include <math.h>
#include <stdint.h>

#include "api_util.cuh"
#include "operators.cuh"

using gs::cuda_fail;
using gs::DeviceGuard;
using gs::misaligned;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;

bool is_dtype(int d) { return d == GS_F32 || d == GS_BF16 || d == GS_F16; }
bool is_operand(int d) { return d == GS_BF16 || d == GS_F16; }
int bytes_of(int d) { return d == GS_F32 ? 4 : 2; }

int check_router(const gs_expert_router *r) {
    if (!r || r->n_experts < 1 || r->n_experts > GS_MAX_EXPERTS) return GS_ERR_INVALID_ARG;
    if (r->score != GS_SCORE_SOFTMAX && r->score != GS_SCORE_SIGMOID) return GS_ERR_INVALID_ARG;
    if (r->n_groups < 1 || r->n_groups > GS_MAX_EXPERT_GROUPS || r->n_experts % r->n_groups) return GS_ERR_INVALID_ARG;
    if (r->top_groups < 1 || r->top_groups > r->n_groups) return GS_ERR_INVALID_ARG;
    if (r->group_top < 1 || r->group_top > 2 || r->renormalise < 0 || r->renormalise > 1) return GS_ERR_INVALID_ARG;
    if (r->top_k < 1 || r->top_k > GS_MAX_TOP_K || r->top_k > r->n_experts / r->n_groups * r->top_groups) return GS_ERR_INVALID_ARG;
    if (!(r->scale > -INFINITY && r->scale < INFINITY)) return GS_ERR_INVALID_ARG;
    return GS_OK;
}

// A row-major matrix argument: there if it has to be, wide enough, rows starting 16-byte aligned.
int check_matrix(const void *p, int64_t ld, int64_t cols, int dtype, bool empty) {
    if (ld < cols || ld > ((int64_t)1 << 31)) return GS_ERR_INVALID_ARG;
    if (ld * bytes_of(dtype) % 16) return GS_ERR_ALIGN;
    if (!p) return empty ? GS_OK : GS_ERR_INVALID_ARG;
    return misaligned(p) ? GS_ERR_ALIGN : GS_OK;
}

int check_array(const void *p, bool empty) {
    if (!p) return empty ? GS_OK : GS_ERR_INVALID_ARG;
    return misaligned(p) ? GS_ERR_ALIGN : GS_OK;
}

#define GS_TRY(expr) do { const int rc_ = (expr); if (rc_ != GS_OK) return rc_; } while (0)

int check_linear(const gs_ctx *ctx, const gs::ExpertLinearArgs &a) {
    if (!ctx || !is_operand(a.dtype)) return GS_ERR_INVALID_ARG;
    if (a.n_experts < 1 || a.n_experts > GS_MAX_EXPERTS) return GS_ERR_INVALID_ARG;
    if (a.in < 1 || a.in > GS_MAX_FEATURES || a.out < 1 || a.out > GS_MAX_FEATURES) return GS_ERR_INVALID_ARG;
    if (a.n_rows < 0 || a.n_rows > GS_MAX_EXPERT_ROWS || a.n_x_rows < 0 || a.n_x_rows > kMaxRows) return GS_ERR_INVALID_ARG;
    if (!a.row_token && a.n_x_rows != a.n_rows) return GS_ERR_INVALID_ARG;
    if (a.row_token && a.n_rows > 0 && a.n_x_rows < 1) return GS_ERR_INVALID_ARG;
    GS_TRY(check_array(a.offsets, false));
    return check_array(a.row_token, true);
}

}  // namespace

extern "C" {

GS_API int gs_expert_route(gs_ctx *ctx, const void *logits, int logits_dtype, int64_t n_tokens, int64_t ld_logits,
                    const float *bias, const gs_expert_router *router,
                    int32_t *out_expert, float *out_weight, int32_t *out_offsets, int32_t *out_row_token,
                    int32_t *out_token_row, void *cuda_stream)
{
    if (!ctx || !is_dtype(logits_dtype)) return GS_ERR_INVALID_ARG;
    GS_TRY(check_router(router));
    if (n_tokens < 0 || n_tokens * (int64_t)router->top_k > kMaxRows || n_tokens > kMaxRows) return GS_ERR_INVALID_ARG;
    if (ld_logits < router->n_experts || ld_logits > ((int64_t)1 << 31)) return GS_ERR_INVALID_ARG;
    const bool empty = n_tokens == 0, order = out_offsets || out_row_token || out_token_row;
    GS_TRY(check_array(logits, empty));
    GS_TRY(check_array(bias, true));
    GS_TRY(check_array(out_expert, empty));
    GS_TRY(check_array(out_weight, empty));
    if (order) {
        GS_TRY(check_array(out_offsets, false));
        GS_TRY(check_array(out_row_token, empty));
        GS_TRY(check_array(out_token_row, empty));
    }
    if (empty && !order) return GS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    const gs::ExpertRouteArgs a = {logits, logits_dtype, n_tokens, ld_logits, bias, *router,
                                   out_expert, out_offsets, out_row_token, out_token_row, out_weight};
    const cudaError_t e = gs::launch_expert_route(ctx, a, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

GS_API int gs_expert_route_backward(gs_ctx *ctx, const void *logits, int logits_dtype, int64_t n_tokens,
                    int64_t ld_logits, const gs_expert_router *router, const int32_t *expert,
                    const float *d_weight, void *out_d_logits, int64_t ld_d_logits, void *cuda_stream)
{
    if (!ctx || !is_dtype(logits_dtype)) return GS_ERR_INVALID_ARG;
    GS_TRY(check_router(router));
    if (n_tokens < 0 || n_tokens * (int64_t)router->top_k > kMaxRows || n_tokens > kMaxRows) return GS_ERR_INVALID_ARG;
    for (int64_t ld : {ld_logits, ld_d_logits})
        if (ld < router->n_experts || ld > ((int64_t)1 << 31)) return GS_ERR_INVALID_ARG;
    if (n_tokens == 0) return GS_OK;
    for (const void *p : {logits, (const void *)expert, (const void *)d_weight, (const void *)out_d_logits}) GS_TRY(check_array(p, false));
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    const gs::ExpertRouteGradArgs a = {logits, logits_dtype, n_tokens, ld_logits, ld_d_logits, *router, expert, d_weight, out_d_logits};
    const cudaError_t e = gs::launch_expert_route_backward(ctx, a, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

GS_API int gs_expert_linear(gs_ctx *ctx, int dtype, const void *x, int64_t n_x_rows, int64_t ld_x,
                    const int32_t *row_token, const int32_t *offsets, int32_t n_experts, int64_t n_rows,
                    const void *w, int64_t ld_w, const float *bias, int32_t in_features, int32_t out_features,
                    unsigned flags, void *out, int64_t ld_out, void *cuda_stream)
{
    gs::ExpertLinearArgs a = {};
    a.dtype = dtype; a.x = x; a.n_x_rows = n_x_rows; a.ld_x = ld_x; a.row_token = row_token; a.offsets = offsets;
    a.n_experts = n_experts; a.n_rows = n_rows; a.w = w; a.ld_w = ld_w; a.in = in_features; a.out = out_features;
    a.flags = flags; a.bias = bias; a.y = out; a.ld_y = ld_out;
    GS_TRY(check_linear(ctx, a));
    if (flags & ~GS_EXPERT_RELU) return GS_ERR_INVALID_ARG;
    const bool empty = n_rows == 0;
    GS_TRY(check_matrix(x, ld_x, in_features, dtype, empty));
    GS_TRY(check_matrix(w, ld_w, in_features, dtype, empty));
    GS_TRY(check_matrix(out, ld_out, out_features, dtype, empty));
    GS_TRY(check_array(bias, true));
    if (empty) return GS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    const cudaError_t e = gs::launch_expert_linear(ctx, a, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

GS_API int64_t gs_expert_linear_backward_workspace(const gs_ctx *ctx, int32_t n_experts, int64_t n_rows,
                    int32_t in_features, int32_t out_features)
{
    if (!ctx || n_experts < 1 || n_experts > GS_MAX_EXPERTS || n_rows < 0 || n_rows > GS_MAX_EXPERT_ROWS || in_features < 1 ||
        in_features > GS_MAX_FEATURES || out_features < 1 || out_features > GS_MAX_FEATURES)
        return GS_ERR_INVALID_ARG;
    return gs::expert_linear_workspace(ctx, n_experts, n_rows, in_features, out_features);
}

GS_API int gs_expert_linear_backward(gs_ctx *ctx, int dtype, const void *dz, int64_t ld_dz,
                    const void *x, int64_t n_x_rows, int64_t ld_x, const int32_t *row_token,
                    const int32_t *offsets, int32_t n_experts, int64_t n_rows, const void *w, int64_t ld_w,
                    int32_t in_features, int32_t out_features, unsigned flags,
                    void *out_dx, int64_t ld_dx, float *out_dw, int64_t ld_dw, float *out_db,
                    void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    gs::ExpertLinearArgs a = {};
    a.dtype = dtype; a.x = x; a.n_x_rows = n_x_rows; a.ld_x = ld_x; a.row_token = row_token; a.offsets = offsets;
    a.n_experts = n_experts; a.n_rows = n_rows; a.w = w; a.ld_w = ld_w; a.in = in_features; a.out = out_features;
    a.flags = flags; a.dz = dz; a.ld_dz = ld_dz; a.dx = out_dx; a.ld_dx = ld_dx; a.dw = out_dw; a.ld_dw = ld_dw;
    a.db = out_db; a.workspace = workspace;
    GS_TRY(check_linear(ctx, a));
    if (flags & ~GS_EXPERT_RELU_INPUT) return GS_ERR_INVALID_ARG;
    const bool empty = n_rows == 0;                  // (an output without elements may have no address)
    if ((!out_dx && !out_dw && !empty) || (out_db && !out_dw)) return GS_ERR_INVALID_ARG;
    const bool masked = out_dx && (flags & GS_EXPERT_RELU_INPUT);
    GS_TRY(check_matrix(dz, ld_dz, out_features, dtype, empty));
    if (out_dw || masked) GS_TRY(check_matrix(x, ld_x, in_features, dtype, empty));
    if (out_dx) {
        GS_TRY(check_matrix(w, ld_w, in_features, dtype, empty));
        GS_TRY(check_matrix(out_dx, ld_dx, in_features, dtype, false));
    }
    if (out_dw) {
        GS_TRY(check_matrix(out_dw, ld_dw, in_features, GS_F32, false));
        GS_TRY(check_array(out_db, true));
        const int64_t need = gs::expert_linear_workspace(ctx, n_experts, n_rows, in_features, out_features);
        if (workspace_bytes < need || (need > 0 && !workspace)) return GS_ERR_WORKSPACE;
        GS_TRY(check_array(workspace, true));
    }
    if (empty && !out_dw) return GS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    cudaError_t e = cudaSuccess;
    if (out_dx && !empty) e = gs::launch_expert_linear_dx(ctx, a, (cudaStream_t)cuda_stream);
    if (e == cudaSuccess && out_dw) e = gs::launch_expert_linear_dw(ctx, a, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

GS_API int gs_expert_combine(gs_ctx *ctx, int dtype, const void *y, int64_t n_rows, int64_t ld_y,
                    const int32_t *token_row, const float *weight, int64_t n_tokens, int32_t top_k,
                    int32_t features, int out_dtype, void *out, int64_t ld_out, void *cuda_stream)
{
    if (!ctx || !is_operand(dtype) || (out_dtype != dtype && out_dtype != GS_F32)) return GS_ERR_INVALID_ARG;
    if (top_k < 1 || top_k > GS_MAX_TOP_K || features < 1 || features > GS_MAX_FEATURES) return GS_ERR_INVALID_ARG;
    if (n_tokens < 0 || n_tokens * (int64_t)top_k > kMaxRows || n_tokens > kMaxRows || n_rows < 0 || n_rows > kMaxRows) return GS_ERR_INVALID_ARG;
    const bool empty = n_tokens == 0;
    GS_TRY(check_matrix(y, ld_y, features, dtype, empty || n_rows == 0));
    GS_TRY(check_matrix(out, ld_out, features, out_dtype, empty));
    GS_TRY(check_array(token_row, empty));
    GS_TRY(check_array(weight, true));
    if (empty) return GS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    gs::ExpertCombineArgs a = {};
    a.dtype = dtype; a.out_dtype = out_dtype; a.y = y; a.n_rows = n_rows; a.ld_y = ld_y; a.token_row = token_row;
    a.weight = weight; a.n_tokens = n_tokens; a.top_k = top_k; a.features = features; a.out = out; a.ld_out = ld_out;
    const cudaError_t e = gs::launch_expert_combine(ctx, a, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

GS_API int gs_expert_combine_backward(gs_ctx *ctx, int dtype, int d_out_dtype, const void *d_out, int64_t ld_d_out,
                    const void *y, int64_t n_rows, int64_t ld_y, const int32_t *token_row, const float *weight,
                    int64_t n_tokens, int32_t top_k, int32_t features, unsigned flags,
                    void *out_dy, int64_t ld_dy, float *out_d_weight, void *cuda_stream)
{
    if (!ctx || !is_operand(dtype) || (d_out_dtype != dtype && d_out_dtype != GS_F32)) return GS_ERR_INVALID_ARG;
    if (top_k < 1 || top_k > GS_MAX_TOP_K || features < 1 || features > GS_MAX_FEATURES) return GS_ERR_INVALID_ARG;
    if (n_tokens < 0 || n_tokens * (int64_t)top_k > kMaxRows || n_tokens > kMaxRows || n_rows < 0 || n_rows > kMaxRows) return GS_ERR_INVALID_ARG;
    if ((flags & ~GS_EXPERT_RELU_INPUT) || (!out_dy && !out_d_weight && n_rows > 0 && n_tokens > 0)) return GS_ERR_INVALID_ARG;
    const bool empty = n_tokens == 0, reads_y = out_d_weight || (flags & GS_EXPERT_RELU_INPUT);
    GS_TRY(check_matrix(d_out, ld_d_out, features, d_out_dtype, empty));
    if (reads_y) GS_TRY(check_matrix(y, ld_y, features, dtype, empty || n_rows == 0));
    if (out_dy) GS_TRY(check_matrix(out_dy, ld_dy, features, dtype, false));
    GS_TRY(check_array(token_row, empty));
    GS_TRY(check_array(weight, true));
    GS_TRY(check_array(out_d_weight, true));
    if (empty) return GS_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    gs::ExpertCombineArgs a = {};
    a.dtype = dtype; a.out_dtype = d_out_dtype; a.y = y; a.n_rows = n_rows; a.ld_y = ld_y; a.token_row = token_row;
    a.weight = weight; a.n_tokens = n_tokens; a.top_k = top_k; a.features = features; a.d_out = d_out;
    a.ld_d_out = ld_d_out; a.flags = flags; a.dy = out_dy; a.ld_dy = ld_dy; a.d_weight = out_d_weight;
    const cudaError_t e = gs::launch_expert_combine_backward(ctx, a, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

GS_API int gs_clip_grad_norm(gs_ctx *ctx, const gs_grad *grads, int32_t n_tensors, float max_norm,
                    float *out_norm, void *cuda_stream)
{
    if (!ctx || n_tensors < 0 || (n_tensors > 0 && !grads) || !(max_norm >= 0.f)) return GS_ERR_INVALID_ARG;
    if (!out_norm) return GS_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(out_norm) & 3u) return GS_ERR_ALIGN;
    bool any = false, all = true;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const gs_grad &g = grads[i];
        if (!is_dtype(g.dtype) || g.n_elements < 0 || g.n_elements > ((int64_t)1 << 40)) return GS_ERR_INVALID_ARG;
        if (g.n_elements == 0) continue;
        if (!g.grad) return GS_ERR_INVALID_ARG;
        const uintptr_t own = (uintptr_t)bytes_of(g.dtype) - 1;
        if ((reinterpret_cast<uintptr_t>(g.grad) | reinterpret_cast<uintptr_t>(g.out)) & own) return GS_ERR_ALIGN;
        any |= g.out != nullptr;
        all &= g.out != nullptr;
    }
    if (any && !all) return GS_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return GS_ERR_NO_DEVICE;
    const cudaError_t e = gs::launch_clip(ctx, grads, n_tensors, max_norm, any, out_norm, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? GS_OK : cuda_fail(ctx, e);
}

}  // extern "C"
