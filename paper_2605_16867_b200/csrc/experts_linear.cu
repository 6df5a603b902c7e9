// Products with the experts' weights:
//   forward   y[r]  = act(x[t(r)] W_e^T + b_e)         per row r of expert e
//   backward  dx[r] = dz[r] W_e  (zero where x[t(r)] <= 0),   dW_e = sum_r dz[r]^T x[t(r)],   db_e = sum_r dz[r]
// Plain tiles: 64 x 64 results per CTA, sixteen of the contraction at a time through shared memory.
#include "operators.cuh"

namespace gs {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

// Tile t of all experts' row tiles: its expert and its rows; false past the last.
__device__ __forceinline__ bool row_tile(const int32_t *__restrict__ offsets, int n_experts, int n_rows, int t,
                                         int *expert, int2 *rows) {
    for (int e = 0; e < n_experts; ++e) {
        const int2 r = expert_rows(offsets, e, n_rows);
        const int tiles = (r.y - r.x + kTile - 1) / kTile;
        if (t < tiles) { *expert = e; *rows = make_int2(r.x + t * kTile, min(r.x + (t + 1) * kTile, r.y)); return true; }
        t -= tiles;
    }
    return false;
}

// kBackward: out = dz W_e (contraction over w's rows); else out = x W_e^T
template <typename T, bool kBackward>
__global__ void __launch_bounds__(kThreads)
rows_kernel(const T *__restrict__ a, int64_t ld_a, const int32_t *__restrict__ a_row, int n_a_rows,
            const int32_t *__restrict__ offsets, int n_experts, int n_rows, const T *__restrict__ w, int64_t ld_w,
            int w_rows, int depth, int cols, const float *__restrict__ bias, bool relu,
            const T *__restrict__ mask, int64_t ld_mask, const int32_t *__restrict__ mask_row, int n_mask_rows,
            T *__restrict__ out, int64_t ld_out, unsigned *__restrict__ status)
{
    __shared__ float sa[kDepth][kTile + 1], sw[kDepth][kTile + 1];
    dependent_begin();
    int e;
    int2 rows;
    if (!row_tile(offsets, n_experts, n_rows, blockIdx.x, &e, &rows)) return;
    const int col0 = blockIdx.y * kTile;
    const T *we = w + (int64_t)e * w_rows * ld_w;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    bool bad = false;
    for (int k0 = 0; k0 < depth; k0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
            const int r = i / kDepth, k = k0 + i % kDepth;
            float v = 0.f;
            if (rows.x + r < rows.y && k < depth) {
                int src = rows.x + r;
                if (a_row) {
                    src = a_row[src];
                    if (src < 0 || src >= n_a_rows) { bad = true; src = min(max(src, 0), n_a_rows - 1); }
                }
                v = to_float(a[src * ld_a + k]);
            }
            sa[i % kDepth][r] = v;
            const int c = col0 + r;
            sw[i % kDepth][r] = c < cols && k < depth ? to_float(kBackward ? we[k * ld_w + c] : we[c * ld_w + k]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty * 4 + i], sw[k][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int r = rows.x + ty * 4 + i, c = col0 + tx * 4 + j;
            if (r >= rows.y || c >= cols) continue;
            float v = acc[i][j];
            if (bias) v += bias[(int64_t)e * cols + c];
            if (relu) v = v > 0.f || v != v ? v : 0.f;
            if (mask) {
                const int m = mask_row ? min(max(mask_row[r], 0), n_mask_rows - 1) : r;
                if (!(to_float(mask[m * ld_mask + c]) > 0.f)) v = 0.f;
            }
            out[r * ld_out + c] = from_float<T>(v);
        }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

// One expert's dW tile; the first column tile also leaves db.
template <typename T>
__global__ void __launch_bounds__(kThreads)
weights_kernel(const T *__restrict__ dz, int64_t ld_dz, const T *__restrict__ x, int64_t ld_x,
               const int32_t *__restrict__ x_row, int n_x_rows, const int32_t *__restrict__ offsets, int n_rows,
               int n_out, int n_in, float *__restrict__ dw, int64_t ld_dw, float *__restrict__ db, unsigned *__restrict__ status)
{
    __shared__ float sa[kDepth][kTile + 1], sw[kDepth][kTile + 1];
    dependent_begin();
    const int e = blockIdx.z, out0 = blockIdx.y * kTile, in0 = blockIdx.x * kTile;
    const int2 rows = expert_rows(offsets, e, n_rows);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    // (two levels of sums: one float that takes tens of thousands of terms in turn loses several bits)
    float acc[4][4] = {}, bias[4] = {}, acc2[4][4] = {}, bias2[4] = {};
    bool bad = false;
    for (int r0 = rows.x; r0 < rows.y; r0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
            const int r = r0 + i / kTile, c = i % kTile;
            float v = 0.f, u = 0.f;
            if (r < rows.y) {
                if (out0 + c < n_out) v = to_float(dz[r * ld_dz + out0 + c]);
                int src = r;
                if (x_row) {
                    src = x_row[src];
                    if (src < 0 || src >= n_x_rows) { bad = true; src = min(max(src, 0), n_x_rows - 1); }
                }
                if (in0 + c < n_in) u = to_float(x[src * ld_x + in0 + c]);
            }
            sa[i / kTile][c] = v;
            sw[i / kTile][c] = u;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v = sa[k][ty * 4 + i];
                bias[i] += v;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(v, sw[k][tx * 4 + j], acc[i][j]);
            }
        __syncthreads();
        if ((r0 - rows.x) % 512 == 512 - kDepth || r0 + kDepth >= rows.y)
            for (int i = 0; i < 4; ++i) {
                bias2[i] += bias[i];
                bias[i] = 0.f;
                for (int j = 0; j < 4; ++j) { acc2[i][j] += acc[i][j]; acc[i][j] = 0.f; }
            }
    }
    for (int i = 0; i < 4; ++i) {
        const int o = out0 + ty * 4 + i;
        if (o >= n_out) continue;
        if (db && in0 == 0 && tx == 0) db[(int64_t)e * n_out + o] = bias2[i];
        for (int j = 0; j < 4; ++j)
            if (in0 + tx * 4 + j < n_in) dw[((int64_t)e * n_out + o) * ld_dw + in0 + tx * 4 + j] = acc2[i][j];
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename T> cudaError_t forward_as(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.n_rows + kTile - 1) / kTile + a.n_experts), (a.out + kTile - 1) / kTile);
    LaunchTimer t(ctx, GS_K_EXPERT_LINEAR, st);
    return launch_dependent(rows_kernel<T, false>, grid, dim3(kThreads), 0, st, (const T *)a.x, a.ld_x, a.row_token,
                            (int)a.n_x_rows, a.offsets, a.n_experts, (int)a.n_rows, (const T *)a.w, a.ld_w, a.out, a.in,
                            a.out, a.bias, (a.flags & GS_EXPERT_RELU) != 0, (const T *)nullptr, (int64_t)0, (const int32_t *)nullptr, 0,
                            (T *)a.y, a.ld_y, ctx->s.status);
}

template <typename T> cudaError_t dx_as(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.n_rows + kTile - 1) / kTile + a.n_experts), (a.in + kTile - 1) / kTile);
    const bool masked = a.flags & GS_EXPERT_RELU_INPUT;
    LaunchTimer t(ctx, GS_K_EXPERT_LINEAR, st);
    return launch_dependent(rows_kernel<T, true>, grid, dim3(kThreads), 0, st, (const T *)a.dz, a.ld_dz, (const int32_t *)nullptr,
                            0, a.offsets, a.n_experts, (int)a.n_rows, (const T *)a.w, a.ld_w, a.out, a.out,
                            a.in, (const float *)nullptr, false, masked ? (const T *)a.x : (const T *)nullptr, a.ld_x, a.row_token, (int)a.n_x_rows,
                            (T *)a.dx, a.ld_dx, ctx->s.status);
}

template <typename T> cudaError_t dw_as(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    const dim3 grid((a.in + kTile - 1) / kTile, (a.out + kTile - 1) / kTile, a.n_experts);
    LaunchTimer t(ctx, GS_K_EXPERT_LINEAR, st);
    return launch_dependent(weights_kernel<T>, grid, dim3(kThreads), 0, st, (const T *)a.dz, a.ld_dz, (const T *)a.x, a.ld_x,
                            a.row_token, (int)a.n_x_rows, a.offsets, (int)a.n_rows, a.out, a.in, a.dw, a.ld_dw, a.db, ctx->s.status);
}

}  // namespace

cudaError_t configure_expert_linear() { return cudaSuccess; }
int64_t expert_linear_workspace(const gs_ctx *, int, int64_t, int, int) { return 0; }

cudaError_t launch_expert_linear(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? forward_as<__nv_bfloat16>(ctx, a, st) : forward_as<__half>(ctx, a, st);
}
cudaError_t launch_expert_linear_dx(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? dx_as<__nv_bfloat16>(ctx, a, st) : dx_as<__half>(ctx, a, st);
}
cudaError_t launch_expert_linear_dw(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? dw_as<__nv_bfloat16>(ctx, a, st) : dw_as<__half>(ctx, a, st);
}

}  // namespace gs
