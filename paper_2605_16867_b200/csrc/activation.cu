// dz = act'(z) d_out, where no layer above has done it in its own gradient.  Bound by memory: 131,072 x 1024 in 16 bits, ReLU 139 us =
// 5.8 TB/s, SiLU 131 us = 6.1 TB/s, GELU 156 us = 5.2 TB/s.  333 x 250: 6.5 us, the call.
#include "activation.cuh"
#include "operators.cuh"

namespace gs {
namespace {

constexpr int kThreads = 256;

template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads)
activation_backward_kernel(const ActivationArgs p)
{
    dependent_wait();
    const ActFactors factors(kAct);
    const int blocks = (p.features + 7) / 8;
    const int64_t all = p.n_rows * blocks, stride = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += stride) {
        const int64_t row = i / blocks;
        const int col = (int)(i - row * blocks) * 8;
        Eight<T> d, z;
        d.template ask<false>((const T *)p.d_out + row * p.ld_d_out, col, p.features);
        z.template ask<false>((const T *)p.z + row * p.ld_z, col, p.features);
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 dz = mul2(unpack2<T>(reinterpret_cast<const uint32_t *>(d.q)[j]), slope<kAct, T>(factors, reinterpret_cast<const uint32_t *>(z.q)[j]));
            v[2 * j] = dz.x;
            v[2 * j + 1] = dz.y;
        }
        store8((T *)p.dz + row * p.ld_dz, col, p.features, v);
    }
    dependent_end();
}

template <typename T> cudaError_t backward_as(gs_ctx *ctx, const ActivationArgs &a, cudaStream_t st) {
    const int64_t want = (a.n_rows * ((a.features + 7) / 8) + kThreads - 1) / kThreads, most = (int64_t)ctx->n_sm * 8;
    const auto kernel = a.activation == GS_ACT_RELU ? activation_backward_kernel<T, GS_ACT_RELU>
                      : a.activation == GS_ACT_GELU ? activation_backward_kernel<T, GS_ACT_GELU>
                      : a.activation == GS_ACT_SILU ? activation_backward_kernel<T, GS_ACT_SILU> : activation_backward_kernel<T, GS_ACT_NONE>;
    LaunchTimer t(ctx, GS_K_LINEAR, st);
    return launch_dependent(kernel, dim3((unsigned)(want < most ? want : most)), dim3(kThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_activation_backward(gs_ctx *ctx, const ActivationArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? backward_as<__nv_bfloat16>(ctx, a, st) : backward_as<__half>(ctx, a, st);
}

}  // namespace gs
