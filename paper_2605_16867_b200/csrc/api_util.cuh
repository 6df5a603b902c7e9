// What every entry point of the C ABI uses: pointer checks, error bookkeeping, the current device.
#pragma once

#include "gs_internal.cuh"

namespace gs {

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

inline int cuda_fail(gs_ctx *ctx, cudaError_t e) {
    if (ctx) ctx->last_cuda_error = (int)e;
    return GS_ERR_CUDA;
}

// Makes the context's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
        if (prev == dev) prev = -1;
    }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

}  // namespace gs
