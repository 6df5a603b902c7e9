// Global gradient norm over many tensors, and clipping by it.
//   norm = sqrt(sum g^2);   out = g * min(1, max_norm / (norm + 1e-6))
// Bound by memory: one read of everything for the norm, one read and one write for the clipping
// (the read comes from L2 as far as the gradients fit).  Squares are added in float over 16 bytes (four or
// eight values: 2^-22 of the norm at most, and roundings to both sides) and in double from there on; where
// the sum of those few is outside what a float holds well (1e-24 to 1e38), in double from the start.  Every CTA leaves one
// partial sum, which the next launch adds in a fixed order, so the norm is the same every time.  268 M elements, most
// of them in 16 bits (0.55 GB): 305 us for 1.64 GB moved, 5.4 TB/s; in 32 bits 527 us for 3.2 GB, 6.1 TB/s.
#include "operators.cuh"

namespace gs {
namespace {

constexpr int kClipThreads = 512;
constexpr int kClipTensors = 256;                    // tensors of one launch at most (their table travels as a kernel argument,
constexpr int kClipFew = 32;                         //  and a short one travels faster)
constexpr int kClipChunk = 16384;                    // elements that a CTA takes at a time

template <int kMost> struct ClipTable {
    int n;
    int chunk_start[kMost + 1];                      // chunks before each tensor
    const void *grad[kMost];
    void *out[kMost];
    int64_t n_elements[kMost];
    unsigned char dtype[kMost];
};

template <int kMost>
__device__ __forceinline__ int tensor_of(const ClipTable<kMost> &t, int chunk) {
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.chunk_start[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Sixteen bytes of T.
template <typename T> struct Pack {
    static constexpr int kN = 16 / (int)sizeof(T);
    uint4 q;
    __device__ __forceinline__ float at(int i) const { return to_float(reinterpret_cast<const T *>(&q)[i]); }
    __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T *>(&q)[i] = from_float<T>(v); }
};

// Squares of 16 bytes of gradients.  A float holds their sum unless it is very large, very small or
// not a number; then the squares are taken in double (a conversion per value is what would bound
// the kernel otherwise).
template <typename T>
__device__ __forceinline__ double pack_square(const Pack<T> &g) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < Pack<T>::kN; ++i) sum = fmaf(g.at(i), g.at(i), sum);
    if ((sum >= 1e-24f && sum <= 1e38f) || (g.q.x | g.q.y | g.q.z | g.q.w) == 0u) return (double)sum;
    double wide = 0.0;
#pragma unroll
    for (int i = 0; i < Pack<T>::kN; ++i) wide = fma((double)g.at(i), (double)g.at(i), wide);
    return wide;
}

// Elements before the first 16-byte boundary.
template <typename T>
__device__ __forceinline__ int to_boundary(const T *p, int n) {
    return min((int)(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(T)), n);
}

template <typename T>
__device__ __forceinline__ double chunk_square(const T *__restrict__ g, int n) {
    constexpr int kN = Pack<T>::kN, kAhead = 2;      // (16 bytes each; at 268 M elements 1 / 2 / 3 / 4 / 8 of them, here and in chunk_scale, take 360 / 300 / 325 / 415 / 655 us)
    const int head = to_boundary(g, n), packs = (n - head) / kN, tail = head + packs * kN;
    const uint4 *q = reinterpret_cast<const uint4 *>(g + head);
    double sum = 0.0;
    for (int i = threadIdx.x; i < packs; i += kAhead * kClipThreads) {
        Pack<T> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            v[k].q = i + k * kClipThreads < packs ? __ldg(q + i + k * kClipThreads) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) sum += pack_square(v[k]);
    }
    const int edge = (int)threadIdx.x < head ? (int)threadIdx.x : tail + (int)threadIdx.x - head;
    if (edge < n) { const double v = (double)to_float(g[edge]); sum = fma(v, v, sum); }
    return sum;
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T *g, T *out, int n, float f) {
    constexpr int kN = Pack<T>::kN, kAhead = 2;
    if (((reinterpret_cast<uintptr_t>(g) ^ reinterpret_cast<uintptr_t>(out)) & 15) != 0) {
        for (int i = threadIdx.x; i < n; i += kClipThreads) out[i] = from_float<T>(to_float(g[i]) * f);
        return;
    }
    const int head = to_boundary(g, n), packs = (n - head) / kN, tail = head + packs * kN;
    const uint4 *q = reinterpret_cast<const uint4 *>(g + head);
    uint4 *o = reinterpret_cast<uint4 *>(out + head);
    for (int i = threadIdx.x; i < packs; i += kAhead * kClipThreads) {
        Pack<T> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) if (i + k * kClipThreads < packs) v[k].q = q[i + k * kClipThreads];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
#pragma unroll
            for (int j = 0; j < kN; ++j) v[k].set(j, v[k].at(j) * f);
            if (i + k * kClipThreads < packs) o[i + k * kClipThreads] = v[k].q;
        }
    }
    const int edge = (int)threadIdx.x < head ? (int)threadIdx.x : tail + (int)threadIdx.x - head;
    if (edge < n) out[edge] = from_float<T>(to_float(g[edge]) * f);
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[kClipThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < kClipThreads / 32; ++w) sum += part[w];
    __syncthreads();
    return sum;
}

template <int kMost>
__global__ void __launch_bounds__(kClipThreads, 2)
norm_kernel(const __grid_constant__ ClipTable<kMost> t, double *__restrict__ partials)
{
    dependent_begin();
    double sum = 0.0;
    for (int c = blockIdx.x; c < t.chunk_start[t.n]; c += gridDim.x) {
        const int k = tensor_of(t, c);
        const int64_t first = (int64_t)(c - t.chunk_start[k]) * kClipChunk;
        const int n = (int)min((int64_t)kClipChunk, t.n_elements[k] - first);
        if (t.dtype[k] == GS_F32) sum += chunk_square((const float *)t.grad[k] + first, n);
        else if (t.dtype[k] == GS_BF16) sum += chunk_square((const __nv_bfloat16 *)t.grad[k] + first, n);
        else sum += chunk_square((const __half *)t.grad[k] + first, n);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

// The factor, from all partial sums (every CTA adds them in the same order).
__device__ __forceinline__ float clip_factor(const double *__restrict__ partials, int n_partials, float max_norm,
                                             float *out_norm, unsigned *status) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_partials; i += kClipThreads) sum += partials[i];
    const float norm = (float)sqrt(block_sum(sum));
    const bool finite = norm <= 3.402823466e38f;
    if (blockIdx.x == 0 && threadIdx.x == 0 && out_norm) {
        *out_norm = norm;
        if (!finite) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
    }
    return finite ? fminf(1.f, max_norm / (norm + 1e-6f)) : 1.f;
}

template <int kMost>
__global__ void __launch_bounds__(kClipThreads, 2)
clip_kernel(const __grid_constant__ ClipTable<kMost> t, const double *__restrict__ partials, int n_partials, float max_norm,
            float *__restrict__ out_norm, unsigned *__restrict__ status)
{
    dependent_begin();
    const float f = clip_factor(partials, n_partials, max_norm, out_norm, status);
    // the other way round: what the norm read last is still in L2
    for (int c = t.chunk_start[t.n] - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const int k = tensor_of(t, c);
        if (f == 1.f && t.grad[k] == t.out[k]) continue;
        const int64_t first = (int64_t)(c - t.chunk_start[k]) * kClipChunk;
        const int n = (int)min((int64_t)kClipChunk, t.n_elements[k] - first);
        if (t.dtype[k] == GS_F32) chunk_scale((const float *)t.grad[k] + first, (float *)t.out[k] + first, n, f);
        else if (t.dtype[k] == GS_BF16) chunk_scale((const __nv_bfloat16 *)t.grad[k] + first, (__nv_bfloat16 *)t.out[k] + first, n, f);
        else chunk_scale((const __half *)t.grad[k] + first, (__half *)t.out[k] + first, n, f);
    }
}

template <int kMost>
cudaError_t launch_tables(gs_ctx *ctx, const gs_grad *grads, int n_tensors, float max_norm, bool write, float *out_norm, cudaStream_t st)
{
    // pass 0: partial sums of every table; pass 1: the factor and the values
    double *partials = operator_scratch(ctx).clip_partials;
    const int n_tables = n_tensors > kMost ? (n_tensors + kMost - 1) / kMost : 1;
    int per_table = kMaxClipCtas / n_tables;
    if (per_table > ctx->n_sm * 2) per_table = ctx->n_sm * 2;        // as many as are resident
    if (per_table < 1) return cudaErrorInvalidValue;
    int n_partials = 0;
    for (int pass = 0; pass < 2; ++pass) {
        for (int table = 0; table < n_tables; ++table) {
            if (pass == 1 && !write && table > 0) break;
            ClipTable<kMost> t;
            t.n = 0;
            t.chunk_start[0] = 0;
            int64_t chunks = 0;
            const int last = n_tensors < (table + 1) * kMost ? n_tensors : (table + 1) * kMost;
            for (int i = table * kMost; i < last && (pass == 0 || write); ++i) {
                if (grads[i].n_elements == 0) continue;
                t.grad[t.n] = grads[i].grad;
                t.out[t.n] = grads[i].out;
                t.n_elements[t.n] = grads[i].n_elements;
                t.dtype[t.n] = (unsigned char)grads[i].dtype;
                chunks += (grads[i].n_elements + kClipChunk - 1) / kClipChunk;
                if (chunks > INT32_MAX) return cudaErrorInvalidValue;
                t.chunk_start[++t.n] = (int)chunks;
            }
            const int ctas = chunks < 1 ? 1 : chunks < per_table ? (int)chunks : per_table;
            LaunchTimer timer(ctx, GS_K_CLIP, st);
            cudaError_t e;
            if (pass == 0) {
                e = launch_dependent(norm_kernel<kMost>, dim3(ctas), dim3(kClipThreads), 0, st, t, partials + n_partials);
                n_partials += ctas;
            } else {
                e = launch_dependent(clip_kernel<kMost>, dim3(ctas), dim3(kClipThreads), 0, st, t, (const double *)partials,
                                     n_partials, max_norm, table == 0 ? out_norm : nullptr, ctx->s.status);
            }
            if (e != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_clip(gs_ctx *ctx, const gs_grad *grads, int n_tensors, float max_norm, bool write,
                        float *out_norm, cudaStream_t st)
{
    return n_tensors <= kClipFew ? launch_tables<kClipFew>(ctx, grads, n_tensors, max_norm, write, out_norm, st)
                                 : launch_tables<kClipTensors>(ctx, grads, n_tensors, max_norm, write, out_norm, st);
}

}  // namespace gs
