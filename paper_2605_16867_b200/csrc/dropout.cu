// Dropout with a residual.  Which values stay is computed from a counter-based generator (Philox-4x32 with ten
// rounds, Salmon et al. 2011), so no mask is stored and the gradient is the same call.
//
// A lane takes eight columns, 16 bytes of 16-bit values: one turn of the generator gives 128 bits, sixteen for
// each of them (p then has steps of 2^-16; with a whole word for every value the generator's instructions, twice as
// many, would bound the kernel and not memory: they take 58 % of the issue slots as it is).  Bound by memory: 131,072 x 1024 in
// 16 bits with a residual 137 us = 5.9 TB/s, 90 % of a plain copy's rate (65,536 x 1024 in 32 bits 116 us = 6.9 TB/s).  Rows that are
// not whole blocks of eight long take two turns a block, since the words of most blocks lie in two counters: the generator's
// instructions bound them (131,072 x 1001 280 us, 65,536 x 1001 in 32 bits 142 us); rows with gaps between them take 169 us.
#include "operators.cuh"
#include "pairs.cuh"

namespace gs {
namespace {

constexpr int kThreads = 256;

// The generator's four words for a counter.
__device__ __forceinline__ uint4 philox(uint64_t counter, uint64_t place, uint64_t seed) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)place, c3 = (uint32_t)(place >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// The words of eight values from number i on, two halves each.  They begin inside a counter's 128 bits where i is no
// multiple of eight: then they end in the next one's.
template <bool kAligned>
__device__ __forceinline__ uint4 words_from(uint64_t i, uint64_t place, uint64_t seed) {
    const uint4 w = philox(i >> 3, place, seed);
    const unsigned skip = kAligned ? 0u : (unsigned)i & 7u;
    if (skip == 0) return w;
    const uint4 n = philox((i >> 3) + 1, place, seed);
    const uint32_t all[8] = {w.x, w.y, w.z, w.w, n.x, n.y, n.z, n.w};
    uint32_t r[5];                               // from word skip / 2 on
#pragma unroll
    for (int j = 0; j < 5; ++j) {
        r[j] = all[j];
#pragma unroll
        for (unsigned s = 1; s < 4; ++s) if (skip >> 1 == s) r[j] = all[j + s < 8 ? j + s : 7];
    }
    const unsigned bits = (skip & 1u) * 16;
    return make_uint4(__funnelshift_r(r[0], r[1], bits), __funnelshift_r(r[1], r[2], bits), __funnelshift_r(r[2], r[3], bits), __funnelshift_r(r[3], r[4], bits));
}

// Block i of eight columns, its neighbours in the words' order at i * 8: rows that follow each other without a gap and are
// whole blocks long are one long row (kFlat); else a block's row takes a division, a short one after the CTA's first.
constexpr int kEach = 2;                        // (four: 112 registers, half as many warps, 266 instead of 137 us)

template <typename T, bool kResidual, bool kFlat>
__global__ void __launch_bounds__(kThreads, 4)
dropout_kernel(const DropoutArgs p, unsigned blocks, int64_t all)
{
    dependent_wait();
    const int64_t first = (int64_t)blockIdx.x * (kThreads * kEach);
    const int64_t row0 = kFlat ? 0 : first / blocks;
    const unsigned block0 = kFlat ? 0 : (unsigned)(first - row0 * blocks);
    Eight<T> x[kEach], r[kEach];
    int64_t row[kEach];
    int col[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const unsigned at = block0 + j * kThreads + threadIdx.x;
        const int64_t i = first + j * kThreads + threadIdx.x;
        if (kFlat) { row[j] = i < all ? i : -1; col[j] = 0; }            // (a "row" of eight columns)
        else {
            const unsigned over = at / blocks;
            row[j] = i < all ? row0 + over : -1;
            col[j] = (int)(at - over * blocks) * 8;
        }
        if (row[j] < 0) continue;
        x[j].template ask<false>((const T *)p.x + row[j] * (kFlat ? 8 : p.ld_x), col[j], kFlat ? 8 : p.features);
        if (kResidual) r[j].template ask<false>((const T *)p.residual + row[j] * (kFlat ? 8 : p.ld_residual), col[j], kFlat ? 8 : p.features);
    }
    const uint64_t seed = (uint64_t)p.rng[0], place = (uint64_t)p.rng[1];
    const float2 factor = both(65536.f / (float)(65536u - p.cut));
    const unsigned cut_high = p.cut << 16;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if (row[j] < 0) break;
        const uint4 w = words_from<kFlat>((uint64_t)row[j] * (kFlat ? 8 : p.features) + col[j], place, seed);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (a half in the upper place is compared where it is: what lies below it changes nothing)
            float2 y = mul2(two(x[j], i), factor);
            if (word[i] << 16 < cut_high) y.x = 0.f;
            if (word[i] < cut_high) y.y = 0.f;
            if (kResidual) y = add2(y, two(r[j], i));
            v[2 * i] = y.x;
            v[2 * i + 1] = y.y;
        }
        store8((T *)p.out + row[j] * (kFlat ? 8 : p.ld_out), col[j], kFlat ? 8 : p.features, v);
    }
    dependent_end();
}

template <typename T> cudaError_t dropout_as(gs_ctx *ctx, const DropoutArgs &a, cudaStream_t st) {
    const bool flat = a.features % 8 == 0 && a.ld_x == a.features && a.ld_out == a.features && (!a.residual || a.ld_residual == a.features);
    const int64_t blocks = (a.features + 7) / 8, all = a.n_rows * blocks, ctas = (all + kThreads * kEach - 1) / (kThreads * kEach);
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    const auto kernel = a.residual ? flat ? dropout_kernel<T, true, true> : dropout_kernel<T, true, false>
                                   : flat ? dropout_kernel<T, false, true> : dropout_kernel<T, false, false>;
    LaunchTimer t(ctx, GS_K_DROPOUT, st);
    return launch_dependent(kernel, dim3((unsigned)ctas), dim3(kThreads), 0, st, a, (unsigned)blocks, all);
}

}  // namespace

cudaError_t launch_dropout(gs_ctx *ctx, const DropoutArgs &a, cudaStream_t st) {
    if (a.dtype == GS_F32) return dropout_as<float>(ctx, a, st);
    return a.dtype == GS_BF16 ? dropout_as<__nv_bfloat16>(ctx, a, st) : dropout_as<__half>(ctx, a, st);
}

}  // namespace gs
