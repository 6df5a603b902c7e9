// Token embeddings and their gradient.
//   out[i] = scale * table[id(i)];      d_table[v] = scale * sum of d_out[i] over the tokens i with id(i) = v
//
// The lookup is bound by memory: a group of lanes copies a row, 16 bytes a load, and what it writes leaves the L2 cache
// to the table.  524,288 tokens of 131,072, 1024 wide in 16 bits: 245 us = 5.3 TB/s of what DRAM moves (1.29 GB; a plain copy
// reaches 6.5).
//
// The gradient adds rows up by token without atomics.  The tokens' places are sorted by token number (a
// stable counting sort of nine bits a pass), so that a token's rows are one run of the sorted list; the list is cut
// into pieces of equal length, a group of lanes adds up a piece's rows, and writes a run that lies inside the
// piece to the table.  What a run leaves in a piece that it crosses the border of goes to the workspace, and
// a last kernel adds those parts in order: however frequent a token is, the work is dealt out evenly,
// and the sums' order depends on the sizes alone.  Bound by memory: d_out is read once, d_table written once (rows
// without a token are found by bisection of the sorted list and zeroed by blocks beside those that add).  The same
// tokens: 395 us, of it 53 for the order (two passes), 300 for the sums (1.62 GB at 5.3 TB/s) and 23 for the runs across pieces.
#include <type_traits>

#include "operators.cuh"
#include "pairs.cuh"

namespace gs {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;

// ---- lookup -----------------------------------------------------------------------------------

constexpr int kLookupThreads = 256, kLookupBlocks = 4;      // of eight columns that a lane has under way

template <typename T> constexpr int kLookupCtas = sizeof(T) == 4 ? 4 : 6;       // of an SM, all at once

template <typename T, int kLanes>
__global__ void __launch_bounds__(kLookupThreads, kLookupCtas<T>)
embedding_kernel(const T *__restrict__ table, int vocabulary, int64_t ld_table, const int32_t *__restrict__ ids, int64_t n_tokens,
                 int features, float scale, T *__restrict__ out, int64_t ld_out, unsigned *__restrict__ status)
{
    dependent_wait();
    const int part = threadIdx.x % kLanes;
    const int64_t step = (int64_t)gridDim.x * (kLookupThreads / kLanes);
    int64_t n = ((int64_t)blockIdx.x * kLookupThreads + threadIdx.x) / kLanes;
    int next = n < n_tokens ? ids[n] : -1;
    const int last = (features - 1) / 8 * 8;                     // the last block of eight columns
    const float2 factor = both(scale);
    bool bad = false;
    for (; n < n_tokens; n += step) {
        const int id = next;
        next = n + step < n_tokens ? ids[n + step] : -1;
        const bool there = (unsigned)id < (unsigned)vocabulary;
        bad |= !there && id != -1;
        const T *row = table + (there ? id : 0) * ld_table;      // (a row that is read for nothing: no branch around the loads)
        for (int col0 = part * 8; col0 < features; col0 += kLanes * 8 * kLookupBlocks) {
            Eight<T> q[kLookupBlocks];
#pragma unroll
            for (int b = 0; b < kLookupBlocks; ++b) q[b].ask(row, min(col0 + b * kLanes * 8, last), features);
#pragma unroll
            for (int b = 0; b < kLookupBlocks; ++b) {
                const int col = col0 + b * kLanes * 8;
                float v[8];
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) if (!there) q[b].q[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 y = mul2(two(q[b], i), factor);
                    v[2 * i] = y.x;
                    v[2 * i + 1] = y.y;
                }
                if (col < features) store8<true>(out + n * ld_out, col, features, v);
            }
        }
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
    dependent_end();
}

// ---- order of the tokens ------------------------------------------------------------------------

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortEach = 4, kSortTile = kSortThreads * kSortEach;
constexpr int kMaxBits = 9, kMaxBins = 1 << kMaxBits;
constexpr size_t kSortSmem = sizeof(int) * kMaxBins * (kSortWarps + 2);
constexpr int kMaxSortCtas = 148;
constexpr int64_t kOneCtaTokens = 2 * kSortTile;           // so many are sorted by one CTA in one launch

struct SortArgs {
    const int32_t *ids;
    int *keys[2], *places[2];
    int *counts;                    // [CTAs][bins]
    int64_t n, per;                 // tokens in all, and of each CTA (a multiple of the tile)
    int vocabulary, bits, passes;
    unsigned *status;
};

// Token number of place i as a sort key: what is in no row sorts behind all rows.
__device__ __forceinline__ int key_at(const SortArgs &p, int pass, int64_t i, bool *bad) {
    if (pass > 0) return p.keys[(pass - 1) & 1][i];
    const int id = p.ids[i];
    if ((unsigned)id < (unsigned)p.vocabulary) return id;
    *bad |= id != -1;
    return p.vocabulary;
}

// Lanes that hold the same digit (of `bits` bits; `in`: it counts), and how many of them come before this one.
__device__ __forceinline__ int rank_among(int digit, int bits, bool in, unsigned lanes_before, unsigned *peers) {
    unsigned same = __ballot_sync(kFull, in);
#pragma unroll
    for (int b = 0; b < kMaxBits; ++b) {
        if (b >= bits) break;
        const bool one = digit >> b & 1;
        const unsigned ones = __ballot_sync(kFull, one);
        same &= one ? ones : ~ones;
    }
    *peers = same;
    return __popc(same & lanes_before);
}

// Digits of the tokens [first, last) counted into shared memory.
__device__ __forceinline__ void count_digits(const SortArgs &p, int pass, int64_t first, int64_t last, int *counts, bool *bad) {
    const int bins = 1 << p.bits, shift = pass * p.bits;
    for (int d = threadIdx.x; d < bins; d += kSortThreads) counts[d] = 0;
    __syncthreads();
    for (int64_t i0 = first; i0 < last; i0 += kSortThreads) {
        const int64_t i = i0 + threadIdx.x;
        if (i < last) atomicAdd(&counts[(key_at(p, pass, i, bad) >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
}

// total[d] becomes the sum of the totals before d (all threads; kSortThreads >= kMaxBins).
__device__ __forceinline__ void scan_bins(int *total, int bins, int *warp_sums) {
    const int d = threadIdx.x, lane = d & 31;
    const int own = d < bins ? total[d] : 0;
    int sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kFull, sum, o);
        if (lane >= o) sum += up;
    }
    if (lane == 31) warp_sums[d >> 5] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < d >> 5 && w < kMaxBins / 32; ++w) before += warp_sums[w];
    if (d < bins) total[d] = before + sum - own;
    __syncthreads();
}

// Tokens [first, last) to their places after this pass; base[d]: where this CTA's first token of digit d goes.
// Stable: warps, rounds and lanes take the tokens in order.
__device__ __forceinline__ void place_tokens(const SortArgs &p, int pass, int64_t first, int64_t last, int *base, int *hist) {
    const int bins = 1 << p.bits, shift = pass * p.bits, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned lanes_before = (1u << lane) - 1;
    int *own = hist + warp * bins;
    bool bad = false;
    for (int64_t tile = first; tile < last; tile += kSortTile) {
        for (int i = threadIdx.x * 4; i < bins * kSortWarps; i += kSortThreads * 4) *reinterpret_cast<int4 *>(hist + i) = make_int4(0, 0, 0, 0);
        __syncthreads();
        int key[kSortEach], at[kSortEach], rank[kSortEach];
        const int64_t i0 = tile + warp * 32 * kSortEach + lane;
#pragma unroll
        for (int j = 0; j < kSortEach; ++j) {
            const int64_t i = i0 + j * 32;
            key[j] = i < last ? key_at(p, pass, i, &bad) : -1;
            at[j] = i < last ? pass > 0 ? p.places[(pass - 1) & 1][i] : (int)i : 0;
        }
#pragma unroll
        for (int j = 0; j < kSortEach; ++j) {
            const bool in = key[j] >= 0;
            const int digit = (key[j] >> shift) & (bins - 1);
            unsigned peers;
            const int before = rank_among(digit, p.bits, in, lanes_before, &peers);
            rank[j] = own[digit] + before;
            __syncwarp();
            if (in && before == 0) own[digit] += __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        for (int d = threadIdx.x; d < bins; d += kSortThreads) {
            int run = base[d];
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) {
                const int here = hist[w * bins + d];
                hist[w * bins + d] = run;
                run += here;
            }
            base[d] = run;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortEach; ++j) {
            if (key[j] < 0) continue;
            const int to = own[(key[j] >> shift) & (bins - 1)] + rank[j];
            p.keys[pass & 1][to] = key[j];
            p.places[pass & 1][to] = at[j];
        }
        __syncthreads();
    }
}

// All passes by one CTA.
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(const SortArgs p)
{
    extern __shared__ int sort_smem[];
    int *hist = sort_smem, *base = hist + kMaxBins * kSortWarps, *sums = base + kMaxBins;
    dependent_begin();
    bool bad = false;
    for (int pass = 0; pass < p.passes; ++pass) {
        count_digits(p, pass, 0, p.n, base, &bad);
        scan_bins(base, 1 << p.bits, sums);
        place_tokens(p, pass, 0, p.n, base, hist);
    }
    if (bad) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs p, int pass)
{
    __shared__ int counts[kMaxBins];
    dependent_begin();
    bool bad = false;
    const int64_t first = blockIdx.x * p.per, last = first + p.per < p.n ? first + p.per : p.n;
    count_digits(p, pass, first, last, counts, &bad);
    for (int d = threadIdx.x; d < 1 << p.bits; d += kSortThreads) p.counts[((int64_t)blockIdx.x << p.bits) + d] = counts[d];
    if (bad) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
}

__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const SortArgs p, int pass)
{
    extern __shared__ int sort_smem[];
    int *hist = sort_smem, *base = hist + kMaxBins * kSortWarps, *sums = base + kMaxBins;
    dependent_begin();
    const int bins = 1 << p.bits, ctas = gridDim.x;
    // two threads (at least) a digit, each with its share of the CTAs' counts: all of them, and those before this CTA
    const int shares = kSortThreads / bins, d = threadIdx.x & (bins - 1), share = threadIdx.x >> p.bits;
    const int each = (ctas + shares - 1) / shares, c0 = min(share * each, ctas), c1 = min(c0 + each, ctas);
    int total = 0, before = 0;
#pragma unroll 16
    for (int c = c0; c < c1; ++c) {
        const int here = p.counts[((int64_t)c << p.bits) + d];
        total += here;
        before += c < (int)blockIdx.x ? here : 0;
    }
    if (threadIdx.x < bins) { base[d] = 0; hist[d] = 0; }
    __syncthreads();
    atomicAdd(&base[d], total);
    atomicAdd(&hist[d], before);
    __syncthreads();
    before = hist[d];
    scan_bins(base, bins, sums);
    if (threadIdx.x < bins) base[d] += before;
    __syncthreads();
    const int64_t first = blockIdx.x * p.per, last = first + p.per < p.n ? first + p.per : p.n;
    place_tokens(p, pass, first, last, base, hist);
}

// ---- sums ---------------------------------------------------------------------------------------

struct SumArgs {
    const void *d_out;
    int64_t ld_d_out;
    const int *keys, *places;
    int64_t n;
    int vocabulary, features, piece;            // piece: sorted places of a group of lanes
    int64_t n_pieces;
    float scale;
    float *d_table;
    int64_t ld_table;
    float *parts;                               // [pieces][2][features padded]: of a run that began before the piece, of one that goes on after it
    int part_ld;
    int zero_ctas, zero_parts;                  // CTAs that zero rows, warps that share 32 of them
};

constexpr int kSumThreads = 128;

__device__ __forceinline__ void store_part(float *to, int col, int features, const float (&v)[8]) {
    // (the workspace's rows are padded to whole blocks of eight)
    reinterpret_cast<float4 *>(to + col)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(to + col)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Rows of 32 table rows from `first` on that no token names: zeros, to every `parts`-th of them from `part` on.  By one warp.
__device__ __forceinline__ void zero_rows(const SumArgs &p, int64_t first, int part, int parts, int lane) {
    const int64_t row = first + lane;
    int64_t lo = 0, hi = p.n;                   // the first place whose key is not below the row
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (p.keys[mid] < row) lo = mid + 1;
        else hi = mid;
    }
    const bool none = row < p.vocabulary && lane % parts == part && !(lo < p.n && p.keys[lo] == row);
    for (unsigned left = __ballot_sync(kFull, none); left; left &= left - 1) {
        float *to = p.d_table + (first + __ffs(left) - 1) * p.ld_table;
        for (int col = lane * 4; col < p.features; col += 128) {
            if (col + 4 <= p.features) *reinterpret_cast<float4 *>(to + col) = make_float4(0.f, 0.f, 0.f, 0.f);
            else
                for (int i = col; i < p.features; ++i) to[i] = 0.f;
        }
    }
}

template <typename T, int kLanes>
__global__ void __launch_bounds__(kSumThreads, 8)
embedding_sum_kernel(const SumArgs p)
{
    dependent_wait();
    if ((int)blockIdx.x < p.zero_ctas) {         // (first, so that they are done before the others)
        const int64_t warps = (int64_t)p.zero_ctas * (kSumThreads / 32);
        if (blockIdx.y == 0)
            for (int64_t w = (int64_t)blockIdx.x * (kSumThreads / 32) + threadIdx.x / 32; w / p.zero_parts * 32 < p.vocabulary; w += warps)
                zero_rows(p, w / p.zero_parts * 32, (int)(w % p.zero_parts), p.zero_parts, threadIdx.x & 31);
        dependent_end();
        return;
    }
    constexpr int kAhead = 8 / sizeof(T);      // (more of them in flight take the registers of more warps: 16 bytes 319, these 296 us)
    const int col = (blockIdx.y * kLanes + threadIdx.x % kLanes) * 8;
    const int64_t piece = ((int64_t)(blockIdx.x - p.zero_ctas) * kSumThreads + threadIdx.x) / kLanes;
    const int64_t first = piece * p.piece, last = first + p.piece < p.n ? first + p.piece : p.n;
    if (first < p.n && col < p.features) {
        const T *d_out = (const T *)p.d_out;
        int key = p.keys[first];
        bool began_before = first > 0 && p.keys[first - 1] == key;
        float sum[8] = {};
        float *part = p.parts + piece * 2 * p.part_ld;
        const auto finish = [&](bool goes_on) {
            if (began_before) store_part(part, col, p.features, sum);
            else if (goes_on) store_part(part + p.part_ld, col, p.features, sum);
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] *= p.scale;
                store8(p.d_table + key * p.ld_table, col, p.features, sum);
            }
        };
        // keys and places of the next rows are asked for before these rows' values are waited for
        int k[kAhead], at[kAhead];
        const auto ask = [&](int64_t i) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const bool in = i + j < last;
                k[j] = in ? p.keys[i + j] : p.vocabulary;
                at[j] = in ? p.places[i + j] : 0;
            }
        };
        ask(first);
        for (int64_t i = first; i < last && key < p.vocabulary; i += kAhead) {
            Eight<T> v[kAhead];
            int here[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) { v[j].ask(d_out + at[j] * p.ld_d_out, col, p.features); here[j] = k[j]; }
            ask(i + kAhead);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (here[j] != key) {
                    if (key < p.vocabulary && i + j < last) finish(false);
                    if (i + j < last) {
                        key = here[j];
                        began_before = false;
                    }
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] = i + j < last ? 0.f : sum[c];
                }
                if (here[j] < p.vocabulary)
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] += v[j][c];
            }
        }
        if (key < p.vocabulary) finish(last < p.n && p.keys[last] == key);
    }
    dependent_end();
}

// Runs that cross the border of a piece: the part of the piece that they begin in, and those of the pieces that
// they go on in, in order.  A warp looks at one piece and adds up a run of few pieces, all columns; runs of more are left
// to other CTAs, which look at 64 pieces each for them and take 128 columns (eight stretches, then those).
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinFew = 4, kJoinGroup = 64;

// How many pieces after this one begin inside its last run: the next 32 are looked at, then 32 at equal distances up to
// the end of what is left, and so on.  By one warp.
__device__ __forceinline__ int pieces_after(const SumArgs &p, int64_t piece, int key, int lane) {
    int64_t lo = piece + 1, hi = p.n_pieces, apart = 1;      // the run holds the beginnings of the pieces before lo, not hi's
    while (lo < hi) {
        const int64_t at = lo + lane * apart;
        const unsigned same = __ballot_sync(kFull, at < hi && p.keys[at * p.piece] == key);
        const int held = same == kFull ? 32 : __ffs(~same) - 1;
        if (held < 32) hi = min(hi, lo + held * apart);
        if (held > 0) lo += (held - 1) * apart + 1;
        apart = (hi - lo + 31) / 32;
    }
    return (int)(lo - piece - 1);
}

__device__ __forceinline__ void add4(float4 &sum, const float4 &v) { sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w; }
__device__ __forceinline__ const float4 &part_at(const SumArgs &p, int64_t piece, int which, int col) {
    return *reinterpret_cast<const float4 *>(p.parts + (piece * 2 + which) * p.part_ld + col);
}
__device__ __forceinline__ void write_sum(const SumArgs &p, int key, int col, const float4 &s) {
    float *to = p.d_table + key * p.ld_table + col;
    const float v[4] = {s.x * p.scale, s.y * p.scale, s.z * p.scale, s.w * p.scale};
    if (col + 4 <= p.features) *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
    else
        for (int i = 0; i < 4; ++i) if (col + i < p.features) to[i] = v[i];
}
// Whether a run begins in a piece and goes on after it (its token: *key), and whether for more than kJoinFew pieces.
__device__ __forceinline__ bool goes_on(const SumArgs &p, int64_t piece, int *key, bool *many) {
    const int64_t first = piece * p.piece, last = first + p.piece, far = last + (int64_t)kJoinFew * p.piece;
    if (piece >= p.n_pieces || last >= p.n) return false;
    const int end = p.keys[last - 1], next = p.keys[last], begin = p.keys[first], before = first ? p.keys[first - 1] : -1, then = far < p.n ? p.keys[far] : -1;
    *key = end;
    *many = then == end;
    return end < p.vocabulary && next == end && (begin != end || before != end);
}

__global__ void __launch_bounds__(kJoinThreads)
embedding_join_kernel(const SumArgs p, int few_ctas, int slabs)
{
    __shared__ int list[kJoinGroup], n_list;
    __shared__ float4 stretches[kJoinWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) n_list = 0;
    dependent_begin();
    int key;
    bool many;
    if ((int)blockIdx.x < few_ctas) {
        const int64_t piece = (int64_t)blockIdx.x * kJoinWarps + warp;
        if (!goes_on(p, piece, &key, &many) || many) return;
        const int after = pieces_after(p, piece, key, lane);
        for (int col = lane * 4; col < p.features; col += 128) {
            float4 sum = part_at(p, piece, 1, col);
#pragma unroll
            for (int j = 1; j <= kJoinFew; ++j)
                if (j <= after) add4(sum, part_at(p, piece + j, 0, col));
            write_sum(p, key, col, sum);
        }
        return;
    }
    const int job = blockIdx.x - few_ctas, col = job % slabs * 128 + lane * 4;
    const int64_t base = (int64_t)(job / slabs) * kJoinGroup;
    __syncthreads();
    if (threadIdx.x < kJoinGroup && goes_on(p, base + threadIdx.x, &key, &many) && many) list[atomicAdd(&n_list, 1)] = threadIdx.x;     // (in whatever order: each is its own)
    __syncthreads();
    for (int i = 0; i < n_list; ++i) {
        const int64_t piece = base + list[i];
        const int token = p.keys[(piece + 1) * p.piece], after = pieces_after(p, piece, token, lane);
        const int each = (after + kJoinWarps - 1) / kJoinWarps, j0 = 1 + warp * each, j1 = min(j0 + each, after + 1);
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (col < p.part_ld) {
            if (warp == 0) sum = part_at(p, piece, 1, col);
#pragma unroll 16
            for (int j = j0; j < j1; ++j) add4(sum, part_at(p, piece + j, 0, col));
        }
        stretches[warp][lane] = sum;
        __syncthreads();
        if (warp == 0 && col < p.features) {
#pragma unroll
            for (int w = 1; w < kJoinWarps; ++w) add4(sum, stretches[w][lane]);
            write_sum(p, token, col, sum);
        }
        __syncthreads();
    }
}

// ---- host side ------------------------------------------------------------------------------------

template <typename F> cudaError_t by_lanes(int features, F &&f) {
    if (features <= 8) return f(std::integral_constant<int, 1>());
    if (features <= 32) return f(std::integral_constant<int, 4>());
    if (features <= 128) return f(std::integral_constant<int, 16>());
    if (features <= 256) return f(std::integral_constant<int, 32>());
    if (features <= 512) return f(std::integral_constant<int, 64>());
    return f(std::integral_constant<int, 128>());
}

template <typename T> cudaError_t forward_as(gs_ctx *ctx, const EmbeddingArgs &a, cudaStream_t st) {
    return by_lanes(a.features, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value < 32 ? decltype(lanes)::value : 32;
        const int64_t want = (a.n_tokens * L + kLookupThreads - 1) / kLookupThreads, most = (int64_t)ctx->n_sm * kLookupCtas<T>;
        LaunchTimer t(ctx, GS_K_EMBEDDING, st);
        return launch_dependent(embedding_kernel<T, L>, dim3((unsigned)(want < most ? want : most)), dim3(kLookupThreads), 0, st,
                                (const T *)a.table, a.vocabulary, a.ld_table, a.ids, a.n_tokens, a.features, a.scale, (T *)a.out, a.ld_out,
                                ctx->s.status);
    });
}

// Sorted places of a group of lanes: many enough groups for short lists, few partial sums for long ones (524,288 tokens,
// pieces of 64 / 128: 37 / 21 us to join them, 297 / 305 for the sums).  A whole gradient of 30,000 rows in a graph, pieces of
// 16 / 32 / 64 / 128: 40,000 tokens 256 wide 48 / 54 / 60 / 67 us, 1024 wide 83 / 83 / 87 / 111; 66,000 tokens 55 / 61 / 75 / 91 and
// 105 / 99 / 98 / 117; 262,144 tokens 143 / 118 / 107 / 138 and 246 / 212 / 202 / 196; 524,288 tokens 233 / 188 / 168 / 153 and
// 427 / 361 / 325 / 318.  Rows of 32 values would have shorter pieces (66,000 tokens 47 / 57 / 72 / 88, 524,288 tokens 117 / 105 /
// 109 / 137): the rule goes by the wide ones.
int piece_of(int64_t n_tokens) { return n_tokens > 262144 ? 128 : n_tokens > 65536 ? 64 : 16; }

int sort_ctas(const gs_ctx *, int64_t n) {
    const int64_t tiles = (n + kSortTile - 1) / kSortTile;
    return (int)(tiles < kMaxSortCtas ? tiles : kMaxSortCtas);
}

// Where everything is in the workspace, in bytes.
struct Layout {
    int64_t keys[2], places[2], counts, parts, end;
    int64_t n_pieces;
    int part_ld;
    Layout(const gs_ctx *ctx, int64_t n, int features) {
        const int64_t list = (n * 4 + 255) / 256 * 256;
        for (int i = 0; i < 2; ++i) { keys[i] = 2 * i * list; places[i] = keys[i] + list; }
        counts = 4 * list;
        parts = counts + (int64_t)sort_ctas(ctx, n) * kMaxBins * 4;
        n_pieces = (n + piece_of(n) - 1) / piece_of(n);
        part_ld = (features + 7) / 8 * 8;
        end = parts + n_pieces * 2 * part_ld * 4;
    }
};

template <typename T> cudaError_t sum_as(gs_ctx *ctx, const EmbeddingArgs &a, SumArgs p, cudaStream_t st) {
    return by_lanes(a.features, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const unsigned sum_ctas = (unsigned)((p.n_pieces * L + kSumThreads - 1) / kSumThreads);
        // Where a table has few rows and most of them no token, four warps share 32 of them, each with its own bisections.  In a
        // graph, one / four / sixteen: 3,191 tokens of 6,422 rows, 1455 wide, 58 / 37 / 37 us; 3,000 of 20,000, 1024 wide 48 / 39 /
        // 44, 16 wide 29 / 27 / 35; with more tokens than rows, 100,000 of 20,000, 256 wide 72 / 78 / 86, of 6,000, 16 wide 60 /
        // 58 / 67; with many rows, 3,000 of 100,000, 64 wide 31 / 39 / 54, 1024 wide 101 / 96 / 92.
        p.zero_parts = a.vocabulary < 32768 && a.n_tokens < a.vocabulary ? 4 : 1;
        const int64_t rows = ((int64_t)a.vocabulary * p.zero_parts + 127) / 128, most = (int64_t)ctx->n_sm * 8;
        p.zero_ctas = (int)(rows < most ? rows : most);
        const unsigned slabs = (unsigned)((a.features + 8 * L - 1) / (8 * L));
        LaunchTimer t(ctx, GS_K_EMBEDDING, st);
        return launch_dependent(embedding_sum_kernel<T, L>, dim3(sum_ctas + p.zero_ctas, slabs), dim3(kSumThreads), 0, st, p);
    });
}

}  // namespace

cudaError_t configure_embedding() {
    cudaError_t e = cudaFuncSetAttribute(sort_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSortSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(sort_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSortSmem);
    return e;
}

cudaError_t launch_embedding(gs_ctx *ctx, const EmbeddingArgs &a, cudaStream_t st) {
    if (a.dtype == GS_F32) return forward_as<float>(ctx, a, st);
    return a.dtype == GS_BF16 ? forward_as<__nv_bfloat16>(ctx, a, st) : forward_as<__half>(ctx, a, st);
}

int64_t embedding_workspace(const gs_ctx *ctx, int64_t n_tokens, int, int features) {
    return n_tokens == 0 ? 0 : Layout(ctx, n_tokens, features).end;
}

cudaError_t launch_embedding_backward(gs_ctx *ctx, const EmbeddingArgs &a, cudaStream_t st) {
    if (a.n_tokens == 0) return cudaMemset2DAsync(a.d_table, (size_t)a.ld_d_table * 4, 0, (size_t)a.features * 4, (size_t)a.vocabulary, st);
    const Layout at(ctx, a.n_tokens, a.features);
    char *base = (char *)a.workspace;
    SortArgs s = {};
    s.ids = a.ids;
    for (int i = 0; i < 2; ++i) { s.keys[i] = (int *)(base + at.keys[i]); s.places[i] = (int *)(base + at.places[i]); }
    s.counts = (int *)(base + at.counts);
    s.n = a.n_tokens;
    s.vocabulary = a.vocabulary;
    s.status = ctx->s.status;
    int bits = 1;                                // of the largest key, the vocabulary's size
    while (a.vocabulary >> bits) ++bits;
    s.passes = (bits + kMaxBits - 1) / kMaxBits;
    s.bits = (bits + s.passes - 1) / s.passes;
    cudaError_t e = cudaSuccess;
    if (a.n_tokens <= kOneCtaTokens) {
        LaunchTimer t(ctx, GS_K_EMBEDDING, st);
        e = launch_dependent(sort_small_kernel, dim3(1), dim3(kSortThreads), kSortSmem, st, s);
    } else {
        const int ctas = sort_ctas(ctx, a.n_tokens);
        const int64_t tiles = (a.n_tokens + kSortTile - 1) / kSortTile;
        s.per = (tiles + ctas - 1) / ctas * kSortTile;
        for (int pass = 0; pass < s.passes && e == cudaSuccess; ++pass) {
            {
                LaunchTimer t(ctx, GS_K_EMBEDDING, st);
                e = launch_dependent(sort_count_kernel, dim3(ctas), dim3(kSortThreads), 0, st, s, pass);
            }
            if (e != cudaSuccess) break;
            LaunchTimer t(ctx, GS_K_EMBEDDING, st);
            e = launch_dependent(sort_place_kernel, dim3(ctas), dim3(kSortThreads), kSortSmem, st, s, pass);
        }
    }
    if (e != cudaSuccess) return e;
    SumArgs p = {};
    p.d_out = a.d_out;
    p.ld_d_out = a.ld_d_out;
    p.keys = s.keys[(s.passes - 1) & 1];
    p.places = s.places[(s.passes - 1) & 1];
    p.n = a.n_tokens;
    p.vocabulary = a.vocabulary;
    p.features = a.features;
    p.piece = piece_of(a.n_tokens);
    p.n_pieces = at.n_pieces;
    p.scale = a.scale;
    p.d_table = a.d_table;
    p.ld_table = a.ld_d_table;
    p.parts = (float *)(base + at.parts);
    p.part_ld = at.part_ld;
    if (a.dtype == GS_F32) e = sum_as<float>(ctx, a, p, st);
    else e = a.dtype == GS_BF16 ? sum_as<__nv_bfloat16>(ctx, a, p, st) : sum_as<__half>(ctx, a, p, st);
    if (e != cudaSuccess || at.n_pieces < 2) return e;
    LaunchTimer t(ctx, GS_K_EMBEDDING, st);
    const int64_t few_ctas = (at.n_pieces + kJoinWarps - 1) / kJoinWarps, slabs = (a.features + 127) / 128;
    const int64_t many_ctas = (at.n_pieces + kJoinGroup - 1) / kJoinGroup * slabs;
    if (few_ctas + many_ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    return launch_dependent(embedding_join_kernel, dim3((unsigned)(few_ctas + many_ctas)), dim3(kJoinThreads), 0, st, p, (int)few_ctas, (int)slabs);
}

}  // namespace gs
