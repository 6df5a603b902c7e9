// Routing of requests to experts: scores, choice, weights, the order of the experts' rows, and the
// gradient of the weights.
//
//   s = softmax(x) or 1 / (1 + exp(-x));  c = s + bias;  groups of experts by the sum of their best c;
//   the top_k best c of the kept groups;  weight = scale * s / (sum of the chosen s + 1e-20)
//
// A choice is a comparison of floats, so it is made on order-preserving 32-bit keys (key 0: not to
// be chosen) with the lowest index winning among equal keys.  The order of the rows is a counting
// sort by expert in launches that share one partition of the tokens into runs, one per CTA: count (in
// the routing kernel), prefix sums (with few experts part of the next), place.  Nothing depends on the
// order of execution (the one atomic on floats adds to a place that a row names once).
//
// A row is 36 to 512 bytes of logits and hundreds of instructions, hence one thread per row with few experts and
// one warp per row with many.  One thread: 1,048,576 x 9, top 2, takes 22 us of choice (466 instructions per
// 32 rows, 61 % of the issue slots: the rest goes to the rows' scalar loads 36 bytes apart and to fixed
// latencies, with 32 warps per SM) and 17 us of placing (38 % of the slots: shared memory and barriers); its gradient
// 33 us.  One warp: 131,072 x 256 in groups takes 118 us (832 instructions a row, 80 % of the slots:
// bound by issue) and 32 us of order; its gradient 54 us (394 instructions, 86 %).  Few experts in groups
// go to a warp per row too, with most of its lanes empty: 1,048,576 x 8 in two groups takes 418 us, in one 33 us.
#include <type_traits>

#include "operators.cuh"

namespace gs {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr float kLargest = 3.402823466e38f;
constexpr float kSumFloor = 1e-20f;
constexpr int kRouteThreads = 256;

// Order-preserving key of a float that is no NaN; 0 is below all of them.
__device__ __forceinline__ unsigned key_of(float v) {
    const unsigned b = __float_as_uint(v);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

struct RouterParams {
    int n_experts, top_k, n_groups, top_groups, group_top, group_size;
    bool sigmoid, renormalise;
    float scale;
};

RouterParams params_of(const gs_expert_router &r) {
    return {r.n_experts, r.top_k, r.n_groups, r.top_groups, r.group_top, r.n_experts / r.n_groups,
            r.score == GS_SCORE_SIGMOID, r.renormalise != 0, r.scale};
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// Logits as the definition reads them: NaN takes the expert out, +infinity is the largest finite number.
__device__ __forceinline__ float clean_logit(float v, bool *nan) {
    if (v != v) { *nan = true; return -INFINITY; }
    return fminf(v, kLargest);
}

// 1 / v to one unit in the last place, v in [1, 2].
__device__ __forceinline__ float reciprocal(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// 1 / (1 + exp(-x)), by the exponential that cannot overflow: e^x / (1 + e^x) below zero.  0 at -infinity.
// (Exponentials here and below are the library's: 2 units, and what a float can hold below 2^-126 too, so
// that scores far below the best one keep their order.  2^y of the special function unit with y = x log2 e
// rounded is off by |x| 2^-24 more and ends at 2^-126; it saves 4 us of 39 at 1,048,576 x 9 and 12 us of 201
// at 131,072 x 256 with the gradient.)
__device__ __forceinline__ float sigmoid(float x) {
    const float e = expf(-fabsf(x)), r = reciprocal(1.f + e);
    return x < 0.f ? e * r : r;
}

// Its slope s (1 - s) = e^-|x| / (1 + e^-|x|)^2, without the difference, which has no digits left from x = 17 on.
__device__ __forceinline__ float sigmoid_slope(float x) {
    const float e = expf(-fabsf(x)), r = reciprocal(1.f + e);
    return e * r * r;
}

// A lane's part of a row, experts lane * V .. lane * V + V - 1, as it lies in memory: the next row's is
// asked for while this one is worked on.  `whole`: rows start so aligned, and experts divide so evenly,
// that it can be read at once.
template <typename T, int V> struct RawRow {
    alignas(16) T v[V];
    __device__ __forceinline__ void load(const T *__restrict__ row, int n_experts, int lane, bool whole) {
        const int first = lane * V;
        if (whole) {
            constexpr int kBytes = V * sizeof(T) < 16 ? V * sizeof(T) : 16;
            using Word = std::conditional_t<kBytes == 16, uint4, std::conditional_t<kBytes == 8, uint2, std::conditional_t<kBytes == 4, unsigned, unsigned short>>>;
            if (first < n_experts) {
#pragma unroll
                for (int w = 0; w < V * (int)sizeof(T) / kBytes; ++w) reinterpret_cast<Word *>(v)[w] = __ldg(reinterpret_cast<const Word *>(row + first) + w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) if (first + i < n_experts) v[i] = row[first + i];
        }
    }
    // -infinity where there is none.  True if one is infinite or not a number (or there is none): the caller then cleans them.
    __device__ __forceinline__ bool unpack(int n_experts, int lane, float (&x)[V]) const {
        float odd = 0.f;                             // 0 * x is not a number for either
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = lane * V + i < n_experts ? to_float(v[i]) : -INFINITY;
            odd = fmaf(x[i], 0.f, odd);
        }
        return odd != odd;
    }
};

template <int V> __device__ __forceinline__ void clean_row(float (&x)[V], bool *nan) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = clean_logit(x[i], nan);
}

template <typename T, int V> bool whole_rows(int64_t ld, int n_experts) {
    const int bytes = V * (int)sizeof(T) < 16 ? V * (int)sizeof(T) : 16;
    return n_experts % V == 0 && ld * (int64_t)sizeof(T) % bytes == 0;
}

// Scores in place of logits; 0 for what cannot be chosen.
template <int V>
__device__ __forceinline__ void scores_of(float (&x)[V], bool sigmoid_score) {
    if (sigmoid_score) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = sigmoid(x[i]);
        return;
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
    top = fmaxf(warp_max(top), -kLargest);           // (nothing left: every exponential is 0)
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) { x[i] = expf(x[i] - top); sum += x[i]; }
    sum = warp_sum(sum);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= inv;
}

__device__ __forceinline__ float value_of(unsigned key) {
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

// A lane's keys in descending order, equal ones by index: an odd-even merge sort, its network laid
// out at compile time (stages P = 1, 2, 4, ...; distances K = P, P / 2, ..., 1).
template <int V, int P, int K>
__device__ __forceinline__ void sort_step(unsigned (&key)[V], int (&at)[V]) {
    if constexpr (P < V) {
#pragma unroll
        for (int lo = 0; lo < V - K; ++lo) {
            const int hi = lo + K, j = K % P;
            if (lo >= j && (lo - j) % (2 * K) < K && lo / (2 * P) == hi / (2 * P)) {
                const bool swap = key[hi] > key[lo] || (key[hi] == key[lo] && at[hi] < at[lo]);
                const unsigned k0 = key[lo], k1 = key[hi];
                const int a0 = at[lo], a1 = at[hi];
                key[lo] = swap ? k1 : k0;
                key[hi] = swap ? k0 : k1;
                at[lo] = swap ? a1 : a0;
                at[hi] = swap ? a0 : a1;
            }
        }
        if constexpr (K > 1) sort_step<V, P, K / 2>(key, at);
        else sort_step<V, 2 * P, 2 * P>(key, at);
    }
}
template <int V>
__device__ __forceinline__ void sort_lane(unsigned (&key)[V], int (&at)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) at[i] = i;
    sort_step<V, 1, 1>(key, at);
}

// Key of the group's score that a lane's experts belong to, where every group is a power of two of
// whole lanes: the two best of every lane, merged between its lanes.
template <int V>
__device__ __forceinline__ unsigned group_key(const unsigned (&key)[V], int lanes, int group_top) {
    unsigned k1 = 0, k2 = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) { k2 = max(k2, min(k1, key[i])); k1 = max(k1, key[i]); }
    for (int o = 1; o < lanes; o <<= 1) {
        const unsigned o1 = __shfl_xor_sync(kFull, k1, o), o2 = __shfl_xor_sync(kFull, k2, o);
        k2 = max(max(k2, o2), min(k1, o1));
        k1 = max(k1, o1);
    }
    return group_top == 2 && k2 ? key_of(value_of(k1) + value_of(k2)) : k1;
}

// ... of group g for any other size; every lane gets it.
template <int V>
__device__ __forceinline__ unsigned group_key_any(const unsigned (&key)[V], int lane, int lo, int hi, int group_top) {
    unsigned k1 = 0, k2 = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        const unsigned k = e >= lo && e < hi ? key[i] : 0u;
        k2 = max(k2, min(k1, k));
        k1 = max(k1, k);
    }
    const unsigned top = __reduce_max_sync(kFull, k1);
    if (group_top < 2) return top;
    const int owner = __ffs(__ballot_sync(kFull, k1 == top)) - 1;
    const unsigned second = __reduce_max_sync(kFull, lane == owner ? k2 : k1);
    return second ? key_of(value_of(top) + value_of(second)) : top;
}

// The groups that are kept, as a mask.  `lanes`: lanes of a group if all groups are the same power of
// two of whole lanes, else 0.
template <int V>
__device__ __forceinline__ unsigned kept_groups(const unsigned (&key)[V], const RouterParams &p, int lanes, int lane) {
    unsigned mine = 0;                               // lane g: key of group g's score
    if (lanes) {
        const unsigned own = group_key<V>(key, lanes, p.group_top);
        mine = __shfl_sync(kFull, own, lane * lanes & 31);
        if (lane >= p.n_groups) mine = 0;
    } else {
        for (int g = 0; g < p.n_groups; ++g) {
            const unsigned k = group_key_any<V>(key, lane, g * p.group_size, (g + 1) * p.group_size, p.group_top);
            if (lane == g) mine = k;
        }
    }
    int before = 0;                                  // groups that rank before this lane's
    for (int g = 0; g < p.n_groups; ++g) {
        const unsigned other = __shfl_sync(kFull, mine, g);
        before += other > mine || (other == mine && g < lane);
    }
    return __ballot_sync(kFull, lane < p.n_groups && before < p.top_groups);
}

// The top_k best keys of the warp, slot j's expert in lane j (-1: none left).  first: the expert of a
// lane's key 0; experts ascend with lanes.  Every round takes the best head of the lanes' sorted lists.
template <int V>
__device__ __forceinline__ int best_experts(unsigned (&key)[V], int first, int top_k, int lane) {
    int mine = -1, at[V];
    sort_lane<V>(key, at);
#pragma unroll
    for (int i = 0; i < V; ++i) at[i] += first;
    for (int j = 0; j < top_k; ++j) {
        const unsigned top = __reduce_max_sync(kFull, key[0]);
        if (top == 0) break;
        const int owner = __ffs(__ballot_sync(kFull, key[0] == top)) - 1;
        const int e = __shfl_sync(kFull, at[0], owner);
        if (lane == j) mine = e;
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i + 1 < V; ++i) { key[i] = key[i + 1]; at[i] = at[i + 1]; }
            key[V - 1] = 0u;
        }
    }
    __syncwarp();
    return mine;
}

// One warp per row, V * 32 experts at most.
template <typename T, int V, int kRouteWarps>
__device__ __forceinline__ void route_rows(const T *__restrict__ logits, int64_t first, int64_t last, int64_t ld, bool whole,
                                           const float *__restrict__ bias, const RouterParams &p,
                                           int32_t *__restrict__ out_expert, float *__restrict__ out_weight,
                                           int *cta_count, float (*scores)[V * 32], unsigned *__restrict__ status)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ unsigned packed[kRouteWarps][V * 16];
    __shared__ unsigned char packed_lane[kRouteWarps][32];
    float b[V];
    unsigned b_off = 0;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        b[i] = bias && e < p.n_experts ? clean_logit(bias[e], &nan) : 0.f;
        if (b[i] == -INFINITY || e >= p.n_experts) { b_off |= 1u << i; b[i] = 0.f; }
    }
    // groups of whole lanes; few enough kept that their experts fit half as many places
    int lanes = 0;
    if (p.n_groups > 1 && p.group_size % V == 0 && (p.group_size / V & (p.group_size / V - 1)) == 0) lanes = p.group_size / V;
    const bool halved = V > 1 && lanes && p.top_groups * p.group_size <= 16 * V;
    const int step = blockDim.x >> 5;
    RawRow<T, V> raw;
    if (first + warp < last) raw.load(logits + (first + warp) * ld, p.n_experts, lane, whole);
    for (int64_t n = first + warp; n < last; n += step) {
        float s[V];
        unsigned key[V], off = 0;
        const bool odd = raw.unpack(p.n_experts, lane, s);
        if (n + step < last) raw.load(logits + (n + step) * ld, p.n_experts, lane, whole);
        if (odd) {
            clean_row<V>(s, &nan);
#pragma unroll
            for (int i = 0; i < V; ++i) off |= (s[i] == -INFINITY ? 1u : 0u) << i;
        }
        scores_of<V>(s, p.sigmoid);
        float *row = scores[warp];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            key[i] = key_of(s[i] + b[i]);
            row[lane * V + i] = s[i];
        }
        if (off | b_off) {
#pragma unroll
            for (int i = 0; i < V; ++i) if (((off | b_off) >> i) & 1) key[i] = 0u;
        }
        int my_expert;                               // lane j: slot j
        if (p.n_groups == 1) {
            my_expert = best_experts<V>(key, lane * V, p.top_k, lane);
        } else {
            const unsigned kept = kept_groups<V>(key, p, lanes, lane);
            if (halved) {
                // the kept groups' keys move together, V / 2 to a lane
                constexpr int H = V > 1 ? V / 2 : 1;
                const int group = lane / lanes, chunk = __popc(kept & ((1u << group) - 1)) * lanes + lane % lanes;
                if (lane < p.n_groups * lanes && ((kept >> group) & 1)) {
#pragma unroll
                    for (int i = 0; i < V; ++i) packed[warp][chunk * V + i] = key[i];
                    packed_lane[warp][chunk] = (unsigned char)lane;
                }
                __syncwarp();
                const bool used = lane / 2 < p.top_groups * lanes;
                unsigned half[H];
#pragma unroll
                for (int i = 0; i < H; ++i) half[i] = used ? packed[warp][lane * H + i] : 0u;
                const int from = used ? packed_lane[warp][lane / 2] : 0;
                my_expert = best_experts<H>(half, from * V + lane % 2 * H, p.top_k, lane);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int e = lane * V + i;
                    if (e < p.n_experts && !((kept >> (e / p.group_size)) & 1)) key[i] = 0u;
                }
                my_expert = best_experts<V>(key, lane * V, p.top_k, lane);
            }
        }
        const float my_score = my_expert >= 0 ? scores[warp][my_expert] : 0.f;
        const float total = warp_sum(my_score) + kSumFloor;
        if (lane < p.top_k) {
            out_expert[n * p.top_k + lane] = my_expert;
            out_weight[n * p.top_k + lane] = p.scale * (p.renormalise ? my_score / total : my_score);
            if (cta_count && my_expert >= 0) atomicAdd(&cta_count[my_expert], 1);
        }
        __syncwarp();
    }
    if (nan) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads)
route_rows_kernel(const T *__restrict__ logits, int64_t n_tokens, int64_t ld, bool whole, const float *__restrict__ bias,
                  RouterParams p, int rows_per_cta, int32_t *__restrict__ out_expert, float *__restrict__ out_weight,
                  int *__restrict__ counts, unsigned *__restrict__ status)
{
    __shared__ int cta_count[V * 32];
    __shared__ float scores[kRouteThreads / 32][V * 32];
    dependent_wait();
    for (int e = threadIdx.x; e < p.n_experts; e += kRouteThreads) cta_count[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * rows_per_cta;
    route_rows<T, V, kRouteThreads / 32>(logits, first, min(first + rows_per_cta, n_tokens), ld, whole, bias, p, out_expert, out_weight,
                     counts ? cta_count : nullptr, scores, status);
    if (!counts) return;
    __syncthreads();
    for (int e = threadIdx.x; e < p.n_experts; e += kRouteThreads)
        counts[e * kMaxRouteCtas + blockIdx.x] = cta_count[e];
    dependent_end();
}

// Few experts without groups: one thread per row, all of its scores in registers (E of them, the
// experts or a few more; those past the last are taken out of the choice).
__host__ __device__ constexpr int fewest_of(int width) { return width <= 4 ? 1 : width <= 12 ? width - 1 : width == 16 ? 13 : width == 24 ? 17 : 25; }

template <typename T, int E>
__device__ __forceinline__ void load_token(const T *__restrict__ row, int n_experts, float (&x)[E]) {
    constexpr int kAlways = fewest_of(E);            // (a width serves no fewer experts than these)
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = e < kAlways || e < n_experts ? to_float(row[e]) : -INFINITY;
}

// Scores up to the factor *inv (softmax: exponentials and one over their sum; sigmoid: 1).
template <int E>
__device__ __forceinline__ float token_scores_once(const float (&x)[E], float (&s)[E], bool sigmoid_score) {
    float sum = 0.f;
    if (sigmoid_score) {
#pragma unroll
        for (int e = 0; e < E; ++e) { s[e] = sigmoid(x[e]); sum += s[e]; }
        return sum;
    }
    float top = -kLargest;                           // (a row with nothing left: every exponential is 0)
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, x[e]);
#pragma unroll
    for (int e = 0; e < E; ++e) { s[e] = expf(x[e] - top); sum += s[e]; }
    return sum;
}
// NaNs and +infinity make the sum a NaN; only then the logits are looked at one by one.
template <int E>
__device__ __forceinline__ void token_scores(float (&x)[E], float (&s)[E], bool sigmoid_score, float *inv, bool *nan) {
    float sum = token_scores_once<E>(x, s, sigmoid_score);
    if (sum != sum) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = clean_logit(x[e], nan);
        sum = token_scores_once<E>(x, s, sigmoid_score);
    }
    *inv = sigmoid_score ? 1.f : sum > 0.f ? 1.f / sum : 0.f;
}

// count: this thread's column of [experts][threads] counters in shared memory, or null
template <typename T, int E, bool kBias>
__device__ __forceinline__ void route_token(const T *__restrict__ row, int64_t n, const float *__restrict__ bias, const RouterParams &p,
                                            int32_t *__restrict__ out_expert, float *__restrict__ out_weight,
                                            int *count, int stride, bool *nan)
{
    // scores up to the factor inv; choice scores, -infinity where an expert cannot be chosen (without a
    // bias the factor, the same for the whole row, does not change their order)
    float x[E], s[E], c[E], inv;
    load_token<T, E>(row, p.n_experts, x);
    token_scores<E>(x, s, p.sigmoid, &inv, nan);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        c[e] = s[e];
        if (kBias && e < p.n_experts) c[e] = fmaf(s[e], inv, clean_logit(__ldg(bias + e), nan));
        if (x[e] == -INFINITY) c[e] = -INFINITY;
    }
    int32_t *experts = out_expert + n * p.top_k;
    float *weights = out_weight + n * p.top_k;
    float total = kSumFloor, q0 = 0.f, q1 = 0.f;     // (two slots' scores stay in registers, more are read back)
    for (int j = 0; j < p.top_k; ++j) {
        float best = -INFINITY, score = 0.f;
        int at = -1;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c[e] > best) { best = c[e]; at = e; if (kBias) score = s[e]; }
        if (at >= 0) {
            score = (kBias ? score : best) * inv;
            if (count) count[at * stride] += 1;
#pragma unroll
            for (int e = 0; e < E; ++e) if (e == at) c[e] = -INFINITY;
        }
        experts[j] = at;
        total += score;
        if (j == 0) q0 = score; else if (j == 1) q1 = score; else weights[j] = score;
    }
    // (the scale comes last: scale / total alone can leave the range of a float)
    const float share = p.renormalise ? 1.f / total : 1.f;
    const auto weigh = [&](float q) { return p.scale * (q * share); };
    weights[0] = weigh(q0);
    if (p.top_k > 1) weights[1] = weigh(q1);
    for (int j = 2; j < p.top_k; ++j) weights[j] = weigh(weights[j]);
}

template <typename T, int E, bool kBias>
__global__ void __launch_bounds__(kRouteThreads)
route_tokens_kernel(const T *__restrict__ logits, int64_t n_tokens, int64_t ld, const float *__restrict__ bias,
                    RouterParams p, int rows_per_cta, int32_t *__restrict__ out_expert, float *__restrict__ out_weight,
                    int *__restrict__ counts, unsigned *__restrict__ status)
{
    __shared__ int count[E * kRouteThreads];
    dependent_wait();
    int *mine = nullptr;
    if (counts) {
        mine = count + threadIdx.x;
#pragma unroll
        for (int e = 0; e < E; ++e) mine[e * kRouteThreads] = 0;
    }
    const int64_t first = (int64_t)blockIdx.x * rows_per_cta, last = min(first + rows_per_cta, n_tokens);
    bool nan = false;
    for (int64_t n = first + threadIdx.x; n < last; n += kRouteThreads)
        route_token<T, E, kBias>(logits + n * ld, n, bias, p, out_expert, out_weight, mine, kRouteThreads, &nan);
    if (nan) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
    if (!counts) return;
    __syncthreads();
    for (int e = threadIdx.x >> 5; e < p.n_experts; e += kRouteThreads / 32) {
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kRouteThreads / 32; ++i) sum += count[e * kRouteThreads + i * 32 + (threadIdx.x & 31)];
        sum = __reduce_add_sync(kFull, sum);
        if ((threadIdx.x & 31) == 0) counts[e * kMaxRouteCtas + blockIdx.x] = sum;
    }
    dependent_end();
}

// Per expert (one warp each): counts per CTA become the rows before that CTA's, and their total.
__global__ void __launch_bounds__(kRouteThreads)
route_prefix_kernel(int *__restrict__ counts, int n_experts, int n_ctas)
{
    dependent_wait();
    const int e = blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (e >= n_experts) return;
    int *c = counts + e * kMaxRouteCtas, before = 0;
    for (int base = 0; base < n_ctas; base += 32) {
        const int i = base + lane;
        const int own = i < n_ctas ? c[i] : 0;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFull, sum, o);
            if (lane >= o) sum += up;
        }
        if (i < n_ctas) c[i] = before + sum - own;
        before += __shfl_sync(kFull, sum, 31);
    }
    if (lane == 0) counts[GS_MAX_EXPERTS * kMaxRouteCtas + e] = before;
    dependent_end();
}

// Places the slots [cta_first, cta_last): each warp takes a stretch of them, first counts its
// experts, then (knowing what the warps before it hold) hands out rows in order.  cnt: [warps]
// [n_experts] counters in shared memory; base(e): first row of expert e for this CTA, called once
// every warp has counted.
template <typename Base>
__device__ __forceinline__ void place_slots(const int32_t *expert, int64_t cta_first, int64_t cta_last, int top_k, int n_experts,
                                            int *cnt, Base &&base, int32_t *__restrict__ row_token, int32_t *__restrict__ token_row)
{
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < warps * n_experts; i += blockDim.x) cnt[i] = 0;
    __syncthreads();
    const int64_t per_warp = ((cta_last - cta_first + warps - 1) / warps + 31) / 32 * 32;
    const int64_t first = min(cta_first + warp * per_warp, cta_last), last = min(first + per_warp, cta_last);
    int *mine = cnt + warp * n_experts;
    constexpr int kAhead = 4;                        // slots of a lane asked for at once
    for (int64_t i0 = first; i0 < last; i0 += 32 * kAhead) {
        int e[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) e[k] = i0 + k * 32 + lane < last ? expert[i0 + k * 32 + lane] : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const unsigned same = __match_any_sync(kFull, e[k]);
            if (e[k] >= 0 && __ffs(same) - 1 == lane) mine[e[k]] += __popc(same);
            __syncwarp();
        }
    }
    __syncthreads();
    base(cnt, warps);
    __syncthreads();
    for (int64_t i0 = first; i0 < last; i0 += 32 * kAhead) {
        int e[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) e[k] = i0 + k * 32 + lane < last ? expert[i0 + k * 32 + lane] : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t i = i0 + k * 32 + lane;
            const unsigned same = __match_any_sync(kFull, e[k]);
            int row = -1;
            if (e[k] >= 0) row = mine[e[k]] + __popc(same & ((1u << lane) - 1));
            __syncwarp();
            if (e[k] >= 0 && __ffs(same) - 1 == lane) mine[e[k]] += __popc(same);
            __syncwarp();
            if (i < last) {
                token_row[i] = row;
                if (row >= 0) row_token[row] = (int)((unsigned)i / (unsigned)top_k);
            }
        }
    }
}

// start[e] = sum of total(e') over e' < e, by one warp; start[n_experts] = all.
template <typename Total>
__device__ __forceinline__ void prefix_experts(int n_experts, int lane, int *start, Total &&total) {
    int before = 0;
    for (int base = 0; base < n_experts; base += 32) {
        const int e = base + lane, own = e < n_experts ? total(e) : 0;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFull, sum, o);
            if (lane >= o) sum += up;
        }
        if (e < n_experts) start[e] = before + sum - own;
        before += __shfl_sync(kFull, sum, 31);
    }
    if (lane == 0) start[n_experts] = before;
}

__global__ void __launch_bounds__(kRouteThreads)
route_place_kernel(const int32_t *__restrict__ expert, int64_t n_slots, int top_k, int slots_per_cta, int n_experts,
                   const int *__restrict__ counts, int32_t *__restrict__ offsets, int32_t *__restrict__ row_token,
                   int32_t *__restrict__ token_row)
{
    extern __shared__ int place_smem[];
    int *start = place_smem, *cnt = start + n_experts + 1;     // [n_experts + 1], [warps][n_experts]
    dependent_wait();
    const int *total = counts + GS_MAX_EXPERTS * kMaxRouteCtas;
    if (threadIdx.x < 32) prefix_experts(n_experts, threadIdx.x, start, [&](int e) { return total[e]; });
    const int64_t first = min((int64_t)blockIdx.x * slots_per_cta, n_slots), last = min(first + slots_per_cta, n_slots);
    place_slots(expert, first, last, top_k, n_experts, cnt, [&](int *c, int warps) {
        for (int e = threadIdx.x; e < n_experts; e += kRouteThreads) {
            int row = start[e] + counts[e * kMaxRouteCtas + blockIdx.x];
            for (int w = 0; w < warps; ++w) { const int own = c[w * n_experts + e]; c[w * n_experts + e] = row; row += own; }
        }
    }, row_token, token_row);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= n_experts; e += kRouteThreads) offsets[e] = start[e];
    // rows that no slot took
    const int64_t step = (int64_t)gridDim.x * kRouteThreads;
    for (int64_t i = start[n_experts] + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; i < n_slots; i += step)
        row_token[i] = -1;
}

// The same for few experts, without any exchange between lanes: every thread takes a run of
// consecutive slots of a block in shared memory (an odd number: no bank conflicts), counts them in a column of its own; the columns' prefix sums per expert are the threads' first rows.  The rows of the CTAs
// before this one are added up here as well (n_experts * gridDim.x numbers), which saves a launch.
constexpr int kRun = 7, kRunSlots = kRun * kRouteThreads;
__global__ void __launch_bounds__(kRouteThreads)
route_place_runs_kernel(const int32_t *__restrict__ expert, int64_t n_slots, int top_k, int slots_per_cta, int n_experts,
                        const int *__restrict__ counts, int32_t *__restrict__ offsets, int32_t *__restrict__ row_token,
                        int32_t *__restrict__ token_row)
{
    __shared__ int slot_row[kRunSlots];              // a block of slots: their experts, then their rows
    extern __shared__ int place_smem[];
    int *total = place_smem, *next = total + n_experts, *start = next + n_experts, *cnt = start + n_experts + 1;
    dependent_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t cta_first = min((int64_t)blockIdx.x * slots_per_cta, n_slots), cta_last = min(cta_first + slots_per_cta, n_slots);
    for (int e = warp; e < n_experts; e += kRouteThreads / 32) {
        int all = 0, early = 0;
        for (int c = lane; c < (int)gridDim.x; c += 32) {
            const int v = counts[e * kMaxRouteCtas + c];
            all += v;
            early += c < (int)blockIdx.x ? v : 0;
        }
        all = __reduce_add_sync(kFull, all);
        early = __reduce_add_sync(kFull, early);
        if (lane == 0) { total[e] = all; next[e] = early; }
    }
    __syncthreads();
    if (warp == 0) prefix_experts(n_experts, lane, start, [&](int e) { return total[e]; });
    __syncthreads();
    for (int e = threadIdx.x; e < n_experts; e += kRouteThreads) next[e] += start[e];
    int *mine = cnt + threadIdx.x;                   // [n_experts][kRouteThreads]
    for (int64_t block = cta_first; block < cta_last; block += kRunSlots) {
        const int n = (int)min((int64_t)kRunSlots, cta_last - block);
        for (int i = threadIdx.x; i < kRunSlots; i += kRouteThreads) slot_row[i] = i < n ? expert[block + i] : -1;
        for (int e = 0; e < n_experts; ++e) mine[e * kRouteThreads] = 0;
        __syncthreads();
        int *run = slot_row + threadIdx.x * kRun;
#pragma unroll
        for (int i = 0; i < kRun; ++i) if (run[i] >= 0) mine[run[i] * kRouteThreads] += 1;
        __syncthreads();
        for (int e = warp; e < n_experts; e += kRouteThreads / 32) {
            int row = next[e];
            for (int base = 0; base < kRouteThreads; base += 32) {
                const int own = cnt[e * kRouteThreads + base + lane];
                int sum = own;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(kFull, sum, o);
                    if (lane >= o) sum += up;
                }
                cnt[e * kRouteThreads + base + lane] = row + sum - own;
                row += __shfl_sync(kFull, sum, 31);
            }
            if (lane == 0) next[e] = row;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const int e = run[i];
            if (e < 0) continue;
            const int row = mine[e * kRouteThreads];
            mine[e * kRouteThreads] = row + 1;
            run[i] = row;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kRouteThreads) {
            const int row = slot_row[i];
            token_row[block + i] = row;
            if (row >= 0) row_token[row] = (int)((unsigned)(block + i) / (unsigned)top_k);
        }
        __syncthreads();
    }
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= n_experts; e += kRouteThreads) offsets[e] = start[e];
    const int64_t step = (int64_t)gridDim.x * kRouteThreads;
    for (int64_t i = start[n_experts] + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; i < n_slots; i += step)
        row_token[i] = -1;
}

// Few tokens: choice and order in one launch of one CTA.
constexpr int kSmallThreads = 512;
template <typename T, int V, bool kTokens>
__global__ void __launch_bounds__(kSmallThreads)
route_small_kernel(const T *__restrict__ logits, int n_tokens, int64_t ld, bool whole, const float *__restrict__ bias,
                   RouterParams p, int32_t *out_expert, float *__restrict__ out_weight, int32_t *__restrict__ offsets,
                   int32_t *__restrict__ row_token, int32_t *__restrict__ token_row, unsigned *__restrict__ status)
{
    extern __shared__ int place_smem[];
    int *start = place_smem, *cnt = start + p.n_experts + 1;   // scores of the rows before cnt is in use
    dependent_wait();
    if constexpr (kTokens) {
        bool nan = false;
        for (int n = threadIdx.x; n < n_tokens; n += kSmallThreads)
            if (bias) route_token<T, V, true>(logits + n * ld, n, bias, p, out_expert, out_weight, nullptr, 0, &nan);
            else route_token<T, V, false>(logits + n * ld, n, bias, p, out_expert, out_weight, nullptr, 0, &nan);
        if (nan) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
    } else {
        route_rows<T, V, kSmallThreads / 32>(logits, 0, n_tokens, ld, whole, bias, p, out_expert, out_weight, nullptr,
                         reinterpret_cast<float (*)[V * 32]>(cnt), status);
    }
    __syncthreads();
    const int n_slots = n_tokens * p.top_k;
    place_slots(out_expert, 0, n_slots, p.top_k, p.n_experts, cnt, [&](int *c, int warps) {
        // rows of every expert: a warp's count becomes the rows of the warps before it, then the experts before it are added
        for (int e = threadIdx.x; e < p.n_experts; e += kSmallThreads) {
            int row = 0;
            for (int w = 0; w < warps; ++w) { const int own = c[w * p.n_experts + e]; c[w * p.n_experts + e] = row; row += own; }
            start[e] = row;
        }
        __syncthreads();
        if (threadIdx.x < 32) {
            // (each lane reads its own totals before any of the batch is overwritten)
            prefix_experts(p.n_experts, threadIdx.x, start, [&](int e) { return start[e]; });
        }
        __syncthreads();
        for (int i = threadIdx.x; i < warps * p.n_experts; i += kSmallThreads) c[i] += start[i % p.n_experts];
    }, row_token, token_row);
    for (int e = threadIdx.x; e <= p.n_experts; e += kSmallThreads) offsets[e] = start[e];
    for (int i = start[p.n_experts] + threadIdx.x; i < n_slots; i += kSmallThreads) row_token[i] = -1;
}

// Gradient of the weights, one warp per row.  With q the chosen scores, t = sum q + 1e-20:
//   renormalised: dq_j = scale * (dw_j - sum_i dw_i q_i / t) / t;   else dq_j = scale * dw_j
//   sigmoid: dx = dq * s (1 - s), by the logit;   softmax: dx = s * (dq - sum_j dq_j s_j)
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads)
route_rows_backward_kernel(const T *__restrict__ logits, int64_t n_tokens, int64_t ld, bool whole, RouterParams p,
                           const int32_t *__restrict__ expert, const float *__restrict__ d_weight,
                           T *__restrict__ d_logits, int64_t ld_d, bool whole_d, unsigned *__restrict__ status)
{
    constexpr int kWarps = kRouteThreads / 32;
    __shared__ __align__(16) float row_smem[kWarps][V * 32];   // a row's scores, then the gradients of those that were chosen
    dependent_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float *mine = row_smem[warp];
    bool bad = false;
    const int64_t step = (int64_t)gridDim.x * kWarps;
    RawRow<T, V> raw;
    int next_expert = -1;
    float next_dw = 0.f;
    const auto ask = [&](int64_t n) {
        if (n >= n_tokens) return;
        raw.load(logits + n * ld, p.n_experts, lane, whole);
        if (lane < p.top_k) { next_expert = expert[n * p.top_k + lane]; next_dw = d_weight[n * p.top_k + lane]; }
    };
    ask((int64_t)blockIdx.x * kWarps + warp);
    for (int64_t n = (int64_t)blockIdx.x * kWarps + warp; n < n_tokens; n += step) {
        float s[V];
        if (raw.unpack(p.n_experts, lane, s)) clean_row<V>(s, &bad);
        int e = next_expert;
        if (e < -1 || e >= p.n_experts) { bad = true; e = -1; }
        const float dw = e >= 0 ? next_dw : 0.f;
        ask(n + step);
        if (p.sigmoid) {                             // the scores to shared memory, their slopes in s
#pragma unroll
            for (int i = 0; i < V; ++i) { mine[lane * V + i] = sigmoid(s[i]); s[i] = sigmoid_slope(s[i]); }
        } else {
            scores_of<V>(s, false);
#pragma unroll
            for (int i = 0; i < V; ++i) mine[lane * V + i] = s[i];
        }
        __syncwarp();
        const float q = e >= 0 ? mine[e] : 0.f;      // lane j: the score of slot j
        __syncwarp();
        float dq = p.scale * dw;
        if (p.renormalise) {
            const float t = warp_sum(q) + kSumFloor, mean = warp_sum(dw * (q / t));
            dq = e >= 0 ? p.scale * ((dw - mean) / t) : 0.f;
        }
        const float mean = p.sigmoid ? 0.f : warp_sum(dq * q);
#pragma unroll
        for (int i = 0; i < V; ++i) mine[lane * V + i] = 0.f;
        __syncwarp();
        if (e >= 0) atomicAdd(&mine[e], dq);         // (a row names an expert once at most)
        __syncwarp();
        float dx[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float ds = mine[lane * V + i];
            dx[i] = p.sigmoid ? ds * s[i] : s[i] * (ds - mean);
        }
        __syncwarp();
        T *out = d_logits + n * ld_d + lane * V;
        if (whole_d) {
            constexpr int kBytes = V * sizeof(T) < 16 ? V * sizeof(T) : 16, kEach = kBytes / sizeof(T);
            using Word = std::conditional_t<kBytes == 16, uint4, std::conditional_t<kBytes == 8, uint2, std::conditional_t<kBytes == 4, unsigned, unsigned short>>>;
            if (lane * V < p.n_experts) {
#pragma unroll
                for (int w = 0; w < V / kEach; ++w) {
                    Word word;
#pragma unroll
                    for (int i = 0; i < kEach; ++i) reinterpret_cast<T *>(&word)[i] = from_float<T>(dx[w * kEach + i]);
                    reinterpret_cast<Word *>(out)[w] = word;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) if (lane * V + i < p.n_experts) out[i] = from_float<T>(dx[i]);
        }
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

template <typename T, int E>
__global__ void __launch_bounds__(kRouteThreads)
route_tokens_backward_kernel(const T *__restrict__ logits, int64_t n_tokens, int64_t ld, RouterParams p,
                             const int32_t *__restrict__ expert, const float *__restrict__ d_weight,
                             T *__restrict__ d_logits, int64_t ld_d, unsigned *__restrict__ status)
{
    dependent_wait();
    bool bad = false;
    for (int64_t n = (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; n < n_tokens; n += (int64_t)gridDim.x * kRouteThreads) {
        float x[E], s[E], ds[E], inv;
        load_token<T, E>(logits + n * ld, p.n_experts, x);
        token_scores<E>(x, s, p.sigmoid, &inv, &bad);
        unsigned chosen = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] *= inv;
        float sum = kSumFloor, mean = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ds[e] = 0.f;
        for (int j = 0; j < p.top_k; ++j) {
            const int at = expert[n * p.top_k + j];
            if (at < -1 || at >= p.n_experts) { bad = true; continue; }
            if (at < 0) continue;
            const float dw = d_weight[n * p.top_k + j];
#pragma unroll
            for (int e = 0; e < E; ++e) if (e == at) { ds[e] += dw; sum += s[e]; }
            chosen |= 1u << at;
        }
        if (p.renormalise) {
#pragma unroll
            for (int e = 0; e < E; ++e) mean += ds[e] * (s[e] / sum);
#pragma unroll
            for (int e = 0; e < E; ++e) ds[e] = (chosen >> e) & 1 ? (ds[e] - mean) / sum : 0.f;
        }
        float across = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) { ds[e] *= p.scale; across += ds[e] * s[e]; }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float dx = p.sigmoid ? ds[e] * sigmoid_slope(x[e]) : s[e] * (ds[e] - across);
            if (e < p.n_experts) d_logits[n * ld_d + e] = from_float<T>(dx);
        }
    }
    if (bad) atomicOr(status, (unsigned)GS_DEV_BAD_VALUE);
}

// One thread per row up to this many experts (without groups), one warp per row above and with groups.
constexpr int kTokenExperts = 32;

template <typename F> cudaError_t by_token_width(int n_experts, F &&f) {
    switch (n_experts) {
        case 1: case 2: case 3: case 4: return f(std::integral_constant<int, 4>());
        case 5: case 6: return f(std::integral_constant<int, 6>());
        case 7: case 8: return f(std::integral_constant<int, 8>());
        case 9: case 10: return f(std::integral_constant<int, 10>());
        case 11: case 12: return f(std::integral_constant<int, 12>());
        case 13: case 14: case 15: case 16: return f(std::integral_constant<int, 16>());
        case 17: case 18: case 19: case 20: case 21: case 22: case 23: case 24: return f(std::integral_constant<int, 24>());
        default: return f(std::integral_constant<int, 32>());
    }
}

template <typename F> cudaError_t by_row_width(int n_experts, F &&f) {
    if (n_experts <= 32) return f(std::integral_constant<int, 1>());
    if (n_experts <= 64) return f(std::integral_constant<int, 2>());
    if (n_experts <= 128) return f(std::integral_constant<int, 4>());
    if (n_experts <= 256) return f(std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 16>());
}

int route_ctas(const gs_ctx *ctx) {
    const int most = ctx->n_sm * 4;
    return most < kMaxRouteCtas ? most : kMaxRouteCtas;
}

template <typename T> cudaError_t route_as(gs_ctx *ctx, const ExpertRouteArgs &a, cudaStream_t st) {
    const RouterParams p = params_of(a.r);
    const bool tokens = p.n_experts <= kTokenExperts && p.n_groups == 1;
    const T *logits = (const T *)a.logits;
    // one CTA: two tokens a thread, or eight rows a warp (its tables fit 48 KB up to 256 experts)
    if (a.offsets && a.n_tokens <= (tokens ? 2 * kSmallThreads : p.n_experts <= 256 ? kSmallThreads / 32 * 8 : -1)) {
        const size_t counters = sizeof(int) * (kSmallThreads / 32) * (size_t)p.n_experts, lead = sizeof(int) * (p.n_experts + 1);
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        if (tokens)
            return by_token_width(p.n_experts, [&](auto v) {
                return launch_dependent(route_small_kernel<T, decltype(v)::value, true>, dim3(1), dim3(kSmallThreads), lead + counters, st,
                                        logits, (int)a.n_tokens, a.ld, false, a.bias, p, a.expert, a.weight, a.offsets, a.row_token,
                                        a.token_row, ctx->s.status);
            });
        return by_row_width(p.n_experts, [&](auto v) {
            constexpr int V = decltype(v)::value < 16 ? decltype(v)::value : 8;
            const size_t scores = sizeof(float) * (kSmallThreads / 32) * V * 32;
            return launch_dependent(route_small_kernel<T, V, false>, dim3(1), dim3(kSmallThreads), lead + (counters > scores ? counters : scores), st,
                                    logits, (int)a.n_tokens, a.ld, whole_rows<T, V>(a.ld, p.n_experts), a.bias, p, a.expert, a.weight,
                                    a.offsets, a.row_token, a.token_row, ctx->s.status);
        });
    }
    const int at_once = tokens ? kRouteThreads : kRouteThreads / 32;         // rows of a CTA
    const int64_t want = a.n_tokens < 1 ? 1 : (a.n_tokens + at_once - 1) / at_once;
    const int n_ctas = want < route_ctas(ctx) ? (int)want : route_ctas(ctx);
    const int rows_per_cta = (int)(((a.n_tokens + n_ctas - 1) / n_ctas + at_once - 1) / at_once * at_once);
    int *counts = a.offsets ? operator_scratch(ctx).expert_counts : nullptr;
    cudaError_t e;
    {
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        if (tokens)
            e = by_token_width(p.n_experts, [&](auto v) {
                constexpr int E = decltype(v)::value;
                return launch_dependent(a.bias ? route_tokens_kernel<T, E, true> : route_tokens_kernel<T, E, false>, dim3(n_ctas), dim3(kRouteThreads),
                                        0, st, logits, a.n_tokens, a.ld, a.bias, p, rows_per_cta, a.expert, a.weight, counts, ctx->s.status);
            });
        else
            e = by_row_width(p.n_experts, [&](auto v) {
                constexpr int V = decltype(v)::value;
                return launch_dependent(route_rows_kernel<T, V>, dim3(n_ctas), dim3(kRouteThreads), 0, st, logits, a.n_tokens, a.ld,
                                        whole_rows<T, V>(a.ld, p.n_experts), a.bias, p, rows_per_cta, a.expert, a.weight, counts, ctx->s.status);
            });
    }
    if (e != cudaSuccess || !counts) return e;
    const int warps = kRouteThreads / 32;
    if (tokens) {
        const size_t smem = sizeof(int) * ((size_t)kRouteThreads * p.n_experts + 3 * p.n_experts + 1);
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        return launch_dependent(route_place_runs_kernel, dim3(n_ctas), dim3(kRouteThreads), smem, st, (const int32_t *)a.expert,
                                a.n_tokens * p.top_k, p.top_k, rows_per_cta * p.top_k, p.n_experts,
                                (const int *)counts, a.offsets, a.row_token, a.token_row);
    }
    {
        LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
        e = launch_dependent(route_prefix_kernel, dim3((p.n_experts + warps - 1) / warps), dim3(kRouteThreads), 0, st,
                             counts, p.n_experts, n_ctas);
    }
    if (e != cudaSuccess) return e;
    const size_t smem = sizeof(int) * ((size_t)warps * p.n_experts + p.n_experts + 1);
    LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
    return launch_dependent(route_place_kernel, dim3(n_ctas), dim3(kRouteThreads), smem, st, (const int32_t *)a.expert,
                            a.n_tokens * p.top_k, p.top_k, rows_per_cta * p.top_k, p.n_experts,
                            (const int *)counts, a.offsets, a.row_token, a.token_row);
}

template <typename T> cudaError_t route_backward_as(gs_ctx *ctx, const ExpertRouteGradArgs &a, cudaStream_t st) {
    const RouterParams p = params_of(a.r);
    const bool tokens = p.n_experts <= kTokenExperts;
    const int at_once = tokens ? kRouteThreads : kRouteThreads / 32;
    const int64_t want = (a.n_tokens + at_once - 1) / at_once, most = (int64_t)ctx->n_sm * 16;
    const dim3 grid((unsigned)(want < most ? want : most));
    LaunchTimer t(ctx, GS_K_EXPERT_ROUTE, st);
    if (tokens)
        return by_token_width(p.n_experts, [&](auto v) {
            return launch_dependent(route_tokens_backward_kernel<T, decltype(v)::value>, grid, dim3(kRouteThreads), 0, st,
                                    (const T *)a.logits, a.n_tokens, a.ld, p, a.expert, a.d_weight, (T *)a.d_logits, a.ld_d, ctx->s.status);
        });
    return by_row_width(p.n_experts, [&](auto v) {
        constexpr int V = decltype(v)::value;
        return launch_dependent(route_rows_backward_kernel<T, V>, grid, dim3(kRouteThreads), 0, st, (const T *)a.logits, a.n_tokens, a.ld,
                                whole_rows<T, V>(a.ld, p.n_experts), p, a.expert, a.d_weight, (T *)a.d_logits, a.ld_d,
                                whole_rows<T, V>(a.ld_d, p.n_experts), ctx->s.status);
    });
}

}  // namespace

cudaError_t launch_expert_route(gs_ctx *ctx, const ExpertRouteArgs &a, cudaStream_t st) {
    return a.dtype == GS_F32 ? route_as<float>(ctx, a, st)
         : a.dtype == GS_BF16 ? route_as<__nv_bfloat16>(ctx, a, st) : route_as<__half>(ctx, a, st);
}

cudaError_t launch_expert_route_backward(gs_ctx *ctx, const ExpertRouteGradArgs &a, cudaStream_t st) {
    return a.dtype == GS_F32 ? route_backward_as<float>(ctx, a, st)
         : a.dtype == GS_BF16 ? route_backward_as<__nv_bfloat16>(ctx, a, st) : route_backward_as<__half>(ctx, a, st);
}

}  // namespace gs
