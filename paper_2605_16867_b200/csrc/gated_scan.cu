// Gated recurrence over ragged sequences, and its gradient.
//   a = s(g),  h = a h + (1 - a) x;      dh_t = dy_t + a_{t+1} dh_{t+1},  dx = (1 - a) dh,  dg = a (1 - a) (h_{t-1} - x) dh
//
// A block of GS_SCAN_BLOCK rows of 64 columns (two a lane) is a map of the state, h -> A h + B, that a warp
// finds in registers; the warps of a CTA take consecutive blocks, exchange their maps through shared memory,
// and each then goes through its block again from the state that the maps before it give.  Where there are few
// sequences, the CTAs of a cluster take consecutive tiles and exchange theirs.  So every value is read once: tensor-map
// copies bring the next tiles into a ring of shared-memory stages meanwhile.  States are in float; the gradient gets
// h_{t-1} from the states that the forward direction left before every block (half a byte a value in place of the two of
// the answers, and not rounded).
//
// Bound by instruction issue as much as by memory: two columns share theirs (packed float instructions), and a
// gate takes one exponential and one reciprocal for both of its factors; 21 instructions a value forwards in long sequences
// (48 % of the issue slots), 29 forwards and 42 backwards where four warps share a sequence (71 and 62 %).  4 x 32,768 rows of 1024
// in 16 bits: 188 us = 4.3 TB/s, backwards 322 us = 4.2 TB/s (half as wide in 32 bits 145 us = 5.6 TB/s and 211 us = 6.4 TB/s); 500
// windows of up to 512 rows, 520 wide: 96 us forwards with the states kept and 146 backwards, 263 us a step, which is 3.1 TB/s of
// the 803 MB that it cannot do without; 4,096 sequences of one row of 1024: 13.9 us = 4.2 TB/s (32 bits: 16.8 us = 5.0 TB/s).
#include <type_traits>

#include "operators.cuh"
#include "pairs.cuh"
#include "tensor_core.cuh"
#include "tensor_map.cuh"

namespace gs {
namespace {

using namespace tc;

constexpr int kRows = GS_SCAN_BLOCK;
constexpr int kColumns = 64;                   // of a warp: two a lane
constexpr int kMaxCluster = 8;

// Two neighbouring columns of a row as they are kept.
template <typename T> struct Pair { using Raw = uint32_t; };
template <> struct Pair<float> { using Raw = float2; };

template <typename T> __device__ __forceinline__ float2 unpack(typename Pair<T>::Raw v) {
    if constexpr (std::is_same<T, float>::value) return v;
    else return unpack2<T>(v);
}
template <typename T> __device__ __forceinline__ typename Pair<T>::Raw packed(float2 v) {
    if constexpr (std::is_same<T, float>::value) return v;
    else return pack2<T>(v.x, v.y);
}
// Columns of a pair that are there, 2, 1 or none, where `left` follow from its first one on.  (A sum of comparisons: a number
// held to 0 .. 2 by max and min and then compared with 2 under another condition, as `i < rows` of an unrolled loop is, nvcc
// 12.9.86 compiles wrongly for sm_100a.  Row 1 of a block was not written then, or written past the last column; a kernel of
// twenty lines does it too.)
__device__ __forceinline__ int pair_count(int left) { return (left > 0) + (left > 1); }
template <typename T> __device__ __forceinline__ typename Pair<T>::Raw load_pair(const T *p, int count) {
    typename Pair<T>::Raw v = {};
    if (count == 2) v = *reinterpret_cast<const typename Pair<T>::Raw *>(p);
    else if (count == 1) *reinterpret_cast<T *>(&v) = *p;
    return v;
}
template <typename T> __device__ __forceinline__ void store_pair(T *p, int count, float2 v) {
    const typename Pair<T>::Raw r = packed<T>(v);
    if (count == 2) *reinterpret_cast<typename Pair<T>::Raw *>(p) = r;
    else if (count == 1) *p = *reinterpret_cast<const T *>(&r);
}

// ---- gates --------------------------------------------------------------------------------------

// Gates held inside [-87, 89], so that s stays a normal float and 1 - s, below the smallest one from 87.34 on, becomes zero.
constexpr float kLeastGate = -87.f, kMostGate = 89.f;
template <typename T> __device__ __forceinline__ float2 gate_values(typename Pair<T>::Raw g) {
    if constexpr (std::is_same<T, float>::value) {
        float2 v;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(v.x) : "f"(g.x), "f"(kLeastGate));
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(v.y) : "f"(g.y), "f"(kLeastGate));
        asm("min.NaN.f32 %0, %1, %2;" : "=f"(v.x) : "f"(v.x), "f"(kMostGate));
        asm("min.NaN.f32 %0, %1, %2;" : "=f"(v.y) : "f"(v.y), "f"(kMostGate));
        return v;
    } else {
        uint32_t v;
        if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(v) : "r"(g), "r"(0xC2AEC2AEu));       // -87
            asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(v) : "r"(v), "r"(0x42B242B2u));       // 89
        } else {
            asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(v) : "r"(g), "r"(0xD570D570u));
            asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(v) : "r"(v), "r"(0x55905590u));
        }
        return unpack<T>(v);
    }
}
// Where a gate is +infinity nothing was observed: x there becomes zero, whatever it is.
template <typename T, int kCount> __device__ __forceinline__ void leave_out(const typename Pair<T>::Raw (&g)[kCount], typename Pair<T>::Raw (&x)[kCount]) {
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if (g[i].x == INFINITY) x[i].x = 0.f;
            if (g[i].y == INFINITY) x[i].y = 0.f;
        }
    } else {
        constexpr uint32_t kInf = std::is_same<T, __nv_bfloat16>::value ? 0x7F80u : 0x7C00u;
        uint32_t top = g[0];                     // one look for all rows
#pragma unroll
        for (int i = 1; i < kCount; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) asm("max.bf16x2 %0, %1, %2;" : "=r"(top) : "r"(top), "r"(g[i]));
            else asm("max.f16x2 %0, %1, %2;" : "=r"(top) : "r"(top), "r"(g[i]));
        }
        if ((top & 0xFFFFu) == kInf || top >> 16 == kInf) {
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                if ((g[i] & 0xFFFFu) == kInf) x[i] &= 0xFFFF0000u;
                if (g[i] >> 16 == kInf) x[i] &= 0x0000FFFFu;
            }
        }
    }
}

// a = s(g) = 1 / (1 + e) and c = 1 - s(g) = e / (1 + e) with e = exp(-g), each to a few units of its last place.  e is 2^t for
// t = -g log2(e) rounded.  What t is off by is had exactly from a fused multiply-add (the error-free product of Ogita, Rump and Oishi
// 2005), with what the factor itself lacks of log2(e) (a constant in two parts, as in Cody and Waite 1980), and is made good to first
// order: 2^off = 1 + off ln 2.  Of e alone, that makes both factors right.
// (The factors are held in registers: as constants each use of a pair would be two moves.)
struct GateFactors {
    float2 log2_e = held(1.44269504f), minus = held(-1.44269504f), rest = held(-1.92596299e-8f), ln_2 = held(0.693147181f), one = held(1.f);
};
__device__ __forceinline__ void gate_of(const GateFactors &f, float2 g, float2 &a, float2 &c) {
    const float2 t = mul2(g, f.minus);
    const float2 off = fma2(g, f.rest, fma2(g, f.minus, mul2(g, f.log2_e)));
    float2 e, n;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(t.y));
    e = fma2(mul2(e, off), f.ln_2, e);
    n = add2(e, f.one);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(n.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(n.y));
    c = mul2(e, a);
}

// ---- maps of the state ----------------------------------------------------------------------------

struct Map { float2 a, b; };                    // h -> a h + b
__device__ __forceinline__ float2 apply(const Map &m, float2 h) { return fma2(m.a, h, m.b); }
__device__ __forceinline__ Map then(const Map &first, const Map &second) { return {mul2(second.a, first.a), fma2(second.a, first.b, second.b)}; }
__device__ __forceinline__ Map nothing() { return {both(1.f), both(0.f)}; }
__device__ __forceinline__ Map map_of(const float4 &v) { return {make_float2(v.x, v.y), make_float2(v.z, v.w)}; }
__device__ __forceinline__ float4 kept(const Map &m) { return make_float4(m.a.x, m.a.y, m.b.x, m.b.y); }

// A sequence's rows; offsets may be anything: what is outside the rows is clamped.
struct Span {
    int begin, end;
    bool bad;
    __device__ __forceinline__ Span(const GatedScanArgs &p, int64_t s) {
        const int from = p.offsets[s], to = p.offsets[s + 1];
        begin = min(max(from, 0), p.n_rows);
        end = min(max(to, begin), p.n_rows);
        bad = from != begin || to != end;
    }
};
// Row of the kept states that belongs to the block of rows from t on.
__device__ __forceinline__ int64_t state_row(int begin, int64_t sequence, int t) { return begin / kRows + sequence + (t - begin) / kRows; }

// ---- long sequences -------------------------------------------------------------------------------

// A copy of a box of 64 columns; its bytes are reported to this CTA's barrier.
__device__ __forceinline__ void copy_box(const CUtensorMap *m, uint32_t dst, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(m), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// To the memory of any CTA of the cluster; its bytes are reported to a barrier there.
__device__ __forceinline__ void store_remote(uint32_t addr, uint32_t bar, const float4 &v) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_exchange() {     // writes to the other CTAs' memory before it are seen after it
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Whether a wait has run out.  The kernel then goes through the turns that are left, as the CTA's barriers want it to, each wait
// ending with its first try; but a barrier whose phase has not ended takes no further arrival, so nothing more is asked for.
__device__ __forceinline__ bool failed_yet(const int *failed) { return *(const volatile int *)failed; }

constexpr int kSkip = 3;

// kWarps of a CTA take kBlock rows each in a turn.  Forwards 16 rows of 16-bit values: what a turn costs beside its rows (the
// exchange, addresses, waiting) is as many instructions as eight rows.
template <typename T, int kWarps_, bool kBack> struct Shape {
    static constexpr int kWarps = kWarps_, kThreads = 32 * kWarps;
    static constexpr int kBlock = kBack || sizeof(T) == 4 || kWarps <= 4 ? kRows : 2 * kRows;
    static constexpr int kTile = kWarps * kBlock;                             // rows
    static constexpr uint32_t kArray = kTile * kColumns * sizeof(T);
    static constexpr int kArrays = kBack ? 3 : 2;
    static constexpr uint32_t kStage = kArrays * kArray;
    static constexpr bool kWide = kWarps > 4;                                 // (the shape that clusters are made of)
    static constexpr int kStages = kWide && !(kBack && sizeof(T) == 2) ? 2 : 3;      // (what fits beside the CTAs of an SM; wide and backwards, 32 bits take 96 KB a stage)
    static constexpr int kClusters = kWide ? kMaxCluster : 1;
    static constexpr int kCtasPerSm = kWide ? (kBack || sizeof(T) == 4 ? 1 : 2) : kBack ? 4 : 7;
    struct Exchange {
        float4 maps[2][kSkip + kWarps][32];    // (the first ones change nothing: a warp goes through four at a time, up to its own)
        float4 totals[2][kClusters][32];       // of the cluster's CTAs
        float2 carry[2][32];
        uint64_t full[kStages], told[2];
        int failed;
    };
    static constexpr size_t kSmem = 128 + kStages * kStage + sizeof(Exchange);
};
template <typename T, bool kBack> constexpr int kWideWarps = kBack || sizeof(T) == 4 ? 16 : 8;

// State before this warp's block, given its map and the state before the first CTA's tile.
template <int kWarps, typename Exchange>
__device__ __forceinline__ float2 state_before(Exchange *x, int turn, int order, int lane, const Map &m, float2 &carry, int ctas, int rank) {
    const int now = turn & 1;
    const float4 (*maps)[32] = x->maps[now] + kSkip;
    x->maps[now][kSkip + order][lane] = kept(m);
    __syncthreads();
    if (ctas == 1) {
        float2 h = turn == 0 ? carry : x->carry[now][lane];
#pragma unroll 1
        for (int w = -(-order & 3); w < order; w += 4) {
            Map next[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) next[i] = map_of(maps[w + i][lane]);
#pragma unroll
            for (int i = 0; i < 4; ++i) h = apply(next[i], h);
        }
        return h;
    }
    const bool failed = failed_yet(&x->failed);
    Map before = nothing();
#pragma unroll 1
    for (int w = -(-order & 3); w < order; w += 4) {
        Map next[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = map_of(maps[w + i][lane]);
#pragma unroll
        for (int i = 0; i < 4; ++i) before = then(before, next[i]);
    }
    // The last warp tells all CTAs its own one's map.  (They have read what the turn before last left there: each has
    // sent its map of the last turn since, and those are here.)
    if (order == kWarps - 1) {
        if (lane == 0 && !failed) expect(smem_u32(&x->told[now]), ctas * 32 * sizeof(float4));
        const float4 all = kept(then(before, m));
        for (int c = 0; c < ctas; ++c) store_remote(in_cta(smem_u32(&x->totals[now][rank][lane]), c), in_cta(smem_u32(&x->told[now]), c), all);
    }
    bar_wait(smem_u32(&x->told[now]), turn >> 1 & 1, &x->failed);
    float2 h = carry;
#pragma unroll 1
    for (int c = 0; c < ctas; ++c) {
        if (c == rank) h = carry;
        carry = apply(map_of(x->totals[now][c][lane]), carry);
    }
    return apply(before, h);
}

template <typename T, int kWarps, bool kBack>
__global__ void __launch_bounds__(32 * kWarps, Shape<T, kWarps, kBack>::kCtasPerSm)
gated_scan_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_gate,
                  const __grid_constant__ CUtensorMap map_d, const GatedScanArgs p)
{
    using S = Shape<T, kWarps, kBack>;
    using Raw = typename Pair<T>::Raw;
    constexpr int kBlock = S::kBlock;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((128 - (smem_u32(smem_raw) & 127)) & 127);
    typename S::Exchange *ex = reinterpret_cast<typename S::Exchange *>(smem + S::kStages * S::kStage);
    const int lane = threadIdx.x & 31, order = threadIdx.x >> 5;
    const int ctas = S::kWide ? (int)cluster_size() : 1, rank = S::kWide ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) bar_init(smem_u32(&ex->full[s]), 1);
        for (int i = 0; i < 2; ++i) bar_init(smem_u32(&ex->told[i]), 1);
        ex->failed = 0;
        bar_init_done();
        prefetch_map(&map_x);
        prefetch_map(&map_gate);
    }
    for (int i = threadIdx.x; i < 2 * kSkip * 32; i += S::kThreads) ex->maps[i / (kSkip * 32)][i / 32 % kSkip][i % 32] = kept(nothing());
    dependent_wait();
    const int strips = (p.features + kColumns - 1) / kColumns, item = blockIdx.x / ctas;
    const int sequence = item / strips, col0 = item % strips * kColumns, col = col0 + lane * 2;
    const int count = pair_count(p.features - col);
    // The state before the sequence is read ahead of the barriers: whoever writes the one after it, perhaps over the same memory
    // (out_last may be h0), does so behind them, whichever CTA of the cluster it is.
    const float *start = kBack ? p.d_last : p.h0;
    float2 carry = both(0.f);
    if (start) carry = unpack<float>(load_pair(start + sequence * (kBack ? p.ld_d_last : p.ld_h0) + col, count));
    __syncthreads();
    if (ctas > 1) cluster_exchange();

    const Span span(p, sequence);
    const int begin = span.begin, end = span.end;
    if (span.bad && threadIdx.x == 0 && col0 == 0) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
    if (begin == end) {
        float *to = kBack ? p.d_h0 : p.last;
        if (to && order == 0 && rank == 0) store_pair(to + sequence * (kBack ? p.ld_d_h0 : p.ld_last) + col, count, carry);
    }
    // Rows by turns of all CTAs' tiles: forwards from the first row on; backwards up to the end of the last block, so that the
    // first tiles may begin before the sequence, and before the matrix.
    const int step = (kBack ? -1 : 1) * S::kTile * ctas, turns = (end - begin + S::kTile * ctas - 1) / (S::kTile * ctas);
    int row = kBack ? begin + (end - begin + kBlock - 1) / kBlock * kBlock - (rank + 1) * S::kTile : begin + rank * S::kTile;   // of this CTA's tile
    // (a tile without rows is not copied; that is a CTA's last one at most)
    const auto there = [&](int first) { return kBack ? first + S::kTile > begin : first < end; };
    const auto copy = [&](int stage, int first) {
        if (!there(first)) return;
        const uint32_t bar = smem_u32(&ex->full[stage]), to = smem_u32(smem + stage * S::kStage);
        const bool with_d = kBack && p.d_out;
        expect(bar, (with_d ? 3 : 2) * S::kArray);
        copy_box(&map_gate, to, bar, col0, first);
        copy_box(&map_x, to + S::kArray, bar, col0, first);
        if (with_d) copy_box(&map_d, to + 2 * S::kArray, bar, col0, first);
    };
    if (threadIdx.x == 0)
        for (int k = 0; k < S::kStages && k < turns; ++k) copy(k, row + k * step);

    const int in_tile = (kBack ? kWarps - 1 - order : order) * kBlock;
    int t = row + in_tile;                       // of this warp's block
    const int64_t state_step = (int64_t)step / kRows * p.ld_states;
    float *states = p.states + state_row(begin, sequence, t) * p.ld_states + col;      // (its row may lie outside: then it is not touched)
    T *out = (T *)(kBack ? p.dx : p.out) + (int64_t)t * (kBack ? p.ld_dx : p.ld_out) + col, *d_gate = (T *)p.d_gate + (int64_t)t * p.ld_d_gate + col;
    const int64_t out_step = (int64_t)step * (kBack ? p.ld_dx : p.ld_out), d_gate_step = (int64_t)step * p.ld_d_gate;
    [[maybe_unused]] float2 next_state = both(0.f);          // (gradient) before this warp's block of the next turn
    if (kBack) next_state = unpack<float>(load_pair(states, t >= begin ? count : 0));
    const bool whole_strip = col0 + kColumns <= p.features;
    const GateFactors factors;
    int stage = 0, phase = 0;
#pragma unroll 1
    for (int turn = 0; turn < turns; ++turn) {
        const int rows = kBack && t < begin ? 0 : max(0, min(kBlock, end - t));       // of this warp's block that are the sequence's
        if (there(row)) bar_wait(smem_u32(&ex->full[stage]), phase, &ex->failed);
        const Raw *gates = reinterpret_cast<const Raw *>(smem + stage * S::kStage) + in_tile * 32 + lane;
        constexpr int kNext = S::kArray / sizeof(Raw);
        float2 a[kBlock], b[kBlock];             // forwards b = (1 - a) x; backwards what comes in from the answers
        [[maybe_unused]] float2 c[kBlock], slope[kBlock];
        Map m = nothing();
        float2 h = next_state;
#pragma unroll
        for (int i0 = 0; i0 < kBlock; i0 += kRows) {
            Raw rg[kRows], rx[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) { rg[i] = gates[(i0 + i) * 32]; rx[i] = gates[kNext + (i0 + i) * 32]; }
            leave_out<T>(rg, rx);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const float2 x = unpack<T>(rx[i]);
                float2 k;
                gate_of(factors, gate_values<T>(rg[i]), a[i0 + i], k);
                const float2 in = mul2(k, x);
                if constexpr (kBack) {
                    c[i] = k;
                    slope[i] = mul2(mul2(a[i], k), fma2(x, both(-1.f), h));
                    h = fma2(a[i], h, in);
                    b[i] = p.d_out ? unpack<T>(gates[2 * kNext + i * 32]) : both(0.f);
                } else b[i0 + i] = in;
            }
        }
        if (rows < kBlock)
#pragma unroll
            for (int i = 0; i < kBlock; ++i)
                if (i >= rows) { a[i] = both(1.f); b[i] = both(0.f); }
        if constexpr (kBack) {
            states += state_step;
            next_state = unpack<float>(load_pair(states, turn + 1 < turns && t + step >= begin ? count : 0));
#pragma unroll
            for (int i = kBlock - 1; i >= 0; --i) {
                m.b = mul2(a[i], add2(b[i], m.b));
                m.a = mul2(m.a, a[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kBlock; ++i) m = then(m, {a[i], b[i]});
        }
        h = state_before<kWarps>(ex, turn, order, lane, m, carry, ctas, rank);
        if (threadIdx.x == 0 && turn + S::kStages < turns && !failed_yet(&ex->failed)) copy(stage, row + S::kStages * step);     // (every warp has read this stage)
        if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        // (blocks that are there whole, most of them: nothing to look at row by row)
        const bool whole = rows == kBlock && whole_strip;
        if constexpr (!kBack) {
            T *to = out;
            const bool writes = whole && p.out;
#pragma unroll
            for (int i0 = 0; i0 < kBlock; i0 += kRows) {
                if (p.states) store_pair(states + i0 / kRows * p.ld_states, i0 < rows ? count : 0, h);
                if (writes) {
#pragma unroll
                    for (int i = i0; i < i0 + kRows; ++i) {
                        h = apply({a[i], b[i]}, h);
                        *reinterpret_cast<Raw *>(to) = packed<T>(h);
                        to += p.ld_out;
                    }
                } else {
#pragma unroll
                    for (int i = i0; i < i0 + kRows; ++i) {
                        h = apply({a[i], b[i]}, h);
                        store_pair(to, p.out && i < rows ? count : 0, h);
                        to += p.ld_out;
                    }
                }
            }
            if (p.last && t + rows == end) store_pair(p.last + sequence * p.ld_last + col, rows ? count : 0, h);
            states += state_step;
        } else {
            T *to = out + (kBlock - 1) * p.ld_dx, *to_gate = d_gate + (kBlock - 1) * p.ld_d_gate;
            if (whole && p.dx && p.d_gate) {
#pragma unroll
                for (int i = kBlock - 1; i >= 0; --i) {
                    const float2 dh = add2(b[i], h);
                    h = mul2(a[i], dh);
                    *reinterpret_cast<Raw *>(to) = packed<T>(mul2(c[i], dh));
                    *reinterpret_cast<Raw *>(to_gate) = packed<T>(mul2(slope[i], dh));
                    to -= p.ld_dx;
                    to_gate -= p.ld_d_gate;
                }
            } else {
#pragma unroll
                for (int i = kBlock - 1; i >= 0; --i) {
                    const float2 dh = add2(b[i], h);
                    h = mul2(a[i], dh);
                    store_pair(to, p.dx && i < rows ? count : 0, mul2(c[i], dh));
                    store_pair(to_gate, p.d_gate && i < rows ? count : 0, mul2(slope[i], dh));
                    to -= p.ld_dx;
                    to_gate -= p.ld_d_gate;
                }
            }
            if (p.d_h0 && t == begin) store_pair(p.d_h0 + sequence * p.ld_d_h0 + col, count, h);
            d_gate += d_gate_step;
        }
        out += out_step;
        t += step;
        row += step;
        if (ctas == 1 && order == kWarps - 1) ex->carry[(turn + 1) & 1][lane] = h;
    }
    __syncthreads();
    if (ctas > 1) cluster_exchange();            // (nobody leaves while others may still write to its memory)
    if (threadIdx.x == 0 && ex->failed) {
        atomicOr(p.status, (unsigned)GS_DEV_TIMEOUT);
        const long long from = clock64();        // copies still under way have to land first
        while (clock64() - from < 2000000ll) { }
    }
    dependent_end();
}

// ---- short sequences ------------------------------------------------------------------------------

// A thread takes two columns of a sequence, block after block.
constexpr int kShortThreads = 128;

template <typename T, bool kBack>
__global__ void __launch_bounds__(kShortThreads)
gated_scan_short_kernel(const GatedScanArgs p)
{
    using Raw = typename Pair<T>::Raw;
    dependent_wait();
    const int64_t pairs = (p.features + 1) / 2, item = (int64_t)blockIdx.x * kShortThreads + threadIdx.x;
    const int64_t sequence = item / pairs;
    if (sequence >= p.n_sequences) return;
    const int col = (int)(item % pairs) * 2, count = pair_count(p.features - col);
    const Span span(p, sequence);
    const int begin = span.begin, end = span.end;
    if (span.bad && col == 0) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
    const float *start = kBack ? p.d_last : p.h0;
    float2 h = both(0.f);
    if (start) h = unpack<float>(load_pair(start + sequence * (kBack ? p.ld_d_last : p.ld_h0) + col, count));
    const int blocks = (end - begin + kRows - 1) / kRows;
    const GateFactors factors;
    for (int q = 0; q < blocks; ++q) {
        const int t = begin + (kBack ? blocks - 1 - q : q) * kRows, rows = min(kRows, end - t);
        Raw gates[kRows], xs[kRows], ds[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int there = i < rows ? count : 0;
            gates[i] = load_pair((const T *)p.gate + (int64_t)(t + i) * p.ld_gate + col, there);
            xs[i] = load_pair((const T *)p.x + (int64_t)(t + i) * p.ld_x + col, there);
            if (kBack) ds[i] = load_pair((const T *)p.d_out + (int64_t)(t + i) * p.ld_d_out + col, p.d_out ? there : 0);
        }
        leave_out<T>(gates, xs);
        float2 a[kRows], c[kRows], slope[kRows], before = both(0.f);
        if (kBack) before = unpack<float>(load_pair(p.states + state_row(begin, sequence, t) * p.ld_states + col, count));
        else store_pair(p.states + state_row(begin, sequence, t) * p.ld_states + col, p.states ? count : 0, h);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (i >= rows) break;
            const float2 x = unpack<T>(xs[i]);
            gate_of(factors, gate_values<T>(gates[i]), a[i], c[i]);
            if constexpr (kBack) {
                slope[i] = mul2(mul2(a[i], c[i]), make_float2(before.x - x.x, before.y - x.y));
                before = fma2(a[i], before, mul2(c[i], x));
            } else {
                h = fma2(a[i], h, mul2(c[i], x));
                store_pair((T *)p.out + (int64_t)(t + i) * p.ld_out + col, p.out ? count : 0, h);
            }
        }
        if constexpr (kBack) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i) {
                if (i >= rows) continue;
                const float2 dh = add2(unpack<T>(ds[i]), h);
                h = mul2(a[i], dh);
                store_pair((T *)p.dx + (int64_t)(t + i) * p.ld_dx + col, p.dx ? count : 0, mul2(c[i], dh));
                store_pair((T *)p.d_gate + (int64_t)(t + i) * p.ld_d_gate + col, p.d_gate ? count : 0, mul2(slope[i], dh));
            }
        }
    }
    float *to = kBack ? p.d_h0 : p.last;
    store_pair(to + sequence * (kBack ? p.ld_d_h0 : p.ld_last) + col, to ? count : 0, h);
    dependent_end();
}

// A row or two a sequence, forwards (serving: every state takes one more): a thread takes four columns of a sequence,
// row after row, and asks for the next one meanwhile.
constexpr int kStepThreads = 128;

template <typename T> struct Four {
    typename Pair<T>::Raw v[2];
    __device__ __forceinline__ void ask(const T *p, int left) {
        if (left >= 4) {
            if constexpr (sizeof(T) == 2) { const uint2 q = *reinterpret_cast<const uint2 *>(p); v[0] = q.x; v[1] = q.y; }
            else { const float4 q = *reinterpret_cast<const float4 *>(p); v[0] = make_float2(q.x, q.y); v[1] = make_float2(q.z, q.w); }
        } else {
            v[0] = load_pair(p, pair_count(left));
            v[1] = load_pair(p + 2, pair_count(left - 2));
        }
    }
};
template <typename T> __device__ __forceinline__ void store_four(T *p, int left, const float2 (&h)[2]) {
    if (left >= 4) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(packed<T>(h[0]), packed<T>(h[1]));
        else *reinterpret_cast<float4 *>(p) = make_float4(h[0].x, h[0].y, h[1].x, h[1].y);
    } else {
        store_pair(p, pair_count(left), h[0]);
        store_pair(p + 2, pair_count(left - 2), h[1]);
    }
}

template <typename T>
__global__ void __launch_bounds__(kStepThreads, 12)
gated_scan_step_kernel(const GatedScanArgs p, unsigned fours)
{
    dependent_wait();
    const int64_t first = (int64_t)blockIdx.x * kStepThreads, sequence0 = first / fours;
    const unsigned at = (unsigned)(first - sequence0 * fours) + threadIdx.x, over = at / fours;
    const int64_t sequence = sequence0 + over;
    if (sequence >= p.n_sequences) return;
    const int col = (int)(at - over * fours) * 4, left = p.features - col;
    Four<float> start;
    if (p.h0) start.ask(p.h0 + sequence * p.ld_h0 + col, left);
    else start.v[0] = start.v[1] = both(0.f);
    const Span span(p, sequence);
    if (span.bad && col == 0) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
    Four<T> x, gate;
    const auto ask = [&](int t) {
        if (t >= span.end) return;
        x.ask((const T *)p.x + (int64_t)t * p.ld_x + col, left);
        gate.ask((const T *)p.gate + (int64_t)t * p.ld_gate + col, left);
    };
    ask(span.begin);
    const GateFactors factors;
    float2 h[2] = {start.v[0], start.v[1]};
    for (int t = span.begin; t < span.end; ++t) {
        if (p.states && (t - span.begin) % kRows == 0) store_four(p.states + state_row(span.begin, sequence, t) * p.ld_states + col, left, h);
        typename Pair<T>::Raw rx[2] = {x.v[0], x.v[1]}, rg[2] = {gate.v[0], gate.v[1]};
        ask(t + 1);
        leave_out<T>(rg, rx);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float2 a, c;
            gate_of(factors, gate_values<T>(rg[i]), a, c);
            h[i] = fma2(a, h[i], mul2(c, unpack<T>(rx[i])));
        }
        if (p.out) store_four((T *)p.out + (int64_t)t * p.ld_out + col, left, h);
    }
    if (p.last) store_four(p.last + sequence * p.ld_last + col, left, h);
    dependent_end();
}

// ---- host side --------------------------------------------------------------------------------------

template <typename T, bool kBack> cudaError_t launch_short(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st) {
    const int64_t ctas = (a.n_sequences * ((a.features + 1) / 2) + kShortThreads - 1) / kShortThreads;
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    LaunchTimer t(ctx, GS_K_GATED_SCAN, st);
    return launch_dependent(gated_scan_short_kernel<T, kBack>, dim3((unsigned)ctas), dim3(kShortThreads), 0, st, a);
}

template <typename T> cudaError_t launch_step(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st) {
    const int64_t fours = (a.features + 3) / 4, ctas = (a.n_sequences * fours + kStepThreads - 1) / kStepThreads;
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    LaunchTimer t(ctx, GS_K_GATED_SCAN, st);
    return launch_dependent(gated_scan_step_kernel<T>, dim3((unsigned)ctas), dim3(kStepThreads), 0, st, a, (unsigned)fours);
}

bool encode_tiles(CUtensorMap *map, int dtype, const void *base, int64_t rows, int64_t ld, int features, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)features, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * (dtype == GS_F32 ? 4 : 2)};
    const cuuint32_t box[2] = {kColumns, (cuuint32_t)box_rows};
    return encode_map(map, dtype, base, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <typename T, int kWarps, bool kBack> cudaError_t launch_tiles(gs_ctx *ctx, const GatedScanArgs &a, int cluster, cudaStream_t st) {
    using S = Shape<T, kWarps, kBack>;
    CUtensorMap x, gate, d;
    if (!encode_tiles(&x, a.dtype, a.x, a.n_rows, a.ld_x, a.features, S::kTile) || !encode_tiles(&gate, a.dtype, a.gate, a.n_rows, a.ld_gate, a.features, S::kTile))
        return cudaErrorInvalidValue;
    d = x;
    if (kBack && a.d_out && !encode_tiles(&d, a.dtype, a.d_out, a.n_rows, a.ld_d_out, a.features, S::kTile)) return cudaErrorInvalidValue;
    const int64_t ctas = a.n_sequences * ((a.features + kColumns - 1) / kColumns) * cluster;
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    LaunchTimer t(ctx, GS_K_GATED_SCAN, st);
    return cudaLaunchKernelEx(&cfg, gated_scan_kernel<T, kWarps, kBack>, x, gate, d, a);
}

// The shape of the kernel by the sequences' average length and their number.
//   a row or two: four columns a thread (4,096 x 1024, one row each: 14 us, with blocks of eight rows 47 us); up to a block: a
//   thread per two columns; up to 64 rows, or where there are strips enough to fill the GPU eight times over: four warps a
//   sequence (500 windows of 256 rows on average, 520 wide: 97 us forwards and 144 backwards; with the wide shape 135 and 250);
//   else the wide shape, with clusters along the sequence while the GPU has room for them (4 x 32,768 x 1024: clusters of two
//   295 us, of four 187).
// The lengths are known on the device alone: a long sequence among many short ones takes their shape (4,096 of one row and one of
// 4,000, 1024 wide: 1.5 ms forwards and 6.5 backwards, where the long one by itself takes 15 and 28 us).
template <typename T, bool kBack> cudaError_t scan_as(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st) {
    constexpr int W = kWideWarps<T, kBack>;
    using S = Shape<T, W, kBack>;
    const int64_t each = a.n_rows / a.n_sequences, items = a.n_sequences * ((a.features + kColumns - 1) / kColumns);
    if (!kBack && each <= 2) return launch_step<T>(ctx, a, st);
    if (each <= kRows) return launch_short<T, kBack>(ctx, a, st);
    if (each <= 64 || items >= 8 * ctx->n_sm) return launch_tiles<T, 4, kBack>(ctx, a, 1, st);
    int cluster = 1;
    while (cluster < kMaxCluster && items * cluster * 2 <= S::kCtasPerSm * ctx->n_sm && each >= (int64_t)cluster * 2 * S::kTile) cluster *= 2;
    return launch_tiles<T, W, kBack>(ctx, a, cluster, st);
}

template <bool kBack> cudaError_t scan_by_type(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st) {
    if (a.dtype == GS_F32) return scan_as<float, kBack>(ctx, a, st);
    return a.dtype == GS_BF16 ? scan_as<__nv_bfloat16, kBack>(ctx, a, st) : scan_as<__half, kBack>(ctx, a, st);
}

template <typename T, int kWarps, bool kBack> cudaError_t configure_tiles() {
    return cudaFuncSetAttribute(gated_scan_kernel<T, kWarps, kBack>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<T, kWarps, kBack>::kSmem);
}
template <typename T> cudaError_t configure_as() {
    for (auto f : {configure_tiles<T, 4, false>, configure_tiles<T, 4, true>, configure_tiles<T, kWideWarps<T, false>, false>, configure_tiles<T, kWideWarps<T, true>, true>}) {
        const cudaError_t e = f();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t configure_gated_scan() {
    cudaError_t e = configure_as<float>();
    if (e == cudaSuccess) e = configure_as<__nv_bfloat16>();
    return e == cudaSuccess ? configure_as<__half>() : e;
}

cudaError_t launch_gated_scan(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st) { return scan_by_type<false>(ctx, a, st); }
cudaError_t launch_gated_scan_backward(gs_ctx *ctx, const GatedScanArgs &a, cudaStream_t st) { return scan_by_type<true>(ctx, a, st); }

}  // namespace gs
