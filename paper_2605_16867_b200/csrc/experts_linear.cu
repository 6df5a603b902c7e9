// Products with the experts' weights, on the tensor cores:
//   forward   y[r]  = act(x[t(r)] W_e^T + b_e)         per row r of expert e
//   backward  dx[r] = dz[r] W_e  (zero where x[t(r)] <= 0),   dW_e = sum_r dz[r]^T x[t(r)],   db_e = sum_r dz[r]
//
// Every kernel is persistent: one pair of CTAs per pair of SMs takes tiles in turn, and its warps have
// fixed parts: warp 0 copies operand tiles into a ring of shared-memory stages (with gathered rows
// others issue the gathers), warp 1 of the leader issues the matrix instructions, four or eight move
// finished sums from tensor memory to global memory while the next tile is already being summed
// (two sets of sums in tensor memory).  Which rows belong to which expert is read from the offsets
// on the device; the host knows only their number.
//
// In y and dx the tile's 256 "M" rows are weights (features of the result), its "N" columns are
// requests: few rows per expert then cost little (N can be small, the weights are read once), and
// with many rows a pair reads 64 KB per 64 of the contraction for 256 x 256 results.  Bound by the
// matrix instructions and the power they take: 65,536 rows each twice, 2048 to 1024, read in order, take 417 us in
// two passes after a pause = 1.32 PFLOP/s, 78 % of a library product's burst on the same card, and 462 us repeated for
// seconds = 1.19 PFLOP/s, 83 % of its sustained rate (1,000 W, SM clock 1,207 MHz; gathered 469 and 522 us, 1,440 MHz).
// 669 cycles per step of 64 where the instructions need 512.
// Waiting on barriers with cluster-wide acquire and release cost half of that speed (695 TFLOP/s): the
// waits and arrivals below therefore order the CTA alone, and the one that follows plain writes to
// shared memory has its own fence.
#include <type_traits>

#include "operators.cuh"
#include "tensor_core.cuh"

namespace gs {
namespace {

using namespace tc;

constexpr int kDepth = 64;                      // of the contraction per stage: one 128-byte row of 16-bit values
constexpr int kHalfM = 128;                     // rows of the result per CTA of a pair
constexpr int kTileM = 2 * kHalfM;
constexpr uint32_t kABytes = kHalfM * 128;
constexpr int kWarpProducer = 0, kWarpMma = 1;
constexpr int kMaxStages = 10;
// A gather instruction fetches four rows, one lane at a time; one warp issues them in some 75 cycles
// each, far below what the copies could carry.  131,072 requests of the first layer in short runs with
// 1 / 4 / 8 / 16 warps: 2,160 / 970 / 889 / 877 us (eight warps at the power limit, 1,425 MHz: 1,035 us).
constexpr int kGatherWarps = 8;                 // (at most: four rows each are the least)

struct Barriers {
    uint64_t full[kMaxStages], empty[kMaxStages], landed[kMaxStages], sums_full[2], sums_empty[2];
    uint32_t tmem;
    int failed;
};

template <typename T> constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;

__device__ __forceinline__ void setup_pair(Barriers *b, int stages, int store_warps, int warp, int lane) {
    if (warp == 0 && lane == 0) {
        for (int s = 0; s < stages; ++s) {
            bar_init(smem_u32(&b->full[s]), 2);                 // one from each CTA, and its copies' bytes
            bar_init(smem_u32(&b->empty[s]), 1);
            bar_init(smem_u32(&b->landed[s]), 1);
        }
        for (int i = 0; i < 2; ++i) { bar_init(smem_u32(&b->sums_full[i]), 1); bar_init(smem_u32(&b->sums_empty[i]), 2 * store_warps); }
        b->failed = 0;
        bar_init_done();
    }
}

// Position in the ring of stages: stage and the parity of its current round.
struct Ring {
    int stage = 0, round = 0;
    __device__ __forceinline__ void next(int stages) { if (++stage == stages) { stage = 0; round ^= 1; } }
};

// By the copying warp at its end: every stage that it filled has been given back.  The matrix instructions'
// arrivals come from the other CTA too, and none may be under way to this one when it leaves.
__device__ __forceinline__ void wait_for_stages(Barriers *b, int stages, Ring ring, volatile int *failed) {
    for (int s = 0; s < stages; ++s) {
        if (!warp_wait(smem_u32(&b->empty[ring.stage]), ring.round ^ 1, failed)) return;
        ring.next(stages);
    }
}

// Rows of expert e = base + lane, for the lanes of one warp (all experts in turn).  Offsets may be
// anything: they are clamped into [0, n_rows] and made ascending, so that no two experts share a
// row; `before` carries the end of the last expert.
__device__ __forceinline__ int2 ascending_rows(const int32_t *__restrict__ offsets, int e, int n_experts, int n_rows, int lane, int *before) {
    int a = e < n_experts ? min(max(offsets[e], 0), n_rows) : 0, b = e < n_experts ? min(max(offsets[e + 1], 0), n_rows) : 0;
    a = max(a, *before);
    b = max(a, b);
    int most = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kFull, most, o);
        if (lane >= o) most = max(most, up);
    }
    const int up = __shfl_up_sync(kFull, most, 1);
    if (lane > 0) a = max(a, up);
    *before = __shfl_sync(kFull, most, 31);
    return make_int2(a, max(a, b));
}

// Where the rows of expert e begin and end, and the tiles of all experts before it.
__device__ __forceinline__ void scan_row_tiles(const int32_t *__restrict__ offsets, int n_experts, int n_rows, int rows_per_tile,
                                               int *tile_start, int *row_start, int *row_end, int lane) {
    int before = 0, end = 0;
    for (int base = 0; base < n_experts; base += 32) {
        const int e = base + lane;
        const int2 r = ascending_rows(offsets, e, n_experts, n_rows, lane, &end);
        const int own = (r.y - r.x + rows_per_tile - 1) / rows_per_tile;
        int sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFull, sum, o);
            if (lane >= o) sum += up;
        }
        if (e < n_experts) { tile_start[e] = before + sum - own; row_start[e] = r.x; row_end[e] = r.y; }
        before += __shfl_sync(kFull, sum, 31);
    }
    if (lane == 0) tile_start[n_experts] = before;
}

// A token index, held inside the matrix it points into.
__device__ __forceinline__ int safe_token(int t, int n, bool *bad) {
    if ((unsigned)t < (unsigned)n) return t;
    *bad = true;
    return min(max(t, 0), n - 1);
}

// ---- y and dx ---------------------------------------------------------------------------------

struct RowsArgs {
    const int32_t *offsets, *row_token;         // row_token: rows of the N operand (forward) or of the mask (backward)
    int n_experts, n_rows, n_tokens;            // n_tokens: rows that row_token points into
    int features, depth;                        // of the result; of the contraction
    const float *bias;
    bool relu;
    const void *mask;
    int64_t ld_mask;
    void *out;
    int64_t ld_out;
    unsigned *status;
};

template <int kN> struct RowsShape {
    static constexpr uint32_t kBBytes = kN / 2 * 128;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = kN == 256 ? 6 : kN == 128 ? 8 : kN == 64 ? 9 : 10;
    static constexpr int kStoreWarps = kN >= 64 ? 8 : 4;
    static constexpr int kStoreBytes = kStoreWarps * 2048;   // per warp: 32 requests x 32 features
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kStoreBytes + sizeof(Barriers) + (3 * GS_MAX_EXPERTS + 4) * sizeof(int);
    static constexpr int kTmem = 2 * kN < 32 ? 32 : 2 * kN;
    // Every gathering warp has rows: one without would follow the ring's barriers for nothing, and since no copy
    // of its own holds a stage back, could fall a round behind and then wait for a phase that never comes.
    static constexpr int kGatherers = kN / 8 < kGatherWarps ? kN / 8 : kGatherWarps;
    static constexpr int kGatherLanes = kN / (8 * kGatherers);                      // of each of them: four rows per lane
    static_assert(kGatherLanes >= 1 && kGatherers * kGatherLanes * 4 == kN / 2, "a gathering warp without rows");
    static constexpr int threads(bool gather) { return 32 * (2 + kStoreWarps + (gather ? kGatherers - 1 : 0)); }
};

// kDx: the weights' tile has its features contiguous (the contraction runs over their rows).
template <typename T, bool kDx, int kN, bool kGather>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(RowsShape<kN>::threads(kGather), 1)
rows_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const RowsArgs p)
{
    using S = RowsShape<kN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char *store = smem + S::kStages * S::kStageBytes;
    Barriers *bars = reinterpret_cast<Barriers *>(store + S::kStoreBytes);
    int *tile_start = reinterpret_cast<int *>(bars + 1), *row_start = tile_start + GS_MAX_EXPERTS + 1, *row_end = row_start + GS_MAX_EXPERTS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    volatile int *failed = &bars->failed;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    setup_pair(bars, S::kStages, S::kStoreWarps, warp, lane);
    if (warp == kWarpMma) tmem_alloc<S::kTmem>(smem_u32(&bars->tmem));
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 0) scan_row_tiles(p.offsets, p.n_experts, p.n_rows, kN, tile_start, row_start, row_end, lane);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();

    const uint32_t tmem = bars->tmem;
    const int m_tiles = (p.features + kTileM - 1) / kTileM, k_steps = (p.depth + kDepth - 1) / kDepth;
    const int64_t n_tiles = (int64_t)tile_start[p.n_experts] * m_tiles;
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

    if (warp == kWarpProducer || warp >= 2 + S::kStoreWarps) {
        const int helper = warp == kWarpProducer ? 0 : warp - (1 + S::kStoreWarps);     // the gathering warps share out the rows
        if (threadIdx.x == 0) { prefetch_map(&map_w); prefetch_map(&map_x); }
        Ring ring;
        int e = 0;
        bool bad = false, ok = true;
        for (int64_t t = pair; t < n_tiles && ok; t += n_pairs) {
            const int rt = (int)(t / m_tiles), m0 = (int)(t % m_tiles) * kTileM + (int)rank * kHalfM;
            while (tile_start[e + 1] <= rt) ++e;
            const int r0 = row_start[e] + (rt - tile_start[e]) * kN + (int)rank * (kN / 2);
            // (of the lanes' condition the second half always holds; without it the compiler issues the gathers
            // more slowly: 131,072 requests of the first layer 1,138 - 1,190 instead of 970 - 1,020 us, same registers)
            constexpr int kLanes = S::kGatherLanes;          // of each warp: four rows per lane
            const int row = (helper * kLanes + lane) * 4;
            int token[4];
            if (kGather && lane < kLanes && row < kN / 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    token[i] = safe_token(p.row_token[min(r0 + row + i, row_end[e] - 1)], p.n_tokens, &bad);
            }
            for (int k = 0; k < k_steps; ++k) {
                if (!warp_wait(smem_u32(&bars->empty[ring.stage]), ring.round ^ 1, failed)) { ok = false; break; }
                const uint32_t a = smem_u32(smem + ring.stage * S::kStageBytes), b = a + kABytes;
                const uint32_t full = in_leader(smem_u32(&bars->full[ring.stage]));
                if (lane == 0 && helper == 0) {
                    bar_expect(full, S::kStageBytes);
                    if (kDx) {
                        copy_3d(&map_w, a, full, m0, k * kDepth, e);
                        copy_3d(&map_w, a + kABytes / 2, full, m0 + 64, k * kDepth, e);
                    } else {
                        copy_3d(&map_w, a, full, k * kDepth, m0, e);
                    }
                    if (!kGather) copy_2d(&map_x, b, full, k * kDepth, r0);
                }
                if (kGather && lane < kLanes && row < kN / 2) copy_rows4(&map_x, b + row * 128, full, k * kDepth, token[0], token[1], token[2], token[3]);
                __syncwarp();
                ring.next(S::kStages);
            }
        }
        if (warp == kWarpProducer && ok) wait_for_stages(bars, S::kStages, ring, failed);
        if (bad) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
    } else if (warp == kWarpMma) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t kInstr = instruction(kBf16<T>, kDx, false, kTileM, kN);
            Ring ring;
            int use = 0;
            bool ok = true;
            for (int64_t t = pair; t < n_tiles && ok; t += n_pairs, ++use) {
                const uint32_t sums = tmem + (use & 1) * kN;
                if (!bar_wait(smem_u32(&bars->sums_empty[use & 1]), ((use >> 1) & 1) ^ 1, failed)) break;
                fence_after();
                for (int k = 0; k < k_steps; ++k) {
                    if (!bar_wait(smem_u32(&bars->full[ring.stage]), ring.round, failed)) { ok = false; break; }
                    fence_after();
                    const uint32_t a = smem_u32(smem + ring.stage * S::kStageBytes);
                    const uint64_t da = operand(a, kDx ? kABytes / 2 : 16), db = operand(a + kABytes, 16);
#pragma unroll
                    for (int i = 0; i < kDepth / 16; ++i)
                        mma(sums, da + (kDx ? i * 2048 : i * 32) / 16, db + i * 32 / 16, kInstr, k + i > 0);
                    commit(smem_u32(&bars->empty[ring.stage]));
                    ring.next(S::kStages);
                }
                if (ok) commit(smem_u32(&bars->sums_full[use & 1]));
            }
        }
    } else {
        // lanes of tensor memory that this warp reads, and its columns
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        constexpr int kCols = kN / (S::kStoreWarps / 4);
        // a block of 32 requests x 32 features passes through shared memory: request i's four pieces of
        // eight features lie in turned order, so that neither side meets a bank twice
        unsigned char *mine = store + (warp - 2) * 2048;
        const uint32_t put = smem_u32(mine) + lane % 8 * 64 + ((lane / 8 ^ (lane % 8 >> 1)) & 3) * 16;
        const unsigned char *get = mine + lane / 4 * 64 + ((lane ^ (lane / 4 >> 1)) & 3) * 16;
        int e = 0, use = 0;
        bool bad = false;
        for (int64_t t = pair; t < n_tiles; t += n_pairs, ++use) {
            const int rt = (int)(t / m_tiles), f0 = (int)(t % m_tiles) * kTileM + (int)rank * kHalfM + quarter * 32;
            while (tile_start[e + 1] <= rt) ++e;
            const int r0 = row_start[e] + (rt - tile_start[e]) * kN + half * kCols, r1 = min(r0 + kCols, row_end[e]);
            float add[4];                                     // of features l / 4 + 8 i, as the sums come
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int f = f0 + i * 8 + lane / 4;
                add[i] = !kDx && p.bias && f < p.features ? p.bias[(int64_t)e * p.features + f] : 0.f;
            }
            // a lane's four pieces of a block of 32 requests: eight features of request i * 8 + lane / 4 each
            const int f = f0 + lane % 4 * 8, width = min(8, p.features - f);
            uint4 keep[4];                                    // the mask's values there, asked for a block ahead
            const auto ask = [&](int c) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = r0 + c + i * 8 + lane / 4;
                    keep[i] = make_uint4(0, 0, 0, 0);
                    if (r < r1 && width == 8) {
                        const int64_t token = p.row_token ? safe_token(p.row_token[r], p.n_tokens, &bad) : r;
                        keep[i] = *reinterpret_cast<const uint4 *>((const T *)p.mask + token * p.ld_mask + f);
                    }
                }
            };
            if (kDx && p.mask) ask(0);
            if (!warp_wait(smem_u32(&bars->sums_full[use & 1]), (use >> 1) & 1, failed)) break;
            fence_after();
            const uint32_t sums = tmem + (use & 1) * kN + half * kCols + ((uint32_t)(quarter * 32) << 16);
            const int end = f0 < p.features ? min(kCols, r1 - r0) : 0;
            uint32_t lo[16], hi[16];                          // features 0-15 and 16-31 of the warp's 32
            if (end > 0) {
                tmem_load_fragments(sums, lo);
                tmem_load_fragments(sums + (16u << 16), hi);
            }
#pragma unroll 1
            for (int c = 0; c < end; c += 32) {
                tmem_wait();
#pragma unroll
                for (int j = 0; j < 4; ++j) {                 // eight requests
                    const auto out = [&](const uint32_t *r, float b) {
                        const uint32_t z = pack2<T>(__uint_as_float(r[0]) + b, __uint_as_float(r[1]) + b);
                        return !kDx && p.relu ? relu2<T>(z) : z;
                    };
                    store_transposed(put + j * 512, out(lo + 4 * j, add[0]), out(lo + 4 * j + 2, add[1]), out(hi + 4 * j, add[2]), out(hi + 4 * j + 2, add[3]));
                }
                if (c + 32 < end) {                           // the next block's sums come while this one's leave
                    tmem_load_fragments(sums + c + 32, lo);
                    tmem_load_fragments(sums + c + 32 + (16u << 16), hi);
                } else {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(in_leader(smem_u32(&bars->sums_empty[use & 1])));
                }
                __syncwarp();
                uint4 q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    q[i] = *reinterpret_cast<const uint4 *>(get + i * 512);
                    if (kDx && p.mask) {
                        T *z = reinterpret_cast<T *>(&q[i]);
                        const T *x = reinterpret_cast<const T *>(&keep[i]);
#pragma unroll
                        for (int j = 0; j < 8; ++j) if (width == 8 && !(to_float(x[j]) > 0.f)) z[j] = from_float<T>(0.f);
                    }
                }
                if (kDx && p.mask && c + 32 < end) ask(c + 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = r0 + c + i * 8 + lane / 4;
                    if (r >= r1 || width <= 0) continue;
                    T *out = (T *)p.out + r * p.ld_out + f;
                    if (width == 8) {
                        *reinterpret_cast<uint4 *>(out) = q[i];
                        continue;
                    }
                    const T *z = reinterpret_cast<const T *>(&q[i]);
                    const T *x = nullptr;
                    if (kDx && p.mask) x = (const T *)p.mask + (p.row_token ? safe_token(p.row_token[r], p.n_tokens, &bad) : r) * p.ld_mask + f;
                    for (int j = 0; j < width; ++j) out[j] = x && !(to_float(x[j]) > 0.f) ? from_float<T>(0.f) : z[j];
                }
                __syncwarp();
            }
            if (end <= 0) {                                   // nothing of this tile is the warp's
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(in_leader(smem_u32(&bars->sums_empty[use & 1])));
            }
        }
        if (bad) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
    }

    // Both CTAs are done with each other's memory before either leaves; after a failed wait the
    // copies still under way have to land first.
    __syncwarp();
    __syncthreads();
    if (*failed) {
        if (threadIdx.x == 0) atomicOr(p.status, (unsigned)GS_DEV_TIMEOUT);
        const long long start = clock64();
        while (clock64() - start < 2000000ll) { }
    }
    __syncwarp();
    cluster_sync();
    if (warp == kWarpMma) tmem_free<S::kTmem>(tmem);
}

// ---- dW and db --------------------------------------------------------------------------------
//
// dW_e: M = out features (dz's columns), N = in features (x's columns), contraction over the
// expert's rows, 64 at a time.  An expert's rows are cut into equal pieces where it holds more than
// its share of all rows, so that no pair is left with most of the work; pieces leave their sums in
// the workspace and a second launch adds them in order.  The tensor cores cut off what does not fit
// a sum (they do not round), so a long chain of additions drifts towards zero: 2e-6 of the result
// after 2,048 rows.  A chain therefore ends after kChain steps, and the storing warps add the
// chains' sums, rounding, in registers (eight warps, half a result row each) while the next chain
// runs.  (65,536 requests, first layer: off by 4.8e-7 of the result with chains of 8 steps, 7.3e-7 with
// 12; where every pair has one tile, chains of 8 / 16 / 32 steps and no chains take 635 / 597 / 575 / 562 us.)
//
// Rows past the expert's last one are those of the next expert (or anything at all): warp 2 clears
// them in shared memory before the matrix instructions may read them.  db is one more product, with a
// block of ones, for the tiles of the first in features.
//
// Cutting (pieces per pair 1 / 2 / 3 / 4, at least 32 steps each): one expert, 16,384 rows, 2368 x 2048
// 303 / 251 / 230 / 238 us; nine experts, 65,536 requests twice 693 / 688 / 638 / 641 us.  Pieces of at least 32 / 64
// steps: nine experts, 65,536 requests of 512 to 256 129 / 85 us, sixteen of 256 to 256 48 / 58 us.

constexpr int kMinPiece = 48;                   // steps of 64 rows; an expert is not cut finer
constexpr int kPiecesPerPair = 3;
constexpr int kChain = 12;                       // steps
// Warps: 0 copies, 1 issues the matrix instructions, 2 clears; the last eight store.  With gathered
// rows 3 to 7 issue the gathers, and registers move from the first eight warps to the storing ones
// (which hold 128 sums a thread): 256 * 56 + 256 * 184 of the 512 * 128 that the block starts with.
constexpr int kWeightsStoreWarps = 8, kWarpClear = 2, kWarpGather = 3, kGatherWarpsDw = 5;
constexpr int kFewRegs = 56, kManyRegs = 184;
__host__ __device__ constexpr int weights_threads(bool gather) { return gather ? 512 : 384; }

struct WeightsArgs {
    const int32_t *offsets, *row_token;
    int n_experts, n_rows, n_tokens, n_out, n_in;
    float *dw, *db;
    int64_t ld_dw;
    float *partial;
    unsigned *status;
};

// How every expert's rows are cut, in shared memory.
struct Pieces {
    int row_start[GS_MAX_EXPERTS], row_end[GS_MAX_EXPERTS], count[GS_MAX_EXPERTS];
    int slot_start[GS_MAX_EXPERTS];             // partial sums of the cut experts before it
    int at[GS_MAX_EXPERTS];                     // experts, those with the longest pieces first
    int unit_start[GS_MAX_EXPERTS + 1];         // units (tiles of pieces) of the experts before the i-th of them
};

template <int kN> struct WeightsShape {
    static constexpr uint32_t kBBytes = kN / 2 * 128;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = kN == 256 ? 6 : 8;
    static constexpr int kStoreBytes = kWeightsStoreWarps * 2048;      // per warp: 32 x 16 floats
    static constexpr int kOnesBytes = 2048;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kStoreBytes + kOnesBytes + sizeof(Barriers) + sizeof(Pieces);
    static constexpr int kTmem = 2 * kN;
    static_assert(kGatherWarpsDw <= 16 * (kN / 128), "a gathering warp without rows");
    static constexpr int kPartial = kTileM * kN + kTileM;    // floats of one piece: sums, then db
};

__device__ __forceinline__ int steps_of(const Pieces &s, int e) { return (s.row_end[e] - s.row_start[e] + kDepth - 1) / kDepth; }
__device__ __forceinline__ int piece_steps(const Pieces &s, int e) { return (steps_of(s, e) + s.count[e] - 1) / s.count[e]; }

__device__ __forceinline__ int warp_prefix(int v, int lane, int *total) {
    int sum = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kFull, sum, o);
        if (lane >= o) sum += up;
    }
    *total = __shfl_sync(kFull, sum, 31);
    return sum - v;
}

// By one warp: rows, pieces and slots of every expert.
__device__ __forceinline__ void scan_pieces(const int32_t *__restrict__ offsets, int n_experts, int n_rows, int tiles, int n_pairs,
                                            Pieces &s, int lane) {
    int64_t steps = 0;
    int end = 0;
    for (int base = 0; base < n_experts; base += 32) {
        const int2 r = ascending_rows(offsets, base + lane, n_experts, n_rows, lane, &end);
        if (base + lane < n_experts) { s.row_start[base + lane] = r.x; s.row_end[base + lane] = r.y; }
        steps += (r.y - r.x + kDepth - 1) / kDepth;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) steps += __shfl_xor_sync(kFull, steps, o);
    const int64_t share = (steps * tiles + n_pairs * kPiecesPerPair - 1) / (n_pairs * kPiecesPerPair);
    const int most = (int)(share < kMinPiece ? kMinPiece : share);
    int slots = 0;
    for (int base = 0; base < n_experts; base += 32) {
        const int e = base + lane, pieces = e < n_experts ? max((steps_of(s, e) + most - 1) / most, 1) : 0;
        int all;
        const int before = warp_prefix(pieces > 1 ? pieces * tiles : 0, lane, &all);
        if (e < n_experts) { s.count[e] = pieces; s.slot_start[e] = slots + before; }
        slots += all;
    }
}

// By the whole block: the order of the units, those with the longest pieces first.  Dealt out to the
// pairs forth and back, every pair gets nearly the same number of steps.
__device__ __forceinline__ void order_units(int n_experts, int tiles, Pieces &s) {
    for (int e = threadIdx.x; e < n_experts; e += blockDim.x) {
        const int own = piece_steps(s, e);
        int rank = 0;
        for (int o = 0; o < n_experts; ++o) {
            const int other = piece_steps(s, o);
            rank += other > own || (other == own && o < e);
        }
        s.at[rank] = e;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int units = 0;
        for (int base = 0; base < n_experts; base += 32) {
            const int i = base + (int)threadIdx.x;
            int all;
            const int before = warp_prefix(i < n_experts ? s.count[s.at[i]] * tiles : 0, threadIdx.x, &all);
            if (i < n_experts) s.unit_start[i] = units + before;
            units += all;
        }
        if (threadIdx.x == 0) s.unit_start[n_experts] = units;
    }
}

// One unit of work: a tile of one piece of an expert's rows.
struct Unit {
    int e, m0, n0, first, last, steps, slot;
};
// The pair's units in turn.
struct Units {
    const Pieces &s;
    const int pair, n_pairs, n_units, tiles, tiles_n, kn;
    int round = 0, i = 0;
    __device__ __forceinline__ bool next(Unit *w) {
        const int64_t u64 = (int64_t)round * n_pairs + ((round & 1) ? n_pairs - 1 - pair : pair);
        ++round;
        if (u64 >= n_units) return false;
        const int u = (int)u64;
        while (s.unit_start[i + 1] <= u) ++i;
        const int e = s.at[i], in_e = u - s.unit_start[i], tile = in_e % tiles, piece = in_e / tiles;
        w->e = e;
        w->m0 = tile / tiles_n * kTileM;
        w->n0 = tile % tiles_n * kn;
        const int steps = steps_of(s, e), per = piece_steps(s, e), s0 = min(piece * per, steps), s1 = min(s0 + per, steps);
        w->steps = s1 - s0;
        w->first = s.row_start[e] + s0 * kDepth;
        w->last = min(s.row_start[e] + s1 * kDepth, s.row_end[e]);
        w->slot = s.count[e] > 1 ? s.slot_start[e] + in_e : -1;
        return true;
    }
};

template <typename T, int kN, bool kGather>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(weights_threads(kGather), 1)
weights_kernel(const __grid_constant__ CUtensorMap map_dz, const __grid_constant__ CUtensorMap map_x, const WeightsArgs p)
{
    using S = WeightsShape<kN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char *ones = smem + S::kStages * S::kStageBytes, *store = ones + S::kOnesBytes;
    Barriers *bars = reinterpret_cast<Barriers *>(store + S::kStoreBytes);
    Pieces &s = *reinterpret_cast<Pieces *>(bars + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    volatile int *failed = &bars->failed;
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int tiles_n = (p.n_in + kN - 1) / kN, tiles = tiles_n * ((p.n_out + kTileM - 1) / kTileM);

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    setup_pair(bars, S::kStages, kWeightsStoreWarps, warp, lane);
    if (warp == kWarpMma) tmem_alloc<S::kTmem>(smem_u32(&bars->tmem));
    if (p.db) {
        for (int i = threadIdx.x; i < S::kOnesBytes / 2; i += blockDim.x) reinterpret_cast<T *>(ones)[i] = from_float<T>(1.f);
        fence_async_smem();
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 0) scan_pieces(p.offsets, p.n_experts, p.n_rows, tiles, n_pairs, s, lane);
    __syncthreads();
    order_units(p.n_experts, tiles, s);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();

    const uint32_t tmem = bars->tmem;
    Units units = {s, pair, n_pairs, s.unit_start[p.n_experts], tiles, tiles_n, kN};
    Unit w;
    constexpr int kFirstStore = weights_threads(kGather) / 32 - kWeightsStoreWarps;
    if constexpr (kGather) {
        if (warp < kFirstStore) fewer_registers<kFewRegs>();
    }

    if (warp == kWarpProducer || (kGather && warp >= kWarpGather && warp < kFirstStore)) {
        const int helper = warp - kWarpGather;               // of kGatherWarpsDw; negative: the copying warp
        if (threadIdx.x == 0) { prefetch_map(&map_dz); prefetch_map(&map_x); }
        // sixteen groups of four rows, kN / 128 columns of boxes, dealt out to the warps and their lanes
        const int job = lane * kGatherWarpsDw + helper, group = job % 16, box = job / 16;
        const bool gathers = kGather && helper >= 0 && job < 16 * (kN / 128);
        Ring ring;
        bool bad = false, ok = true;
        while (ok && units.next(&w)) {
            const int a0 = w.m0 + (int)rank * kHalfM, b0 = w.n0 + (int)rank * (kN / 2);
            int token[4];
            if (gathers && w.steps > 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) token[i] = p.row_token[min(w.first + group * 4 + i, w.last - 1)];
            }
            for (int k = 0; k < w.steps; ++k) {
                const int r = w.first + k * kDepth;
                const bool tail = r + kDepth > w.last;       // the clearing warp passes this step on
                if (!warp_wait(smem_u32(&bars->empty[ring.stage]), ring.round ^ 1, failed)) { ok = false; break; }
                const uint32_t a = smem_u32(smem + ring.stage * S::kStageBytes), b = a + kABytes;
                // (a step that has to be cleared lands on this CTA's own barrier; an address of the CTA itself is one of the cluster too)
                const uint32_t full = tail ? smem_u32(&bars->landed[ring.stage]) : in_leader(smem_u32(&bars->full[ring.stage]));
                if (warp == kWarpProducer && lane == 0) {
                    bar_expect(full, S::kStageBytes);
                    copy_2d(&map_dz, a, full, a0, r);
                    copy_2d(&map_dz, a + kABytes / 2, full, a0 + 64, r);
                    if (!kGather)
#pragma unroll
                        for (int i = 0; i < kN / 128; ++i) copy_2d(&map_x, b + i * 8192, full, b0 + i * 64, r);
                }
                if (gathers) {
                    int t[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[i] = safe_token(token[i], p.n_tokens, &bad);
                    copy_rows4(&map_x, b + box * 8192 + group * 512, full, b0 + box * 64, t[0], t[1], t[2], t[3]);
                    if (k + 1 < w.steps) {                    // the next step's rows
#pragma unroll
                        for (int i = 0; i < 4; ++i) token[i] = p.row_token[min(r + kDepth + group * 4 + i, w.last - 1)];
                    }
                }
                __syncwarp();
                ring.next(S::kStages);
            }
        }
        if (warp == kWarpProducer && ok) wait_for_stages(bars, S::kStages, ring, failed);
        if (bad) atomicOr(p.status, (unsigned)GS_DEV_BAD_VALUE);
    } else if (warp == kWarpMma) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t kInstr = instruction(kBf16<T>, true, true, kTileM, kN);
            constexpr uint32_t kInstrOnes = instruction(kBf16<T>, true, true, kTileM, 32);
            const uint64_t d_ones = operand(smem_u32(ones), 16);
            Ring ring;
            int use = 0;
            bool ok = true;
            while (ok && units.next(&w)) {
                const bool with_db = p.db && w.n0 == 0;
                for (int k0 = 0; k0 < w.steps && ok; k0 += kChain) {
                    const uint32_t sums = tmem + (use & 1) * kN, other = tmem + (~use & 1) * kN;
                    if (!bar_wait(smem_u32(&bars->sums_empty[use & 1]), ((use >> 1) & 1) ^ 1, failed) ||
                        (with_db && !bar_wait(smem_u32(&bars->sums_empty[~use & 1]), (((use + 1) >> 1) & 1) ^ 1, failed))) {
                        ok = false;
                        break;
                    }
                    fence_after();
                    const int k1 = min(k0 + kChain, w.steps);
                    for (int k = k0; k < k1; ++k) {
                        if (!bar_wait(smem_u32(&bars->full[ring.stage]), ring.round, failed)) { ok = false; break; }
                        fence_after();
                        const uint32_t a = smem_u32(smem + ring.stage * S::kStageBytes);
                        const uint64_t da = operand(a, kABytes / 2), db = operand(a + kABytes, 8192);
#pragma unroll
                        for (int i = 0; i < kDepth / 16; ++i) {
                            mma(sums, da + i * 2048 / 16, db + i * 2048 / 16, kInstr, k > k0 || i > 0);
                            if (with_db) mma(other, da + i * 2048 / 16, d_ones, kInstrOnes, k > k0 || i > 0);
                        }
                        commit(smem_u32(&bars->empty[ring.stage]));
                        ring.next(S::kStages);
                    }
                    if (!ok) break;
                    commit(smem_u32(&bars->sums_full[use & 1]));
                    ++use;
                    if (with_db) { commit(smem_u32(&bars->sums_full[use & 1])); ++use; }
                }
            }
        }
    } else if (warp == kWarpClear) {
        Ring ring;
        unsigned rounds = 0;                                 // bit s: parity of stage s's next landing
        bool ok = true;
        while (ok && units.next(&w)) {
            for (int k = 0; k < w.steps; ++k) {
                const int left = w.last - (w.first + k * kDepth);
                if (left < kDepth) {
                    if (!warp_wait(smem_u32(&bars->landed[ring.stage]), (rounds >> ring.stage) & 1, failed)) { ok = false; break; }
                    rounds ^= 1u << ring.stage;
                    unsigned char *box = smem + ring.stage * S::kStageBytes;
                    const int bytes = (kDepth - left) * 128;
                    for (int i = 0; i < (int)(S::kStageBytes / 8192); ++i)
                        for (int at = lane * 16; at < bytes; at += 512)
                            *reinterpret_cast<uint4 *>(box + i * 8192 + left * 128 + at) = make_uint4(0, 0, 0, 0);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) bar_arrive_release(in_leader(smem_u32(&bars->full[ring.stage])));
                }
                ring.next(S::kStages);
            }
        }
    } else if (warp >= kFirstStore) {
        if constexpr (kGather) more_registers<kManyRegs>();
        const int quarter = warp & 3, half = (warp - kFirstStore) >> 2;       // lanes of tensor memory, columns of the tile
        constexpr int kCols = kN / 2;
        float *mine = reinterpret_cast<float *>(store + (warp - kFirstStore) * 2048);
        const uint32_t sums = tmem + ((uint32_t)(quarter * 32) << 16);
        int use = 0;
        bool ok = true;
        while (ok && units.next(&w)) {
            const int row = (int)rank * kHalfM + quarter * 32, o0 = w.m0 + row;      // this warp's rows in the tile and in dW
            const bool with_db = p.db && w.n0 == 0;
            float v[kCols], bias = 0.f;
#pragma unroll
            for (int i = 0; i < kCols; ++i) v[i] = 0.f;
            for (int k = 0; k < w.steps; k += kChain) {
                if (!warp_wait(smem_u32(&bars->sums_full[use & 1]), (use >> 1) & 1, failed)) { ok = false; break; }
                fence_after();
#pragma unroll
                for (int c = 0; c < kCols; c += 16) {
                    float q[16];
                    tmem_load16(sums + (use & 1) * kN + half * kCols + c, q);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[c + i] += q[i];
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(in_leader(smem_u32(&bars->sums_empty[use & 1])));
                ++use;
                if (!with_db) continue;
                if (!warp_wait(smem_u32(&bars->sums_full[use & 1]), (use >> 1) & 1, failed)) { ok = false; break; }
                fence_after();
                bias += tmem_load1(sums + (use & 1) * kN);
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(in_leader(smem_u32(&bars->sums_empty[use & 1])));
                ++use;
            }
            if (!ok) break;
            if (w.slot >= 0) {                                // four columns of every row, then the next four
                float *part = p.partial + (int64_t)w.slot * S::kPartial;
#pragma unroll
                for (int i = 0; i < kCols / 4; ++i)
                    *reinterpret_cast<float4 *>(part + ((int64_t)(half * (kCols / 4) + i) * kTileM + row + lane) * 4) =
                        make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                if (with_db && half == 0) part[kTileM * kN + row + lane] = bias;
                continue;
            }
            if (with_db && half == 0 && o0 + lane < p.n_out) p.db[(int64_t)w.e * p.n_out + o0 + lane] = bias;
            // through shared memory, so that a warp writes 64-byte stretches of rows
#pragma unroll
            for (int c = 0; c < kCols; c += 16) {
                const int col0 = w.n0 + half * kCols + c;
                if (o0 >= p.n_out || col0 >= p.n_in) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4 *>(mine + lane * 16 + ((i ^ (lane >> 1)) & 3) * 4) =
                        make_float4(v[c + 4 * i], v[c + 4 * i + 1], v[c + 4 * i + 2], v[c + 4 * i + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = i * 8 + lane / 4, col = col0 + lane % 4 * 4;
                    const float4 q = *reinterpret_cast<const float4 *>(mine + at * 16 + ((lane ^ (at >> 1)) & 3) * 4);
                    if (o0 + at < p.n_out && col < p.n_in) {
                        float *out = p.dw + ((int64_t)w.e * p.n_out + o0 + at) * p.ld_dw + col;
                        if (col + 4 <= p.n_in) *reinterpret_cast<float4 *>(out) = q;
                        else {
                            out[0] = q.x;
                            if (col + 1 < p.n_in) out[1] = q.y;
                            if (col + 2 < p.n_in) out[2] = q.z;
                        }
                    }
                }
                __syncwarp();
            }
        }
    }

    __syncwarp();
    __syncthreads();
    if (*failed) {
        if (threadIdx.x == 0) atomicOr(p.status, (unsigned)GS_DEV_TIMEOUT);
        const long long start = clock64();
        while (clock64() - start < 2000000ll) { }
    }
    __syncwarp();
    cluster_sync();
    if (warp == kWarpMma) tmem_free<S::kTmem>(tmem);
}

// Adds up the pieces of the experts that were cut, in order.  A CTA takes 32 rows of a tile.
template <int kN>
__global__ void __launch_bounds__(256)
weights_sum_kernel(const WeightsArgs p, int n_pairs)
{
    using S = WeightsShape<kN>;
    __shared__ Pieces s;
    dependent_begin();
    const int tiles_n = (p.n_in + kN - 1) / kN, tiles = tiles_n * ((p.n_out + kTileM - 1) / kTileM);
    if (threadIdx.x < 32) scan_pieces(p.offsets, p.n_experts, p.n_rows, tiles, n_pairs, s, threadIdx.x);
    __syncthreads();
    constexpr int kParts = kTileM / 32;
    int before = 0;                                          // cut tiles of the experts before e
    int64_t job = blockIdx.x;
    for (int e = 0; e < p.n_experts; ++e) {
        if (s.count[e] < 2) continue;
        for (; job < (int64_t)(before + tiles) * kParts; job += gridDim.x) {
            const int tile = (int)(job / kParts) - before, part = (int)(job % kParts);
            const int m0 = tile / tiles_n * kTileM, n0 = tile % tiles_n * kN;
            const float *base = p.partial + ((int64_t)s.slot_start[e] + tile) * S::kPartial;
            for (int i = threadIdx.x; i < 32 * (kN / 4); i += 256) {
                const int row = part * 32 + i / (kN / 4), col4 = i % (kN / 4), o = m0 + row, col = n0 + col4 * 4;
                if (o >= p.n_out || col >= p.n_in) continue;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                for (int piece = 0; piece < s.count[e]; ++piece) {
                    const float4 q = *reinterpret_cast<const float4 *>(base + (int64_t)piece * tiles * S::kPartial + ((int64_t)col4 * kTileM + row) * 4);
                    sum.x += q.x; sum.y += q.y; sum.z += q.z; sum.w += q.w;
                }
                float *out = p.dw + ((int64_t)e * p.n_out + o) * p.ld_dw + col;
                if (col + 4 <= p.n_in) *reinterpret_cast<float4 *>(out) = sum;
                else {
                    out[0] = sum.x;
                    if (col + 1 < p.n_in) out[1] = sum.y;
                    if (col + 2 < p.n_in) out[2] = sum.z;
                }
            }
            if (p.db && n0 == 0 && threadIdx.x < 32 && m0 + part * 32 + (int)threadIdx.x < p.n_out) {
                const int row = part * 32 + threadIdx.x;
                float sum = 0.f;
                for (int piece = 0; piece < s.count[e]; ++piece) sum += base[(int64_t)piece * tiles * S::kPartial + kTileM * kN + row];
                p.db[(int64_t)e * p.n_out + m0 + row] = sum;
            }
        }
        before += tiles;
    }
}

// ---- host side --------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled g_encode = nullptr;

// Tensor map of 16-bit values whose boxes are 64 wide (128 bytes, swizzled) and `box_rows` high.
bool encode(CUtensorMap *map, int dtype, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides, int box_rows) {
    const cuuint32_t box[3] = {(cuuint32_t)kDepth, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    return g_encode(map, dtype == GS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank,
                    const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_matrix(CUtensorMap *map, int dtype, const void *base, int64_t rows, int64_t ld, int cols, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    return encode(map, dtype, base, 2, dims, strides, box_rows);
}

bool encode_weights(CUtensorMap *map, const ExpertLinearArgs &a, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)a.in, (cuuint64_t)a.out, (cuuint64_t)a.n_experts};
    const cuuint64_t strides[2] = {(cuuint64_t)a.ld_w * 2, (cuuint64_t)a.ld_w * 2 * a.out};
    return encode(map, a.dtype, a.w, 3, dims, strides, box_rows);
}

int pairs_of(const gs_ctx *ctx) { return ctx->n_sm / 2; }

// Calls f with the width of the N tile, by the average expert's rows.  A step of 64 takes some 0.35 us
// whatever the width (the weights' 128 rows per CTA bound it), so a tile that covers most experts whole
// is best, and a wider one only adds copies.  2048 to 1024, nine experts, widths 32 / 64 / 128 / 256:
// 57 rows each 26 / 16 / 17 / 20 us, 133 rows 38 / 27 / 18 / 25 us, 266 rows 60 / 39 / 29 / 21 us;
// 512 to 512, 64 experts: 15 rows 11.5 / 11.8 / 12.3 / 13.7 us, 62 rows 20 / 15 / 14 / 16 us, 156 rows 36 / 24 / 20 / 20 us.
template <typename F> cudaError_t by_rows(const ExpertLinearArgs &a, F &&f) {
    const int64_t each = a.n_rows / a.n_experts;
    if (each >= 140) return f(std::integral_constant<int, 256>());
    if (each >= 60) return f(std::integral_constant<int, 128>());
    if (each >= 24) return f(std::integral_constant<int, 64>());
    return f(std::integral_constant<int, 32>());
}

template <typename T, bool kDx, int kN, bool kGather>
cudaError_t launch_rows(gs_ctx *ctx, const CUtensorMap &map_w, const CUtensorMap &map_x, const RowsArgs &p, cudaStream_t st) {
    const int64_t tiles = (p.n_rows / kN + p.n_experts) * (int64_t)((p.features + kTileM - 1) / kTileM);
    const int pairs = (int)(tiles < pairs_of(ctx) ? tiles : pairs_of(ctx));
    LaunchTimer t(ctx, GS_K_EXPERT_LINEAR, st);
    return launch_dependent(rows_kernel<T, kDx, kN, kGather>, dim3(2 * pairs), dim3(RowsShape<kN>::threads(kGather)), RowsShape<kN>::kSmem, st, map_w, map_x, p);
}

template <typename T> cudaError_t forward_as(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    RowsArgs p = {a.offsets, a.row_token, a.n_experts, (int)a.n_rows, (int)a.n_x_rows, a.out, a.in, a.bias,
                  (a.flags & GS_EXPERT_RELU) != 0, nullptr, 0, a.y, a.ld_y, ctx->s.status};
    return by_rows(a, [&](auto width) {
        constexpr int N = decltype(width)::value;
        CUtensorMap map_w, map_x;
        if (!encode_weights(&map_w, a, kHalfM) ||
            !encode_matrix(&map_x, a.dtype, a.x, a.n_x_rows, a.ld_x, a.in, a.row_token ? 1 : N / 2)) return cudaErrorInvalidValue;
        return a.row_token ? launch_rows<T, false, N, true>(ctx, map_w, map_x, p, st) : launch_rows<T, false, N, false>(ctx, map_w, map_x, p, st);
    });
}

template <typename T> cudaError_t dx_as(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    const bool masked = (a.flags & GS_EXPERT_RELU_INPUT) != 0;
    RowsArgs p = {a.offsets, a.row_token, a.n_experts, (int)a.n_rows, (int)a.n_x_rows, a.in, a.out, nullptr, false,
                  masked ? a.x : nullptr, a.ld_x, a.dx, a.ld_dx, ctx->s.status};
    return by_rows(a, [&](auto width) {
        constexpr int N = decltype(width)::value;
        CUtensorMap map_w, map_dz;
        if (!encode_weights(&map_w, a, kDepth) || !encode_matrix(&map_dz, a.dtype, a.dz, a.n_rows, a.ld_dz, a.out, N / 2)) return cudaErrorInvalidValue;
        return launch_rows<T, true, N, false>(ctx, map_w, map_dz, p, st);
    });
}

int weights_tile(int in) { return in > 128 ? 256 : 128; }

template <typename T, int kN> cudaError_t dw_as(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    if (a.n_rows == 0) {
        cudaError_t e = cudaMemset2DAsync(a.dw, (size_t)a.ld_dw * 4, 0, (size_t)a.in * 4, (size_t)a.n_experts * a.out, st);
        if (e == cudaSuccess && a.db) e = cudaMemsetAsync(a.db, 0, (size_t)a.n_experts * a.out * 4, st);
        return e;
    }
    const WeightsArgs p = {a.offsets, a.row_token, a.n_experts, (int)a.n_rows, (int)a.n_x_rows, a.out, a.in, a.dw, a.db, a.ld_dw,
                           (float *)a.workspace, ctx->s.status};
    CUtensorMap map_dz, map_x;
    if (!encode_matrix(&map_dz, a.dtype, a.dz, a.n_rows, a.ld_dz, a.out, kDepth) ||
        !encode_matrix(&map_x, a.dtype, a.x, a.n_x_rows, a.ld_x, a.in, a.row_token ? 1 : kDepth)) return cudaErrorInvalidValue;
    const int pairs = pairs_of(ctx);
    cudaError_t e;
    {
        LaunchTimer t(ctx, GS_K_EXPERT_LINEAR, st);
        e = a.row_token ? launch_dependent(weights_kernel<T, kN, true>, dim3(2 * pairs), dim3(weights_threads(true)), WeightsShape<kN>::kSmem, st, map_dz, map_x, p)
                        : launch_dependent(weights_kernel<T, kN, false>, dim3(2 * pairs), dim3(weights_threads(false)), WeightsShape<kN>::kSmem, st, map_dz, map_x, p);
    }
    if (e != cudaSuccess || expert_linear_workspace(ctx, a.n_experts, a.n_rows, a.in, a.out) == 0) return e;
    // (not as a programmatic dependent: its CTAs would gather on the SMs whose pairs end first and stay
    // there; 16,384 requests of 1024 to 512: 113 instead of 69 us for both launches)
    LaunchTimer t(ctx, GS_K_EXPERT_LINEAR, st);
    return launch_after(weights_sum_kernel<kN>, dim3(4 * ctx->n_sm), dim3(256), 0, st, p, pairs);
}

template <typename T> cudaError_t dw_by_tile(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return weights_tile(a.in) == 256 ? dw_as<T, 256>(ctx, a, st) : dw_as<T, 128>(ctx, a, st);
}

template <typename T, int kN> cudaError_t configure_rows() {
    cudaError_t e = cudaFuncSetAttribute(rows_kernel<T, false, kN, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RowsShape<kN>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(rows_kernel<T, false, kN, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RowsShape<kN>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(rows_kernel<T, true, kN, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)RowsShape<kN>::kSmem);
    return e;
}

// The storing warps of the gathering kernel wait for registers that the others give back: there have to be enough.
template <typename T, int kN> cudaError_t configure_weights() {
    cudaFuncAttributes f;
    cudaError_t e = cudaFuncGetAttributes(&f, weights_kernel<T, kN, true>);
    if (e == cudaSuccess && f.numRegs * weights_threads(true) < 256 * (kFewRegs + kManyRegs)) e = cudaErrorInvalidConfiguration;
    if (e == cudaSuccess) e = cudaFuncSetAttribute(weights_kernel<T, kN, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)WeightsShape<kN>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(weights_kernel<T, kN, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)WeightsShape<kN>::kSmem);
    return e;
}

template <typename T> cudaError_t configure_as() {
    for (auto f : {configure_rows<T, 32>, configure_rows<T, 64>, configure_rows<T, 128>, configure_rows<T, 256>, configure_weights<T, 128>, configure_weights<T, 256>}) {
        const cudaError_t e = f();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t configure_expert_linear() {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
    g_encode = reinterpret_cast<EncodeTiled>(f);
    e = configure_as<__nv_bfloat16>();
    return e == cudaSuccess ? configure_as<__half>() : e;
}

// An expert is cut only if it has more steps than kMinPiece and than a share (the whole work over
// kPiecesPerPair pieces per pair); it then has at most 2 * steps / most pieces of either, and all cut
// experts together at most twice the number of shares, and twice all steps over kMinPiece (no two
// experts share a row, whatever the offsets say).
int64_t expert_linear_workspace(const gs_ctx *ctx, int n_experts, int64_t n_rows, int in, int out) {
    if (n_rows <= kMinPiece * kDepth) return 0;
    const int kn = weights_tile(in);
    const int64_t tiles = (int64_t)((in + kn - 1) / kn) * ((out + kTileM - 1) / kTileM);
    const int64_t by_share = 2 * (int64_t)pairs_of(ctx) * kPiecesPerPair, by_steps = 2 * tiles * (n_rows / kDepth + n_experts) / kMinPiece + 1;
    return (by_share < by_steps ? by_share : by_steps) * (kTileM * kn + kTileM) * 4;
}

cudaError_t launch_expert_linear(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? forward_as<__nv_bfloat16>(ctx, a, st) : forward_as<__half>(ctx, a, st);
}
cudaError_t launch_expert_linear_dx(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? dx_as<__nv_bfloat16>(ctx, a, st) : dx_as<__half>(ctx, a, st);
}
cudaError_t launch_expert_linear_dw(gs_ctx *ctx, const ExpertLinearArgs &a, cudaStream_t st) {
    return a.dtype == GS_BF16 ? dw_by_tile<__nv_bfloat16>(ctx, a, st) : dw_by_tile<__half>(ctx, a, st);
}

}  // namespace gs
