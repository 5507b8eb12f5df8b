// The products of the gated feed-forward block on the tensor cores, one kernel template.
//
//   kForward   [g | u] = x [w_gate | w_up]^T      rows m, columns n (gate and up side by side), contraction k
//   kBackward  both gradients in one launch, tiles of either kind in one list (a launch of its own for each would cost
//              seven microseconds more, which is most of a small step):
//              kInput   dx = dg w_gate + du w_up           rows m, columns k, contraction over both halves of n
//              kWeight  dw_gate | dw_up = (dg | du)^T x    rows n (gate tiles, then up tiles), columns k, contraction m
//
// A pair of CTAs (one cluster) computes a 256 x BN tile with tcgen05.mma.cta_group::2, K = 16 an instruction: a pair
// reads half as much of B from shared memory per flop as two single CTAs would.  Operands arrive by TMA in blocks of 64
// along the contraction, 128-byte swizzle, a ring of stages; the layouts of x, weights and dgu in memory are taken as
// they are: where the contraction index is not the contiguous one (the weights in kInput, both operands in kWeight) the
// MMA reads the block across rows.  For the forward product CTA 0 brings gate columns and CTA 1 up columns of the same
// BN/2 hidden units, so g and u of a unit meet in one thread of the epilogue and h = act(g)*u leaves without another pass.
// Accumulators: two sets of BN tensor-memory columns in turn, so a tile's epilogue runs under the next tile's MMAs.
// (Tiles of 512 columns over both sets, one ahead of the other, were tried: 842 us against 725 at 8192 x 4096 x 8192 forward.)
// Eight epilogue warps: two to each quarter of the lanes, steps of columns in turn.
//
// Persistent: at most one cluster per pair of SMs; tiles in groups of sixteen row tiles, columns inside a group in turn, so
// that the operands of the tiles in flight stay in the L2 (8192 x 4096 x 8192 forward: 934 us with groups of four, 900
// with eight, 880 with sixteen, sustained, before the issue loop counted its stages; 800 since).  8192 x 4096 x 10922
// forward: 1127 us, 1300 TFLOP/s at the power limit.  Tiles of the backward products may be cut along the contraction when there
// are fewer of them than clusters; each share then leaves binary32 sums in the workspace and a last kernel adds the shares
// in order.
//
// Every wait is bounded (about a second; the epilogue's wait for a tile by two microseconds more for each block of its
// contraction): a thread whose wait runs out sets its CTA's
// `dead` word, all roles leave their loops, and both CTAs wait (bounded again) for the MMAs and the loads in flight, which
// use either one's shared memory, before tensor memory is freed (drain()).
#pragma once

#include "umma_pair.cuh"
#include "worker_common.cuh"

namespace bz {

static __device__ unsigned int g_glu_timeouts = 0;

enum GluProduct { kForward, kBackward };
enum GluKind { kInput, kWeight };

constexpr int kRowTile = 256, kBlockK = 64, kEpilogueWarps = 8, kProductThreads = 128 + 32 * kEpilogueWarps;
constexpr uint32_t kWaitProbes = 1u << 19, kStallBlocks = 2;   // probes of two microseconds at most

// One result: h, or dx, or both weights' gradients.
struct ProductPart {
    int64_t rows, cols;          // extents (kWeight: rows of one half; kForward: hidden units)
    int64_t row_tiles, col_tiles;
    int64_t blocks;              // of kBlockK along the contraction
    int64_t half_blocks;         // kInput: of one half of it
    int splits;                  // shares of the contraction
    void* out;                   // h / dx / dw_gate
    void* out2;                  // dw_up
    int64_t ld_out;
    int out_f32, wide, pairs;    // binary32 output; 16-byte stores possible; stores of two elements possible
    float* partial;              // splits > 1: [split][tile][256][BN]
    __host__ __device__ int64_t tiles() const { return row_tiles * col_tiles * splits; }
};
struct ProductParams {
    ProductPart part[2];         // kForward: the first; kBackward: by GluKind
    int weight_first;            // the order of the two in the list of tiles: longer contractions first
    int act;
    int stall;                   // 1 + the rank whose loads stop after kStallBlocks, for tests of expired waits; 0: none
    float* preact;               // kForward: [2][rows][cols] or null
    int preact_wide, preact_pairs;
};
// kForward: x, w_gate, w_up.  kBackward: dgu by rows, w_gate, w_up, dgu across rows, x.
struct ProductMaps {
    CUtensorMap map[5];
};

// ---- stores -------------------------------------------------------------------------------------
// The accumulator gives a thread one row; memory wants a warp on one row.  A warp turns 32 rows x 32 words (128 bytes of
// each row) through shared memory, the 16-byte groups of row r exchanged by r mod 8, so that both the writes (eight rows)
// and the reads (one row) of a quarter warp meet every bank once.

constexpr int kTurnBytes = 32 * 128;

__device__ __forceinline__ int turned(int row, int word) { return row * 32 + (word ^ ((row & 7) << 2)); }
__device__ __forceinline__ void turn_in(float* turn, int word, const uint4& w) {
    *reinterpret_cast<uint4*>(turn + turned(threadIdx.x & 31, word)) = w;
}
// Writes elements [c0, c0 + 128 / sizeof(E)) of rows r0 .. r0 + 31 of `out`; `rows`, `cols` exist.  wide: 16-byte stores
// possible; pairs: stores of two elements possible.
template <typename E>
__device__ __forceinline__ void turn_out(const float* turn, E* out, int64_t ld, int64_t r0, int64_t rows, int64_t c0, int64_t cols, bool wide, bool pairs) {
    constexpr int kEach = 128 / static_cast<int>(sizeof(E)), kPer = 4 / static_cast<int>(sizeof(E));
    const int lane = threadIdx.x & 31;
    const int n_rows = static_cast<int>(min(int64_t(32), rows - r0)), n = static_cast<int>(min(int64_t(kEach), cols - c0));
    if (n_rows <= 0 || n <= 0) return;
    E* base = out + r0 * ld + c0;
    if (wide && n % (16 / static_cast<int>(sizeof(E))) == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + lane / 8, w = lane % 8 * 4;
            if (r < n_rows && w * kPer < n) *reinterpret_cast<uint4*>(base + r * ld + w * kPer) = *reinterpret_cast<const uint4*>(turn + turned(r, w));
        }
    } else if (kPer == 1 && pairs && n % 2 == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = i * 2 + lane / 16, w = lane % 16 * 2;
            if (r < n_rows && w < n) *reinterpret_cast<float2*>(base + r * ld + w) = *reinterpret_cast<const float2*>(turn + turned(r, w));
        }
    } else if (kPer == 1 || (pairs && n % 2 == 0)) {
        if (lane * kPer < n) {
#pragma unroll 8
            for (int r = 0; r < 32; ++r)
                if (r < n_rows) *reinterpret_cast<float*>(base + r * ld + lane * kPer) = turn[turned(r, lane)];
        }
    } else {
#pragma unroll 8
        for (int r = 0; r < 32; ++r) {
            if (r >= n_rows) break;
            const E* from = reinterpret_cast<const E*>(turn);
            if (lane < n) base[r * ld + lane] = from[turned(r, lane / kPer) * kPer + lane % kPer];
            if (lane + 32 < n) base[r * ld + lane + 32] = from[turned(r, (lane + 32) / kPer) * kPer + lane % kPer];
        }
    }
}

template <int BN> struct ProductShape {
    static constexpr int kABytes = 128 * kBlockK * 2, kBBytes = BN / 2 * kBlockK * 2, kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = BN == 256 ? 5 : (BN == 128 ? 7 : 9);
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kEpilogueWarps * kTurnBytes + (2 * kStages + 5) * 8 + 16;
};

// ---- activations --------------------------------------------------------------------------------

__device__ __forceinline__ float logistic(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
template <int ACT> __device__ __forceinline__ float act(float g) {
    if constexpr (ACT == BZ_ACT_SILU) return g * logistic(g);
    // (1 + tanh y)/2 = 1/(1 + exp(-2y))
    if constexpr (ACT == BZ_ACT_GELU_TANH) return g * logistic(1.5957691216f * (g + 0.044715f * g * g * g));
    // 1 + erf y = erfc(-y): the sum would lose every digit from g = -5.6 down, where bfloat16 still holds the product
    if constexpr (ACT == BZ_ACT_GELU) return 0.5f * g * erfcf(g * -0.70710678f);
    return g > 0.f ? g : (g == g ? 0.f : g);
}
template <int ACT> __device__ __forceinline__ float act_slope(float g) {
    if constexpr (ACT == BZ_ACT_SILU) {
        const float s = logistic(g);
        return s * (1.f + g * (1.f - s));
    }
    if constexpr (ACT == BZ_ACT_GELU_TANH) {
        const float s = logistic(1.5957691216f * (g + 0.044715f * g * g * g));
        return s + g * s * (1.f - s) * 1.5957691216f * (1.f + 0.134145f * g * g);
    }
    if constexpr (ACT == BZ_ACT_GELU) return 0.5f * erfcf(g * -0.70710678f) + g * 0.39894228f * __expf(-0.5f * g * g);
    return g > 0.f ? 1.f : 0.f;
}
template <int ACT> __device__ __forceinline__ void gate(float (&g)[8], const float (&u)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = act<ACT>(g[i]) * u[i];
}

struct ProductTile {
    int kind;          // GluKind
    int64_t index;     // in its part
    int64_t row, col;  // in tiles
    int64_t from, to;  // contraction blocks
};
__device__ __forceinline__ void place_tile(const ProductPart& p, int64_t i, ProductTile& t) {
    constexpr int64_t G = 16;
    const int64_t per = p.row_tiles * p.col_tiles, split = i / per;
    t.index = i;
    i -= split * per;
    const int64_t g = i / (G * p.col_tiles), first = g * G, n = min(G, p.row_tiles - first);
    i -= g * G * p.col_tiles;
    t.row = first + i % n;
    t.col = i / n;
    t.from = p.blocks * split / p.splits;
    t.to = p.blocks * (split + 1) / p.splits;
}
template <GluProduct P> __device__ __forceinline__ ProductTile tile_at(const ProductParams& p, int64_t i) {
    ProductTile t;
    t.kind = kInput;
    if (P == kBackward) {
        t.kind = p.weight_first ? kWeight : kInput;
        const int64_t n = p.part[t.kind].tiles();
        if (i >= n) i -= n, t.kind ^= 1;
    }
    place_tile(p.part[t.kind], i, t);
    return t;
}

// Up to an eighth of a second.
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity) {
    volatile int expired = 0;   // mbar_wait_live() tells through it; nobody else does
    mbar_wait_live(bar, parity, &expired, 2000, 1u << 16);
}
// After an expired wait, by both CTAs: waits for all MMAs and loads issued.  The loads of a block report to the leader's
// barrier, which expects both CTAs' bytes from when the leader issued its own; a CTA that stopped earlier than the other leaves
// some of the last blocks half announced or half loaded, which the leader makes up for.  `blocks`: room for both CTAs'
// counts; `drained`: a barrier of one arrival, not used before.
template <typename S>
__device__ __forceinline__ void drain(uint32_t rank, uint32_t issued, volatile uint32_t* blocks, uint64_t* full, uint64_t* drained) {
    if (threadIdx.x == 0) store_cluster(const_cast<uint32_t*>(blocks + rank), 0, issued);
    __syncwarp();
    cluster_sync();
    if (threadIdx.x == 32) {   // the thread that issued the MMAs
        if (rank == 0) mma_commit_pair(drained);
        drain_wait(drained, 0);
    }
    if (threadIdx.x == 0 && rank == 0) {
        const uint32_t own = blocks[0], other = blocks[1], most = max(own, other);
        for (uint32_t j = most > S::kStages ? most - S::kStages : 0; j < most; ++j) {
            uint64_t* bar = &full[j % S::kStages];
            if (j >= own) mbar_expect_tx(bar, S::kStageBytes);
            if (j >= other) mbar_complete_tx(bar, S::kStageBytes);
            drain_wait(bar, j / S::kStages & 1);
        }
    }
    __syncwarp();
    cluster_sync();
}

template <typename T, GluProduct P, int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
    glu_product_kernel(const __grid_constant__ ProductMaps maps, const __grid_constant__ ProductParams p) {
    using S = ProductShape<BN>;
    constexpr int kBf16 = !__is_same(T, __half);
    constexpr int kBlockBytes = 64 * kBlockK * 2;   // 64 rows of 128 bytes
    extern __shared__ unsigned char raw[];
    unsigned char* smem = raw + (1024 - smem_u32(raw) % 1024) % 1024;
    float* turns = reinterpret_cast<float*>(smem + S::kStages * S::kStageBytes);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStageBytes + kEpilogueWarps * kTurnBytes);
    uint64_t* empty = full + S::kStages;
    uint64_t* acc_full = empty + S::kStages;   // [2]
    uint64_t* acc_empty = acc_full + 2;        // [2], the leader's are used
    uint64_t* drained = acc_empty + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
    volatile int* dead = reinterpret_cast<volatile int*>(tmem_slot + 1);
    uint32_t* blocks_issued = tmem_slot + 2;   // [2]

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int64_t cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1;
    const int64_t tiles = p.part[0].tiles() + (P == kBackward ? p.part[1].tiles() : 0);
    if (warp == 3 && lane < (P == kForward ? 3 : 5)) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.map[lane]) : "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 1);
        for (int s = 0; s < 2; ++s) mbar_init(&acc_full[s], 1), mbar_init(&acc_empty[s], 2 * kEpilogueWarps);
        mbar_init(drained, 1);
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_alloc_pair(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    RingAt<S::kStages> at;          // of the loads (thread 0), of the MMAs (the issuing thread)
    uint32_t issued = 0;            // blocks loaded (thread 0)

    if (warp == 0 && lane == 0) {
        // ---------------------------------------------------------------- loads
        bool alive = true;
        const uint32_t smem_addr = smem_u32(smem), leader_full = leader_addr(full);
        for (int64_t i = cluster; i < tiles && alive; i += clusters) {
            const ProductTile t = tile_at<P>(p, i);
            const int row = static_cast<int>(t.row * 256 + rank * 128), half_blocks = static_cast<int>(p.part[kInput].half_blocks);
            const int column0 = static_cast<int>(P == kForward ? t.col * (BN / 2) : t.col * BN + rank * (BN / 2));
            const int64_t half_tiles = p.part[kWeight].row_tiles / 2;
            const int weight_half = t.row >= half_tiles, weight_x = static_cast<int>((t.row - weight_half * half_tiles) * 256 + rank * 128);
            for (int kb = static_cast<int>(t.from); kb < static_cast<int>(t.to); ++kb, at.next()) {
                const int s = at.stage;
                if (issued >= S::kStages) {
                    if (!mbar_wait_live(&empty[s], at.parity ^ 1, dead)) {
                        alive = false;
                        break;
                    }
                } else if (issued == kStallBlocks && p.stall == static_cast<int>(rank) + 1) {
                    alive = false;
                    break;
                }
                ++issued;
                const uint32_t bar = leader_full + s * 8;
                if (rank == 0) mbar_expect_tx(&full[s], 2 * S::kStageBytes);
                const uint32_t a = smem_addr + s * S::kStageBytes, b = a + S::kABytes;
                if constexpr (P == kForward) {
                    const int x = kb * kBlockK;
                    tma_load_pair(a, &maps.map[0], bar, x, row);
                    tma_load_pair(b, &maps.map[1 + rank], bar, x, column0);
                } else {
                    // this CTA's half of the columns, in blocks of 64
                    auto column = [&](int c) { return column0 + c * 64; };
                    if (t.kind == kInput) {
                        const int half = kb >= half_blocks, x = (kb - half * half_blocks) * kBlockK;
                        tma_load_pair(a, &maps.map[0], bar, x, row, half);
#pragma unroll
                        for (int c = 0; c < BN / 128; ++c) tma_load_pair(b + c * kBlockBytes, &maps.map[1 + half], bar, column(c), x);
                    } else {
                        const int y = kb * kBlockK;
                        tma_load_pair(a, &maps.map[3], bar, weight_x, y, weight_half);
                        tma_load_pair(a + kBlockBytes, &maps.map[3], bar, weight_x + 64, y, weight_half);
#pragma unroll
                        for (int c = 0; c < BN / 128; ++c) tma_load_pair(b + c * kBlockBytes, &maps.map[4], bar, column(c), y);
                    }
                }
            }
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---------------------------------------------------------------- MMA issue
        int64_t n = 0;
        bool alive = true;
        for (int64_t i = cluster; i < tiles && alive; i += clusters, ++n) {
            const ProductTile t = tile_at<P>(p, i);
            const bool across_a = P == kBackward && t.kind == kWeight;
            constexpr bool kAcrossB = P == kBackward;
            const uint32_t idesc = across_a ? idesc_16bit(256, BN, kBf16, 1, kAcrossB) : idesc_16bit(256, BN, kBf16, 0, kAcrossB);
            // descriptors of stage 0; a stage and a step of 16 along the contraction add to their address fields
            constexpr uint32_t kStepA = 32 >> 4, kAcrossStep = 2048 >> 4, kStageStep = S::kStageBytes >> 4;
            const uint64_t a0 = across_a ? smem_desc_mn128(smem_u32(smem), kBlockBytes) : smem_desc_k128(smem_u32(smem));
            const uint64_t b0 = kAcrossB ? smem_desc_mn128(smem_u32(smem) + S::kABytes, kBlockBytes) : smem_desc_k128(smem_u32(smem) + S::kABytes);
            const uint32_t step_a = across_a ? kAcrossStep : kStepA;
            auto multiply = [&](int stage, uint32_t acc, bool first) {
                const uint64_t da = a0 + stage * kStageStep, db = b0 + stage * kStageStep;
#pragma unroll
                for (int k = 0; k < kBlockK / 16; ++k)
                    mma_16bit_pair(tmem + acc * 256, da + k * step_a, db + k * (kAcrossB ? kAcrossStep : kStepA), idesc, !first || k > 0);
            };
            const int acc = static_cast<int>(n & 1);
            if (n >= 2 && !mbar_wait_live(&acc_empty[acc], static_cast<uint32_t>((n >> 1) - 1) & 1, dead)) break;
            tc_fence_after_sync();
            const int blocks = static_cast<int>(t.to - t.from);
            for (int kb = 0; kb < blocks; ++kb, at.next()) {
                if (!mbar_wait_live(&full[at.stage], at.parity, dead)) {
                    alive = false;
                    break;
                }
                tc_fence_after_sync();
                multiply(at.stage, acc, kb == 0);
                mma_commit_pair(&empty[at.stage]);
            }
            if (alive) mma_commit_pair(&acc_full[acc]);
        }
    } else if (warp >= 4) {
        // ---------------------------------------------------------------- epilogue: one row and half of the columns a thread
        const int quarter = warp & 3, half_of_columns = (warp - 4) >> 2;
        float* turn = turns + (warp - 4) * (kTurnBytes / 4);
        int64_t n = 0;
        for (int64_t i = cluster; i < tiles; i += clusters, ++n) {
            const ProductTile t = tile_at<P>(p, i);
            const ProductPart& o = p.part[t.kind];
            const int acc = static_cast<int>(n & 1);
            if (!__all_sync(~0u, mbar_wait_live(&acc_full[acc], static_cast<uint32_t>(n >> 1) & 1, dead, 2000, kWaitProbes + static_cast<uint32_t>(t.to - t.from)))) break;  // a warp leaves as one
            tc_fence_after_sync();
            const uint32_t base = tmem + acc * 256 + (static_cast<uint32_t>(quarter * 32) << 16);
            const int in_tile = static_cast<int>(rank) * 128 + quarter * 32;   // first row of this warp
            if constexpr (P == kForward) {
                const int64_t r0 = t.row * 256 + in_tile;
                constexpr int kStep = BN / 2 < 128 ? 32 : 64;   // a warp takes every other step
                // Loops of a few columns: with the four activations unrolled over whole steps the code alone took microseconds
                // to arrive (1024 x 512 x 2048: 15.3 us).
#pragma unroll 1
                for (int c = half_of_columns * kStep; c < BN / 2; c += 2 * kStep) {
                    const int64_t c0 = t.col * (BN / 2) + c;
                    if (p.preact != nullptr) {
#pragma unroll 1
                        for (int e = 0; e < 2 * (kStep / 32); ++e) {   // gate, then up, of each 32 columns
                            float x[32];
                            const int up = e & 1, more = e / 2 * 32;
                            tmem_ld32(base + up * (BN / 2) + c + more, x);
                            tmem_ld32_wait(x);
#pragma unroll
                            for (int k = 0; k < 8; ++k) turn_in(turn, 4 * k, Word<float>::pack(x + 4 * k));
                            __syncwarp();
                            turn_out<float>(turn, p.preact + up * o.rows * o.cols, o.cols, r0, o.rows, c0 + more, o.cols, p.preact_wide, p.preact_pairs);
                            __syncwarp();
                        }
                    }
#pragma unroll 1
                    for (int e = 0; e < kStep / 8; ++e) {
                        float g[8], u[8];
                        tmem_ld8(base + c + e * 8, g);
                        tmem_ld8(base + BN / 2 + c + e * 8, u);
                        tmem_ld8_wait(g);
                        tmem_ld8_wait(u);
                        switch (p.act) {
                            case BZ_ACT_SILU: gate<BZ_ACT_SILU>(g, u); break;
                            case BZ_ACT_GELU_TANH: gate<BZ_ACT_GELU_TANH>(g, u); break;
                            case BZ_ACT_GELU: gate<BZ_ACT_GELU>(g, u); break;
                            default: gate<BZ_ACT_RELU>(g, u); break;
                        }
                        turn_in(turn, 4 * e, Word<T>::pack(g));
                    }
                    __syncwarp();
                    turn_out<T>(turn, static_cast<T*>(o.out), o.ld_out, r0, o.rows, c0, min(o.cols, c0 + kStep), o.wide, o.pairs);
                    __syncwarp();
                }
            } else {
                const int64_t half_tiles = t.kind == kWeight ? o.row_tiles / 2 : 0;
                const int half = t.kind == kWeight && t.row >= half_tiles;
                const int64_t r0 = (t.row - half * half_tiles) * 256 + in_tile;
                void* out = half ? o.out2 : o.out;
                const bool f32 = o.out_f32 || o.splits > 1;
#pragma unroll 1
                for (int c = half_of_columns * 64; c < BN; c += 128) {
                    float x[2][32];
                    tmem_ld32(base + c, x[0]);
                    tmem_ld32(base + c + 32, x[1]);
                    tmem_ld32_wait(x[0]);
                    tmem_ld32_wait(x[1]);
                    if (f32) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) turn_in(turn, 4 * e, Word<float>::pack(x[k] + 4 * e));
                            __syncwarp();
                            if (o.splits > 1)
                                turn_out<float>(turn, o.partial + t.index * 256 * BN, BN, in_tile, 256, c + k * 32, BN, true, false);
                            else
                                turn_out<float>(turn, static_cast<float*>(out), o.ld_out, r0, o.rows, t.col * BN + c + k * 32, o.cols, o.wide, o.pairs);
                            __syncwarp();
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) turn_in(turn, 4 * e, Word<T>::pack(x[e / 4] + e % 4 * 8));
                        __syncwarp();
                        turn_out<T>(turn, static_cast<T*>(out), o.ld_out, r0, o.rows, t.col * BN + c, o.cols, o.wide, o.pairs);
                        __syncwarp();
                    }
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) arrive_cluster(leader_addr(&acc_empty[acc]));
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && *dead) {
        atomicAdd(&g_glu_timeouts, 1u);
        store_cluster(const_cast<int*>(dead), rank ^ 1, 1);
    }
    __syncwarp();
    tc_fence_before_sync();
    cluster_sync();
    tc_fence_after_sync();
    if (*dead) drain<S>(rank, issued, blocks_issued, full, drained);   // both CTAs or neither: each one's is the other's too
    if (warp == 2) tmem_dealloc_pair(tmem, 512);
}

// The shares' sums of a part, in order: one thread a group of four columns.
template <typename T, int BN> __device__ __forceinline__ void add_shares(const ProductPart& p, bool weight) {
    if (p.splits < 2) return;
    const int64_t per = p.row_tiles * p.col_tiles, groups = per * 256 * (BN / 4);
    const int64_t half_tiles = weight ? p.row_tiles / 2 : 0;
    for (int64_t e = blockIdx.x * int64_t(256) + threadIdx.x; e < groups; e += gridDim.x * int64_t(256)) {
        const int64_t i = e / (256 * (BN / 4));
        const int in = static_cast<int>(e % (256 * (BN / 4))), in_row = in / (BN / 4), c = in % (BN / 4) * 4;
        ProductTile t;
        place_tile(p, i, t);
        const int half = weight && t.row >= half_tiles;
        const int64_t r = (t.row - half * half_tiles) * 256 + in_row, c0 = t.col * BN + c;
        if (r >= p.rows || c0 >= p.cols) continue;
        float4 s = *reinterpret_cast<const float4*>(p.partial + (i * 256 + in_row) * BN + c);
        for (int k = 1; k < p.splits; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(p.partial + ((k * per + i) * 256 + in_row) * BN + c);
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        const float x[4] = {s.x, s.y, s.z, s.w};
        void* out = half ? p.out2 : p.out;
        for (int k = 0; k < 4; ++k)
            if (c0 + k < p.cols) {
                if (p.out_f32)
                    static_cast<float*>(out)[r * p.ld_out + c0 + k] = x[k];
                else
                    static_cast<T*>(out)[r * p.ld_out + c0 + k] = from_f32<T>(x[k]);
            }
    }
}
template <typename T, int BN> __global__ void __launch_bounds__(256) glu_shares_kernel(const __grid_constant__ ProductParams p) {
    add_shares<T, BN>(p.part[kInput], false);
    add_shares<T, BN>(p.part[kWeight], true);
}

}  // namespace bz
