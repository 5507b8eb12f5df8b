// Gated feed-forward block for few rows (tokens): bound by reading both weights once.
//
// A CTA takes eight hidden units; its eight warps take 32-wide steps of k in turn, so the units' weights stream through
// registers by 16-byte loads that a quad of lanes makes contiguous (64 bytes of each of 8 rows at a time, four steps in
// flight).  The products run on mma.sync (m16n8k16: the eight gate rows above the eight up rows, times 8 tokens), so one
// thread ends with g and u of its unit: at one to 32 tokens the arithmetic is far below either tensor path's rate, and this
// one takes its operands from the registers the loads end in.  The order of k inside an MMA is free as long as weights and
// tokens agree, so lane t of a quad feeds its own eight consecutive elements as the pairs (2t, 2t+1), (2t+8, 2t+9) of two
// MMAs, and no element moves between lanes.
// The eight warps' sums meet in shared memory and are added in order.
#pragma once

#include "glu_product.cuh"

namespace bz {

// Up to kFewMost rows (against the 256-row tiles, out of memory: 16 rows of 1024 x 4096 9.4 against 14.3 us, 32 rows 13.2 against
// 14.6, 32 rows of 512 x 1365 6.1 against 10.2; 32 rows of 4096 x 10920 70 against 63, the one side that loses).
constexpr int kFewUnits = 8, kFewWarps = 8, kFewMost = 32;

struct FewParams {
    const void *x, *wg, *wu;
    int64_t ld_x, ld_w, n, k;
    int m, act;
    void* h;
    int64_t ld_h;
    float* preact;
};

template <typename T> __device__ __forceinline__ void mma_few(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (__is_same(T, __half))
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight 16-bit elements from `p` on a 16-byte boundary, or zeros.  One instruction under a predicate: a load under a branch
// would end in a copy that waits for it.
__device__ __forceinline__ uint4 load_eight(const uint16_t* p, bool go) {
    uint32_t w[4] = {0, 0, 0, 0};
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%5];\n}\n"
                 : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])
                 : "r"(static_cast<int>(go)), "l"(p));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The first `n` of eight elements at any address, the others zero.
__device__ __forceinline__ uint4 gather_eight(const uint16_t* p, int64_t n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i / 2] |= static_cast<uint32_t>(__ldg(p + i)) << (i % 2 * 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float few_gate(int which, float g) {
    switch (which) {
        case BZ_ACT_SILU: return act<BZ_ACT_SILU>(g);
        case BZ_ACT_GELU_TANH: return act<BZ_ACT_GELU_TANH>(g);
        case BZ_ACT_GELU: return act<BZ_ACT_GELU>(g);
        default: return act<BZ_ACT_RELU>(g);
    }
}

// NT: groups of eight tokens.  WIDE: whole steps by 16-byte loads (up to eight rows; more take the ring below).
template <typename T, int NT, bool WIDE>
__global__ void __launch_bounds__(32 * kFewWarps) glu_few_kernel(const __grid_constant__ FewParams p) {
    static_assert(!WIDE || NT == 1, "no call takes it");
    constexpr int kUnroll = 4;   // steps in flight
    __shared__ float part[kFewWarps][2][kFewUnits][8 * NT + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kFewUnits;
    const bool there = unit + g < p.n;
    const int64_t at = there ? (unit + g) * p.ld_w : 0;
    const uint16_t *gate = static_cast<const uint16_t*>(p.wg) + at, *up = static_cast<const uint16_t*>(p.wu) + at;
    const uint16_t* token[NT];
    bool asked[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        asked[c] = c * 8 + g < p.m;
        token[c] = static_cast<const uint16_t*>(p.x) + (asked[c] ? (c * 8 + g) * p.ld_x : 0);
    }
    float acc[NT][4] = {};
    auto multiply_step = [&](const uint4& a, const uint4& b, const uint4 (&x)[NT]) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            mma_few<T>(acc[c], a.x, b.x, a.y, b.y, x[c].x, x[c].y);
            mma_few<T>(acc[c], a.z, b.z, a.w, b.w, x[c].z, x[c].w);
        }
    };
    const int64_t steps = WIDE ? p.k / 32 : 0;   // whole ones, by 16-byte loads
    for (int64_t s0 = warp; s0 < steps; s0 += kFewWarps * kUnroll) {
        uint4 a[kUnroll], b[kUnroll], x[kUnroll][NT];
#pragma unroll
        for (int s = 0; s < kUnroll; ++s) {
            const int64_t step = s0 + s * kFewWarps, k0 = step * 32 + t * 8;
            const bool go = step < steps;
            a[s] = load_eight(gate + k0, go && there);
            b[s] = load_eight(up + k0, go && there);
#pragma unroll
            for (int c = 0; c < NT; ++c) x[s][c] = load_eight(token[c] + k0, go && asked[c]);
        }
#pragma unroll
        for (int s = 0; s < kUnroll; ++s) multiply_step(a[s], b[s], x[s]);
    }
    // the rest of k, or all of it where the operands do not begin on 16-byte boundaries
    for (int64_t step = steps + warp; step * 32 < p.k; step += kFewWarps) {
        const int64_t k0 = step * 32 + t * 8;
        uint4 x[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) x[c] = gather_eight(token[c] + k0, asked[c] ? p.k - k0 : 0);
        multiply_step(gather_eight(gate + k0, there ? p.k - k0 : 0), gather_eight(up + k0, there ? p.k - k0 : 0), x);
    }
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[warp][e >> 1][g][c * 8 + 2 * t + (e & 1)] = acc[c][e];
    __syncthreads();
    for (int e = threadIdx.x; e < kFewUnits * p.m; e += 32 * kFewWarps) {
        const int u = e % kFewUnits, token = e / kFewUnits;   // eight units of a token: 16 bytes
        if (unit + u >= p.n) continue;
        float gate = part[0][0][u][token], up = part[0][1][u][token];
#pragma unroll
        for (int w = 1; w < kFewWarps; ++w) gate += part[w][0][u][token], up += part[w][1][u][token];
        if (p.preact != nullptr) {
            p.preact[token * p.n + unit + u] = gate;
            p.preact[(p.m + token) * p.n + unit + u] = up;
        }
        static_cast<T*>(p.h)[token * p.ld_h + unit + u] = from_f32<T>(few_gate(p.act, gate) * up);
    }
}

// ---- many weights: the same products fed through a ring -------------------------------------------
//
// What the registers of the kernel above can keep in flight ends with every CTA; here two CTAs an SM go from group to
// group of eight units while one thread brings the units' rows by TMA (boxes of eight rows x 256 elements, gate and up, a
// stage) eight stages ahead.  Warp w multiplies elements 32w .. 32w + 31 of a stage.  Rows lie 512 bytes apart, so that the
// two rows of a quarter warp's 16-byte read share banks; padded rows would need a copy a row, and those were slower to
// issue than to arrive (one token, 5461 units of 2048: 18.6 us against 14.2).

constexpr int kFewChunk = 32 * kFewWarps, kFewBox = kFewUnits * kFewChunk * 2, kFewStage = 2 * kFewBox, kFewStages = 8;
constexpr int kFewStreamThreads = 32 * kFewWarps + 32;

__device__ __forceinline__ void tma_load_2d(void* smem_dst, const CUtensorMap* map, uint64_t* bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(smem_dst)),
                 "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y)
                 : "memory");
}

template <int NT> struct FewSums {
    float v[kFewWarps][2][kFewUnits][8 * NT + 1];
};
template <int NT> constexpr int few_stream_smem() { return kFewStages * kFewStage + 2 * static_cast<int>(sizeof(FewSums<NT>)) + 2 * kFewStages * 8 + 16; }

template <typename T, int NT>
__global__ void __launch_bounds__(kFewStreamThreads, 2)
    glu_few_stream_kernel(const __grid_constant__ CUtensorMap gate_map, const __grid_constant__ CUtensorMap up_map, const __grid_constant__ FewParams p) {
    extern __shared__ __align__(128) unsigned char ring[];
    FewSums<NT>* sums = reinterpret_cast<FewSums<NT>*>(ring + kFewStages * kFewStage);   // two, in turn
    uint64_t* full = reinterpret_cast<uint64_t*>(sums + 2);
    uint64_t* empty = full + kFewStages;
    __shared__ int dead_word;
    volatile int* dead = &dead_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if (threadIdx.x == 0) {
        dead_word = 0;
        for (int s = 0; s < kFewStages; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], kFewWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const int64_t groups = (p.n + kFewUnits - 1) / kFewUnits;
    const int k = static_cast<int>(p.k), chunks = (k + kFewChunk - 1) / kFewChunk;
    RingAt<kFewStages> at;
    int filled = 0;
    if (warp == kFewWarps) {
        // ---------------------------------------------------------------- loads; zeros outside the weights
        if (lane == 0) {
            bool alive = true;
            for (int64_t i = blockIdx.x; i < groups && alive; i += gridDim.x)
                for (int c = 0; c < chunks; ++c, at.next()) {
                    if (filled < kFewStages) {
                        ++filled;
                    } else if (!mbar_wait_live(&empty[at.stage], at.parity ^ 1, dead)) {
                        alive = false;
                        break;
                    }
                    unsigned char* to = ring + at.stage * kFewStage;
                    mbar_expect_tx(&full[at.stage], kFewStage);
                    tma_load_2d(to, &gate_map, &full[at.stage], c * kFewChunk, static_cast<int>(i * kFewUnits));
                    tma_load_2d(to + kFewBox, &up_map, &full[at.stage], c * kFewChunk, static_cast<int>(i * kFewUnits));
                }
        }
    } else {
        // ---------------------------------------------------------------- products
        const uint16_t* token[NT];
        bool asked[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            asked[c] = c * 8 + g < p.m;
            token[c] = static_cast<const uint16_t*>(p.x) + (asked[c] ? (c * 8 + g) * p.ld_x : 0);
        }
        int turn = 0;
        for (int64_t i = blockIdx.x; i < groups; i += gridDim.x, turn ^= 1) {
            const int64_t unit = i * kFewUnits;
            float acc[NT][4] = {};
            uint4 x[NT];
            int k0 = warp * 32 + t * 8;
#pragma unroll
            for (int c = 0; c < NT; ++c) x[c] = load_eight(token[c] + k0, asked[c] && k0 + 8 <= k);
            for (int chunk = 0; chunk < chunks; ++chunk, at.next()) {
                const int next = k0 + kFewChunk;
                uint4 ahead[NT];
#pragma unroll
                for (int c = 0; c < NT; ++c) ahead[c] = load_eight(token[c] + next, asked[c] && next + 8 <= k);
                if (k0 < k && k0 + 8 > k) {   // a row's last elements, fewer than eight
                    asm volatile("");
#pragma unroll
                    for (int c = 0; c < NT; ++c) x[c] = gather_eight(token[c] + k0, asked[c] ? k - k0 : 0);
                }
                mbar_wait_live(&full[at.stage], at.parity, dead);   // expired: go on with what is there
                const unsigned char* from = ring + at.stage * kFewStage + g * (kFewChunk * 2) + warp * 64 + t * 16;
                const uint4 a = *reinterpret_cast<const uint4*>(from), b = *reinterpret_cast<const uint4*>(from + kFewBox);
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    mma_few<T>(acc[c], a.x, b.x, a.y, b.y, x[c].x, x[c].y);
                    mma_few<T>(acc[c], a.z, b.z, a.w, b.w, x[c].z, x[c].w);
                    x[c] = ahead[c];
                }
                release_stage(&empty[at.stage]);
                k0 = next;
            }
            FewSums<NT>& part = sums[turn];
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) part.v[warp][e >> 1][g][c * 8 + 2 * t + (e & 1)] = acc[c][e];
            // one barrier a group: the other set of sums is written before the next
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kFewWarps) : "memory");
            const int e = threadIdx.x, u = e % kFewUnits, tk = e / kFewUnits;
            if (tk < p.m && unit + u < p.n) {
                float gate = part.v[0][0][u][tk], up = part.v[0][1][u][tk];
#pragma unroll
                for (int w = 1; w < kFewWarps; ++w) gate += part.v[w][0][u][tk], up += part.v[w][1][u][tk];
                if (p.preact != nullptr) {
                    p.preact[tk * p.n + unit + u] = gate;
                    p.preact[(p.m + tk) * p.n + unit + u] = up;
                }
                static_cast<T*>(p.h)[tk * p.ld_h + unit + u] = from_f32<T>(few_gate(p.act, gate) * up);
            }
        }
    }
    __syncthreads();
    if (*dead && warp == kFewWarps && lane == 0) {
        atomicAdd(&g_glu_timeouts, 1u);
        for (int j = 0; j < filled; ++j, at.next()) mbar_wait(&full[filled < kFewStages ? j : at.stage], filled < kFewStages ? 0 : at.parity ^ 1);  // copies in flight
    }
}

}  // namespace bz
