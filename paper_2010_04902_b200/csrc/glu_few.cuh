// Gated feed-forward block for few rows (tokens): bound by reading both weights once.
//
// A CTA takes 16 hidden units; its eight warps take 32-wide steps of k in turn, so a unit's weights stream through
// registers by 16-byte loads that a quad of lanes makes contiguous (64 bytes of each of 8 rows at a time, four steps in
// flight, two for more than 16 tokens, whose own registers would leave one CTA an SM).  The products run on mma.sync (m16n8k16: 16 units x 8 tokens): at one to 32 tokens the arithmetic is far below
// either tensor path's rate, and this one takes its operands from the registers the loads end in.  The order of k inside
// an MMA is free as long as weights and tokens agree, so lane t of a quad feeds its own eight consecutive elements as the
// pairs (2t, 2t+1), (2t+8, 2t+9) of two MMAs, and no element moves between lanes.
// The eight warps' sums meet in shared memory and are added in order.
#pragma once

#include "glu_product.cuh"

namespace bz {

constexpr int kFewUnits = 16, kFewWarps = 8, kFewMost = 32;

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
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight 16-bit elements from `p`, of which `n` exist (n <= 0: none); the others are zero.  WIDE: p on a 16-byte boundary.
// The load is one instruction under a predicate: one under a branch would end in a copy that waits for it.
template <bool WIDE> __device__ __forceinline__ uint4 load_eight(const uint16_t* p, int64_t n) {
    uint32_t w[4] = {0, 0, 0, 0};
    if constexpr (WIDE) {
        const int go = n >= 8;
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%5];\n}\n"
                     : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])
                     : "r"(go), "l"(p));
        if (n <= 0 || n >= 8) return make_uint4(w[0], w[1], w[2], w[3]);
        asm volatile("");   // rare: the last elements of a row whose length is no multiple of eight
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i / 2] |= static_cast<uint32_t>(__ldg(p + i)) << (i % 2 * 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// NT: groups of eight tokens.
template <typename T, int NT, bool WIDE>
__global__ void __launch_bounds__(32 * kFewWarps) glu_few_kernel(const __grid_constant__ FewParams p) {
    constexpr int kUnroll = NT == 4 ? 2 : 4;
    __shared__ float part[kFewWarps][2][kFewUnits][8 * NT + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kFewUnits;
    const uint16_t* rows[4];   // gate g, gate g + 8, up g, up g + 8
    bool there[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = unit + g + (i & 1) * 8;
        there[i] = r < p.n;
        rows[i] = static_cast<const uint16_t*>(i < 2 ? p.wg : p.wu) + (there[i] ? r * p.ld_w : 0);
    }
    float acc[2][NT][4] = {};
    for (int64_t s0 = warp * 32; s0 < p.k; s0 += 32 * kFewWarps * kUnroll) {
        uint4 w[kUnroll][4], x[kUnroll][NT];
#pragma unroll
        for (int s = 0; s < kUnroll; ++s) {
            const int64_t k0 = s0 + s * 32 * kFewWarps + t * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[s][i] = load_eight<WIDE>(rows[i] + k0, there[i] ? p.k - k0 : 0);
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const int token = c * 8 + g;
                x[s][c] = load_eight<WIDE>(static_cast<const uint16_t*>(p.x) + (token < p.m ? token * p.ld_x : 0) + k0, token < p.m ? p.k - k0 : 0);
            }
        }
#pragma unroll
        for (int s = 0; s < kUnroll; ++s)
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 &a = w[s][2 * i], &b = w[s][2 * i + 1], &v = x[s][c];
                    mma_few<T>(acc[i][c], a.x, b.x, a.y, b.y, v.x, v.y);
                    mma_few<T>(acc[i][c], a.z, b.z, a.w, b.w, v.z, v.w);
                }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[warp][i][g + (e >> 1) * 8][c * 8 + 2 * t + (e & 1)] = acc[i][c][e];
    __syncthreads();
    for (int e = threadIdx.x; e < kFewUnits * p.m; e += 32 * kFewWarps) {
        const int u = e % kFewUnits, token = e / kFewUnits;
        if (unit + u >= p.n) continue;
        float gate = part[0][0][u][token], up = part[0][1][u][token];
#pragma unroll
        for (int w = 1; w < kFewWarps; ++w) gate += part[w][0][u][token], up += part[w][1][u][token];
        if (p.preact != nullptr) {
            p.preact[token * p.n + unit + u] = gate;
            p.preact[(p.m + token) * p.n + unit + u] = up;
        }
        float a;
        switch (p.act) {
            case BZ_ACT_SILU: a = act<BZ_ACT_SILU>(gate); break;
            case BZ_ACT_GELU_TANH: a = act<BZ_ACT_GELU_TANH>(gate); break;
            case BZ_ACT_GELU: a = act<BZ_ACT_GELU>(gate); break;
            default: a = act<BZ_ACT_RELU>(gate); break;
        }
        static_cast<T*>(p.h)[token * p.ld_h + unit + u] = from_f32<T>(a * up);
    }
}

}  // namespace bz
