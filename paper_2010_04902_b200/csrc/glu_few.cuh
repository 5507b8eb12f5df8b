// Gated feed-forward block for few rows (tokens): bound by reading both weights once.
//
// A CTA takes eight hidden units; its eight warps take 32-wide steps of k in turn, so the units' weights stream through
// registers by 16-byte loads that a quad of lanes makes contiguous (64 bytes of each of 8 rows at a time, four or eight steps in
// flight).  The products run on mma.sync (m16n8k16: the eight gate rows above the eight up rows, times 8 tokens), so one
// thread ends with g and u of its unit: at one to 32 tokens the arithmetic is far below either tensor path's rate, and this
// one takes its operands from the registers the loads end in.  The order of k inside an MMA is free as long as weights and
// tokens agree, so lane t of a quad feeds its own eight consecutive elements as the pairs (2t, 2t+1), (2t+8, 2t+9) of two
// MMAs, and no element moves between lanes.
// The eight warps' sums meet in shared memory and are added in order.
#pragma once

#include "glu_product.cuh"

namespace bz {

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
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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

// NT: groups of eight tokens.
template <typename T, int NT, bool WIDE>
__global__ void __launch_bounds__(32 * kFewWarps) glu_few_kernel(const __grid_constant__ FewParams p) {
    constexpr int kUnroll = NT == 1 ? 4 : 8;   // 24 tokens, 5461 units of 2048: 14.8 us against 16.9 with four
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
