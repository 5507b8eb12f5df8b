// Random bits by counter: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011).
#pragma once

#include <stdint.h>

namespace bz {

// Ten rounds, as the paper's default: 20 wide products and 40 logic operations for eight elements' bits.
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = static_cast<uint64_t>(c.x) * 0xD2511F53u, q = static_cast<uint64_t>(c.z) * 0xCD9E8D57u;
        c = make_uint4(static_cast<uint32_t>(q >> 32) ^ c.y ^ k0, static_cast<uint32_t>(q), static_cast<uint32_t>(p >> 32) ^ c.w ^ k1, static_cast<uint32_t>(p));
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return c;
}

// Which elements stay, 16 bits an element.
struct Dropout {
    const uint64_t* rng;   // seed, offset
    uint32_t least;        // an element stays if its bits are at least this
    float scale;           // of what stays
};
struct Keep {
    uint32_t k0, k1, o0, o1, least;
    __device__ __forceinline__ explicit Keep(const Dropout& d) : least(d.least) {
        uint64_t seed = 0, offset = 0;
        if (d.rng != nullptr) seed = d.rng[0], offset = d.rng[1];
        k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32), o0 = static_cast<uint32_t>(offset), o1 = static_cast<uint32_t>(offset >> 32);
    }
    // the 128 bits of elements 8 * number ... 8 * number + 7
    __device__ __forceinline__ uint4 words(uint64_t number) const {
        return philox(make_uint4(static_cast<uint32_t>(number), static_cast<uint32_t>(number >> 32), o0, o1), k0, k1);
    }
    // whether the element of the lower, the upper 16 bits of a word stays
    __device__ __forceinline__ bool lower(uint32_t w) const { return w << 16 >= least << 16; }
    __device__ __forceinline__ bool upper(uint32_t w) const { return w >= least << 16; }
    // bit i: element 8 * number + i stays
    __device__ __forceinline__ uint32_t group(uint64_t number) const {
        const uint4 w = words(number);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) bits |= (lower(u[i]) ? 1u << (2 * i) : 0u) | (upper(u[i]) ? 2u << (2 * i) : 0u);
        return bits;
    }
    // x[i] = element 8 * number + i, scaled or 0
    __device__ __forceinline__ void apply(uint64_t number, float scale, float (&x)[8]) const {
        const uint4 w = words(number);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 y = __fmul2_rn(make_float2(x[2 * i], x[2 * i + 1]), make_float2(scale, scale));
            x[2 * i] = lower(u[i]) ? y.x : 0.f;
            x[2 * i + 1] = upper(u[i]) ? y.y : 0.f;
        }
    }
};

}  // namespace bz
