// Element types and row access shared by the operators of a worker's step (glu, bias_softmax, distill).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bz_common.cuh"

namespace bz {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

inline int element_bytes(int dtype) { return dtype == BZ_F32 ? 4 : (dtype == BZ_F16 || dtype == BZ_BF16 ? 2 : 0); }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Elements of one 16-byte word as binary32, and back.
template <typename T> struct Word;
template <> struct Word<float> {
    static constexpr int kN = 4;
    __device__ static __forceinline__ void unpack(const uint4& w, float* x) {
        x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y), x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
    }
    __device__ static __forceinline__ uint4 pack(const float* x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
__device__ __forceinline__ float2 unpack2(__nv_bfloat16, uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 unpack2(__half, uint32_t w) {
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
}
__device__ __forceinline__ uint32_t pack2(__nv_bfloat16, float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ uint32_t pack2(__half, float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
template <typename T> struct Word16 {
    static constexpr int kN = 8;
    __device__ static __forceinline__ void unpack(const uint4& w, float* x) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(T(), u[i]);
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
    __device__ static __forceinline__ uint4 pack(const float* x) {
        return make_uint4(pack2(T(), x[0], x[1]), pack2(T(), x[2], x[3]), pack2(T(), x[4], x[5]), pack2(T(), x[6], x[7]));
    }
};
template <> struct Word<__half> : Word16<__half> {};
template <> struct Word<__nv_bfloat16> : Word16<__nv_bfloat16> {};

// A row of `n` elements cut into slots of VEC.  VEC = the elements of a 16-byte word: slots lie on 16-byte boundaries,
// so the first one begins `lead` elements before the row; slots that reach over an end are read and written element by
// element.  VEC = 1: a slot is an element, for tensors whose rows do not sit alike relative to 16-byte boundaries.
template <typename T, int VEC> __device__ __forceinline__ int row_lead(const T* row) {
    return VEC == 1 ? 0 : static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
}
// x[i] = element j0 + i of the row where that lies in [0, n); the others keep `fill`.
template <typename T, int VEC> __device__ __forceinline__ void load_slot(const T* row, int64_t j0, int64_t n, float fill, float (&x)[VEC]) {
    if constexpr (VEC == 1) {
        x[0] = j0 < n ? to_f32(row[j0]) : fill;
    } else if (j0 >= 0 && j0 + VEC <= n) {
        Word<T>::unpack(*reinterpret_cast<const uint4*>(row + j0), x);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = j0 + i >= 0 && j0 + i < n ? to_f32(row[j0 + i]) : fill;
    }
}
template <typename T, int VEC> __device__ __forceinline__ void store_slot(T* row, int64_t j0, int64_t n, const float (&x)[VEC]) {
    if constexpr (VEC == 1) {
        if (j0 < n) row[j0] = from_f32<T>(x[0]);
    } else if (j0 >= 0 && j0 + VEC <= n) {
        *reinterpret_cast<uint4*>(row + j0) = Word<T>::pack(x);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (j0 + i >= 0 && j0 + i < n) row[j0 + i] = from_f32<T>(x[i]);
    }
}

// 2^x in one instruction (ex2.approx: at most two units in the last place; results below 2^-126 become 0).
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A part of a row of softmax arguments: (largest z, sum of e^((z - that)/T)).  An empty part is (-inf, 0).
//
// With c = log2(e)/T an exponent is one multiply-add, z*c - m*c.  The product m*c is rounded, but everything that is
// compared or joined uses the same rounded number, so its error (up to 2^-25 of the product) cancels.  Where the product is
// beyond 128 - up to a row of the type's lowest values, whose product may not even be finite - that error is no longer
// small, and exponents are (z - m)*c, one operation more.  Parts of either kind may be joined: they differ by less than
// 128 * 2^-25 in the exponent.
struct MaxSum {
    float m, s;
};
// A product that no multiply-add takes in.
__device__ __forceinline__ float rounded_product(float a, float b) {
    float y;
    asm("mul.rn.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
struct Reference {
    float m, mc;   // a part's largest z (0 for an empty part) and its rounded product with c
    bool apart;
    __device__ __forceinline__ Reference(float largest, float c) : m(largest == -INFINITY ? 0.f : largest), mc(rounded_product(m, c)), apart(fabsf(mc) > 128.f && !isinf(m)) {}
    // exponent of z, which is at most m; z may be -inf
    __device__ __forceinline__ float of(float z, float c) const { return apart ? (z - m) * c : fmaf(z, c, -mc); }
    // 2^(what the rounding of m*c left out): sums are kept relative to mc inside a kernel and to m itself outside
    __device__ __forceinline__ float left_out(float c) const { return apart || isinf(m) ? 1.f : exp2_fast(fmaf(m, c, -mc)); }
    // exponent of another part's reference: between the two rounded products
    __device__ __forceinline__ float of_part(float other, float c) const { return apart ? (other - m) * c : rounded_product(other, c) - mc; }
};
__device__ __forceinline__ float warp_sum(float v);
__device__ __forceinline__ float warp_max(float v);
// The parts of a warp's lanes as one.
__device__ __forceinline__ MaxSum warp_join(const MaxSum& v, float c) {
    const float m = warp_max(v.m);
    const Reference r(m, c);
    return {m, warp_sum(v.s == 0.f ? 0.f : v.s * exp2_fast(r.of_part(v.m, c)))};
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
    float m;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}

// ---- rings of stages in shared memory -------------------------------------------------------------

// Position in a ring: the stage and the parity of its current round.  Counted, not divided out: the threads that load and
// issue run one instruction after another, and 64-bit remainders between
// two MMAs cost a seventh of the rate (8192 x 4096 x 8192 forward: 825 against 725 us).
template <int STAGES> struct RingAt {
    int stage = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() {
        if (++stage == STAGES) stage = 0, parity ^= 1;
    }
};

// ---- loads that stay in flight -------------------------------------------------------------------

// Bounds of a tensor's memory: from its first element to behind its last.
struct Extent {
    const char *begin, *end;
    // whether every 16-byte word that a row of n elements touches lies in the tensor
    template <typename T> __device__ __forceinline__ bool around(const T* row, int64_t n) const {
        return reinterpret_cast<const char*>(row) - 16 >= begin && reinterpret_cast<const char*>(row + n) + 16 <= end;
    }
};
// A slot as it was loaded.  A load under a branch ends in a copy of its registers, and a copy waits for the load; so the load
// is one instruction under a predicate, into registers that keep what they held.  A slot that reaches over an end of its
// row is read whole where the tensor goes on (what is not the row's is masked later); in the few rows at the tensor's ends
// it is read element by element when it is used.
template <typename T, int VEC> struct Raw {
    uint32_t w[4] = {0, 0, 0, 0};
    __device__ __forceinline__ void fetch(const T* p, bool go) {
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "setp.ne.b32 p, %4, 0;\n"
            "@p ld.global.v4.u32 {%0, %1, %2, %3}, [%5];\n"
            "}\n"
            : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])
            : "r"(static_cast<int>(go)), "l"(p));
    }
    __device__ __forceinline__ void get(float (&x)[VEC]) const { Word<T>::unpack(make_uint4(w[0], w[1], w[2], w[3]), x); }
};
template <typename T> struct Raw<T, 1> {
    uint32_t w = 0;
    __device__ __forceinline__ void fetch(const T* p, bool go) {
        if constexpr (sizeof(T) == 4) {
            asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %1, 0;\n@p ld.global.u32 %0, [%2];\n}\n" : "+r"(w) : "r"(static_cast<int>(go)), "l"(p));
        } else {
            uint16_t h = static_cast<uint16_t>(w);
            asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %1, 0;\n@p ld.global.u16 %0, [%2];\n}\n" : "+h"(h) : "r"(static_cast<int>(go)), "l"(p));
            w = h;
        }
    }
    __device__ __forceinline__ void get(float (&x)[1]) const {
        if constexpr (sizeof(T) == 4) {
            x[0] = __uint_as_float(w);
        } else {
            T e;
            const uint16_t h = static_cast<uint16_t>(w);
            memcpy(&e, &h, 2);
            x[0] = to_f32(e);
        }
    }
};
// Keeps what follows in a branch of its own: not worth executing under a predicate.
__device__ __forceinline__ void rare() { asm volatile(""); }
// For a slot that was not fetched because it reaches over an end of a tensor.
template <typename T, int VEC> __device__ __forceinline__ void read_apart(const T* row, int64_t j0, int64_t n, float (&x)[VEC]) {
    rare();
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = j0 + i >= 0 && j0 + i < n ? to_f32(row[j0 + i]) : 0.f;
}
template <typename T, int VEC> __device__ __forceinline__ void store_whole(T* p, const float (&x)[VEC]) {
    if constexpr (VEC == 1)
        *p = from_f32<T>(x[0]);
    else
        *reinterpret_cast<uint4*>(p) = Word<T>::pack(x);
}

// ---- arrays in registers, two elements an instruction where there are two -------------------------

// x[i] = x[i]*a + b[i]
template <int N> __device__ __forceinline__ void multiply_add(float (&x)[N], float a, const float (&b)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 y = __ffma2_rn(make_float2(x[i], x[i + 1]), make_float2(a, a), make_float2(b[i], b[i + 1]));
            x[i] = y.x, x[i + 1] = y.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(x[i], a, b[i]);
    }
}
template <int N> __device__ __forceinline__ void multiply(float (&x)[N], float a) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 y = __fmul2_rn(make_float2(x[i], x[i + 1]), make_float2(a, a));
            x[i] = y.x, x[i + 1] = y.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= a;
    }
}
// x[i] *= a[i]
template <int N> __device__ __forceinline__ void multiply_by(float (&x)[N], const float (&a)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 y = __fmul2_rn(make_float2(x[i], x[i + 1]), make_float2(a[i], a[i + 1]));
            x[i] = y.x, x[i + 1] = y.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= a[i];
    }
}
// s += x*y in two partial sums.
template <int N> __device__ __forceinline__ void add_products(float2& s, const float (&x)[N], const float (&y)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) s = __ffma2_rn(make_float2(x[i], x[i + 1]), make_float2(y[i], y[i + 1]), s);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s.x = fmaf(x[i], y[i], s.x);
    }
}
// Largest of m and x (NaNs do not count).
template <int N> __device__ __forceinline__ float largest(float m, const float (&x)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(x[i]), "f"(x[i + 1]));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
    }
    return m;
}
// s += x, element by element in two partial sums.
template <int N> __device__ __forceinline__ void add_up(float2& s, const float (&x)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) s = __fadd2_rn(s, make_float2(x[i], x[i + 1]));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s.x += x[i];
    }
}
// x[i] = 2^(exponent of x[i]) relative to r.
template <int N> __device__ __forceinline__ void exponentials(float (&x)[N], const Reference& r, float c) {
    if (r.apart) {
        rare();
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] -= r.m;
    }
    float b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) b[i] = r.apart ? 0.f : -r.mc;
    multiply_add(x, c, b);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = exp2_fast(x[i]);
}

}  // namespace bz
