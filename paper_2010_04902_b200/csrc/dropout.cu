// Dropout whose mask is a function of (seed, offset, element number) and never stored.
#include <cmath>

#include "dropout_rule.h"
#include "philox.cuh"
#include "worker_common.cuh"

namespace bz {

namespace {

constexpr int kThreads = 256;

// Eight elements as loaded: one 16-byte word of 16-bit elements, two of 32-bit ones.
template <typename T> struct Eight {
    static constexpr int kWords = 8 / Word<T>::kN;
    uint4 w[kWords];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = reinterpret_cast<const uint4*>(p)[k];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int k = 0; k < kWords; ++k) Word<T>::unpack(w[k], x + k * Word<T>::kN);
    }
    __device__ __forceinline__ void put(const float (&x)[8]) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = Word<T>::pack(x + k * Word<T>::kN);
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int k = 0; k < kWords; ++k) reinterpret_cast<uint4*>(p)[k] = w[k];
    }
};

// Rows of whole groups of eight on 16-byte boundaries (a contiguous tensor is one such row, but for its last elements).  A thread has
// kFlight groups on their way while it makes their bits.  The generator is most of the work: with single multiplies
// and 64-bit places the loop took 19 instructions an element and 75 % of the issue slots at 131072 x 1024 bfloat16 (93 us); in pairs and with
// constant distances 89 us, 93 % of the copy's rate.
constexpr int kFlight = 4;
template <typename T, bool ONE_ROW>
__global__ void __launch_bounds__(kThreads) dropout_groups_kernel(const T* x, int64_t ld_x, T* out, int64_t ld_out, uint32_t per_row, int64_t groups, int rest, Dropout d) {
    const Keep keep(d);
    // this CTA's groups: base + 0 ... kThreads * kFlight - 1, as far as there are
    const int64_t base = blockIdx.x * static_cast<int64_t>(kThreads * kFlight);
    const int count = static_cast<int>(groups - base < kThreads * kFlight ? groups - base : kThreads * kFlight);
    Eight<T> v[kFlight];
    if constexpr (ONE_ROW) {
        const T* from = x + (base + threadIdx.x) * 8;
        T* to = out + (base + threadIdx.x) * 8;
        auto work = [&](bool whole) {
#pragma unroll
            for (int k = 0; k < kFlight; ++k)
                if (whole || static_cast<int>(threadIdx.x) + k * kThreads < count) v[k].load(from + k * kThreads * 8);
#pragma unroll
            for (int k = 0; k < kFlight; ++k)
                if (whole || static_cast<int>(threadIdx.x) + k * kThreads < count) {
                    float e[8];
                    v[k].get(e);
                    keep.apply(base + threadIdx.x + k * kThreads, d.scale, e);
                    v[k].put(e);
                    v[k].store(to + k * kThreads * 8);
                }
        };
        if (count == kThreads * kFlight)
            work(true);
        else
            work(false);
        if (blockIdx.x == 0 && threadIdx.x < rest) {   // the elements behind the last whole group
            const uint32_t bits = keep.group(groups);
            const int64_t e = groups * 8 + threadIdx.x;
            out[e] = bits >> threadIdx.x & 1 ? from_f32<T>(to_f32(x[e]) * d.scale) : from_f32<T>(0.f);
        }
    } else {
        int64_t to[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int g = static_cast<int>(threadIdx.x) + k * kThreads;
            if (g >= count) continue;
            const uint32_t number = static_cast<uint32_t>(base) + g, i = number / per_row, j = number - i * per_row;   // groups < 2^32
            to[k] = i * ld_out + j * int64_t(8);
            v[k].load(x + i * ld_x + j * int64_t(8));
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
            const int g = static_cast<int>(threadIdx.x) + k * kThreads;
            if (g >= count) continue;
            float e[8];
            v[k].get(e);
            keep.apply(base + g, d.scale, e);
            v[k].put(e);
            v[k].store(out + to[k]);
        }
    }
}

// All other strides.  A CTA takes kTile elements in row-major order (parts of a row, or whole rows): first the bits of their groups,
// each made once (a slot of a row of odd length lies in two groups: twice the generator's work otherwise), then the elements in slots
// (16-byte words where x and out sit alike, else single elements).  5994 x 517 binary32: 8 us, 3.8 at the copy's rate; a thread for
// each group with single elements took 18.
constexpr int kTile = 8192;
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) dropout_tile_kernel(const T* x, int64_t ld_x, T* out, int64_t ld_out, int64_t n, int64_t m, int rows, int64_t parts, Dropout d) {
    __shared__ uint8_t bits[kTile / 8 + 8];
    const Keep keep(d);
    // rows of the tile, and their columns
    const int64_t i0 = parts > 1 ? blockIdx.x / parts : blockIdx.x * static_cast<int64_t>(rows);
    const int64_t c0 = parts > 1 ? blockIdx.x % parts * kTile : 0;
    const int width = static_cast<int>(n - c0 < kTile ? n - c0 : kTile);
    const int count = static_cast<int>(m - i0 < rows ? m - i0 : rows);
    const int64_t first = i0 * n + c0, groups = ((first + static_cast<int64_t>(count) * width + 7) >> 3) - (first >> 3);
    for (int g = threadIdx.x; g < groups; g += kThreads) bits[g] = static_cast<uint8_t>(keep.group((first >> 3) + g));
    __syncthreads();
    const int lead_in = static_cast<int>(first & 7);
    const uint32_t slots = VEC == 1 ? width : width / VEC + 2;   // of a row, some of them empty
#pragma unroll 4
    for (uint32_t q = threadIdx.x; q < slots * count; q += kThreads) {
        const uint32_t r = q / slots, slot = q - r * slots;
        const T* row = x + (i0 + r) * ld_x + c0;
        T* to = out + (i0 + r) * ld_out + c0;
        const int j0 = static_cast<int>(slot) * VEC - row_lead<T, VEC>(row);
        if (j0 >= width) continue;
        float e[VEC];
        load_slot<T, VEC>(row, j0, width, 0.f, e);
        // the bits of elements at ... at + VEC - 1 of the tile; those before a row's first are not used
        const int at = lead_in + static_cast<int>(r) * width + j0, from = at < 0 ? 0 : at;
        const uint32_t pair = (bits[from >> 3] | static_cast<uint32_t>(bits[(from >> 3) + 1]) << 8) >> (from & 7) << (from - at);
#pragma unroll
        for (int k = 0; k < VEC; ++k) e[k] = pair >> k & 1 ? e[k] * d.scale : 0.f;
        store_slot<T, VEC>(to, j0, width, e);
    }
}

template <typename T> int dispatch(const void* x, int64_t ld_x, void* out, int64_t ld_out, int64_t m, int64_t n, const Dropout& d, cudaStream_t s) {
    const T* in = static_cast<const T*>(x);
    T* to = static_cast<T*>(out);
    if (m > 1 && ld_x == n && ld_out == n) n *= m, m = 1;
    const bool aligned = aligned16(x) && aligned16(out);
    const int64_t groups = m * (n / 8), blocks = (groups + kThreads * kFlight - 1) / (kThreads * kFlight);
    if (aligned && m == 1 && blocks < (int64_t(1) << 31)) {
        dropout_groups_kernel<T, true><<<static_cast<unsigned>(blocks > 0 ? blocks : 1), kThreads, 0, s>>>(in, 0, to, 0, 0, groups, static_cast<int>(n & 7), d);
    } else if (aligned && n % 8 == 0 && ld_x * static_cast<int64_t>(sizeof(T)) % 16 == 0 && ld_out * static_cast<int64_t>(sizeof(T)) % 16 == 0 &&
               groups < (int64_t(1) << 32) - kThreads * kFlight) {
        dropout_groups_kernel<T, false><<<static_cast<unsigned>(blocks), kThreads, 0, s>>>(in, ld_x, to, ld_out, static_cast<uint32_t>(n / 8), groups, 0, d);
    } else {
        const int64_t parts = (n + kTile - 1) / kTile;
        const int rows = parts > 1 ? 1 : static_cast<int>(kTile / n < m ? kTile / n : m);
        const int64_t tiles = parts > 1 ? m * parts : (m + rows - 1) / rows;
        if (tiles >= (int64_t(1) << 31)) return BZ_ERR_UNSUPPORTED;
        const uintptr_t apart = reinterpret_cast<uintptr_t>(x) - reinterpret_cast<uintptr_t>(out);
        const bool alike = (apart & 15) == 0 && (m == 1 || (ld_x - ld_out) * static_cast<int64_t>(sizeof(T)) % 16 == 0);
        if (alike)
            dropout_tile_kernel<T, Word<T>::kN><<<static_cast<unsigned>(tiles), kThreads, 0, s>>>(in, ld_x, to, ld_out, n, m, rows, parts, d);
        else
            dropout_tile_kernel<T, 1><<<static_cast<unsigned>(tiles), kThreads, 0, s>>>(in, ld_x, to, ld_out, n, m, rows, parts, d);
    }
    note_launch();
    return check_launch();
}

}  // namespace

}  // namespace bz

using namespace bz;

extern "C" int bz_dropout(const void* x, int64_t ld_x, int dtype, int64_t m, int64_t n, double rate, const uint64_t* rng, void* out, int64_t ld_out,
                          void* stream) {
    const int bytes = element_bytes(dtype);
    uint32_t least;
    if (bytes == 0 || m < 0 || n < 0 || !drop_threshold(rate, &least)) return BZ_ERR_INVALID_ARG;
    if (m >= (int64_t(1) << 40) || n >= (int64_t(1) << 40) || (n > 0 && m >= (int64_t(1) << 50) / n)) return BZ_ERR_UNSUPPORTED;
    if (m == 0 || n == 0) return BZ_OK;
    if (x == nullptr || out == nullptr || rng == nullptr || !aligned8(rng) || (m > 1 && (ld_x < n || ld_out < n)) || reinterpret_cast<uintptr_t>(x) % bytes ||
        reinterpret_cast<uintptr_t>(out) % bytes)
        return BZ_ERR_INVALID_ARG;
    if (m > 1 && (ld_x >= (int64_t(1) << 40) || ld_out >= (int64_t(1) << 40))) return BZ_ERR_UNSUPPORTED;
    const Dropout d{rng, least, drop_scale(least)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == BZ_F32) return dispatch<float>(x, ld_x, out, ld_out, m, n, d, s);
    if (dtype == BZ_F16) return dispatch<__half>(x, ld_x, out, ld_out, m, n, d, s);
    return dispatch<__nv_bfloat16>(x, ld_x, out, ld_out, m, n, d, s);
}
