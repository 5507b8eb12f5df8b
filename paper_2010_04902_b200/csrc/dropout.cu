// Dropout whose mask is a function of (seed, offset, element number) and never stored.
#include <cmath>

#include "dropout_rule.h"
#include "philox.cuh"
#include "worker_common.cuh"

namespace bz {

namespace {

// A thread takes the eight elements of one output of the generator.  Works for all strides.
template <typename T>
__global__ void __launch_bounds__(256) dropout_any_kernel(const T* x, int64_t ld_x, T* out, int64_t ld_out, int64_t n, int64_t size, Dropout d) {
    const Keep keep(d);
    const int64_t groups = (size + 7) / 8, step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t g = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; g < groups; g += step) {
        const uint32_t bits = keep.group(g);
        int64_t i = g * 8 / n, j = g * 8 % n;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (g * 8 + k < size) out[i * ld_out + j] = bits >> k & 1 ? from_f32<T>(to_f32(x[i * ld_x + j]) * d.scale) : from_f32<T>(0.f);
            if (++j == n) j = 0, ++i;
        }
    }
}

template <typename T> int dispatch(const void* x, int64_t ld_x, void* out, int64_t ld_out, int64_t m, int64_t n, const Dropout& d, cudaStream_t s) {
    const int64_t blocks = ((m * n + 7) / 8 + 255) / 256;
    dropout_any_kernel<T><<<static_cast<unsigned>(blocks < 8 * kNumSMs ? blocks : 8 * kNumSMs), 256, 0, s>>>(static_cast<const T*>(x), ld_x, static_cast<T*>(out), ld_out, n, m * n, d);
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
