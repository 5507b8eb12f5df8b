// Gated feed-forward block and its gradient.
#include "worker_common.cuh"

namespace bz {

namespace {

template <int ACT> __device__ __forceinline__ float act(float g) {
    if constexpr (ACT == BZ_ACT_SILU) return g / (1.f + __expf(-g));
    if constexpr (ACT == BZ_ACT_GELU_TANH) return g / (1.f + __expf(-1.5957691216f * (g + 0.044715f * g * g * g)));
    if constexpr (ACT == BZ_ACT_GELU) return 0.5f * g * (1.f + erff(g * 0.70710678f));
    return fmaxf(g, 0.f);
}
template <int ACT> __device__ __forceinline__ float act_slope(float g) {
    if constexpr (ACT == BZ_ACT_SILU) {
        const float s = 1.f / (1.f + __expf(-g));
        return s * (1.f + g * (1.f - s));
    }
    if constexpr (ACT == BZ_ACT_GELU_TANH) {  // (1 + tanh y)/2 = 1/(1 + exp(-2y))
        const float s = 1.f / (1.f + __expf(-1.5957691216f * (g + 0.044715f * g * g * g)));
        return s + g * s * (1.f - s) * 1.5957691216f * (1.f + 0.134145f * g * g);
    }
    if constexpr (ACT == BZ_ACT_GELU) return 0.5f * (1.f + erff(g * 0.70710678f)) + g * 0.39894228f * __expf(-0.5f * g * g);
    return g > 0.f ? 1.f : 0.f;
}

// acc[r][c] = sum over l of A(i0 + 4 ty + r, l) * B(j0 + 4 tx + c, l), A(i, l) = a[i*ai + l*al] for i < ni, l < nl.
template <typename T>
__device__ __forceinline__ void tile_product(const T* a, int64_t ai, int64_t al, const T* b, int64_t bj, int64_t bl, int64_t i0, int64_t ni,
                                             int64_t j0, int64_t nj, int64_t nl, float (&acc)[4][4], float (*sa)[65], float (*sb)[65]) {
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int64_t l0 = 0; l0 < nl; l0 += 16) {
        for (int e = threadIdx.x; e < 1024; e += 256) {
            const int l = al == 1 ? e % 16 : e / 64, i = al == 1 ? e / 16 : e % 64;
            sa[l][i] = i0 + i < ni && l0 + l < nl ? to_f32(a[(i0 + i) * ai + (l0 + l) * al]) : 0.f;
            const int l2 = bl == 1 ? e % 16 : e / 64, j = bl == 1 ? e / 16 : e % 64;
            sb[l2][j] = j0 + j < nj && l0 + l2 < nl ? to_f32(b[(j0 + j) * bj + (l0 + l2) * bl]) : 0.f;
        }
        __syncthreads();
        for (int l = 0; l < 16; ++l)
            for (int r = 0; r < 4; ++r)
                for (int c = 0; c < 4; ++c) acc[r][c] = fmaf(sa[l][4 * ty + r], sb[l][4 * tx + c], acc[r][c]);
        __syncthreads();
    }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) glu_kernel(const T* x, int64_t ld_x, const T* wg, const T* wu, int64_t ld_w, int64_t m, int64_t n,
                                                  int64_t k, T* h, int64_t ld_h, float* preact) {
    __shared__ float sa[16][65], sb[16][65];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 64, j0 = static_cast<int64_t>(blockIdx.y) * 64;
    float g[4][4] = {}, u[4][4] = {};
    tile_product(x, ld_x, int64_t(1), wg, ld_w, int64_t(1), i0, m, j0, n, k, g, sa, sb);
    tile_product(x, ld_x, int64_t(1), wu, ld_w, int64_t(1), i0, m, j0, n, k, u, sa, sb);
    for (int r = 0; r < 4; ++r)
        for (int c = 0; c < 4; ++c) {
            const int64_t i = i0 + threadIdx.x / 16 * 4 + r, j = j0 + threadIdx.x % 16 * 4 + c;
            if (i >= m || j >= n) continue;
            h[i * ld_h + j] = from_f32<T>(act<ACT>(g[r][c]) * u[r][c]);
            if (preact != nullptr) preact[i * n + j] = g[r][c], preact[(m + i) * n + j] = u[r][c];
        }
}

// dgu[0] = dh * u * act'(g), dgu[1] = dh * act(g), each [m][n].
template <typename T, int ACT>
__global__ void __launch_bounds__(256) glu_dgu_kernel(const float* preact, const T* dh, int64_t ld_dh, int64_t m, int64_t n, T* dgu) {
    for (int64_t e = blockIdx.x * int64_t(256) + threadIdx.x; e < m * n; e += gridDim.x * int64_t(256)) {
        const float g = preact[e], u = preact[m * n + e], d = to_f32(dh[e / n * ld_dh + e % n]);
        dgu[e] = from_f32<T>(d * u * act_slope<ACT>(g));
        dgu[m * n + e] = from_f32<T>(d * act<ACT>(g));
    }
}

template <typename T>
__global__ void __launch_bounds__(256) glu_dx_kernel(const T* dgu, const T* wg, const T* wu, int64_t ld_w, int64_t m, int64_t n, int64_t k, T* dx, int64_t ld_dx) {
    __shared__ float sa[16][65], sb[16][65];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 64, j0 = static_cast<int64_t>(blockIdx.y) * 64;
    float acc[4][4] = {};
    tile_product(dgu, n, int64_t(1), wg, int64_t(1), ld_w, i0, m, j0, k, n, acc, sa, sb);
    tile_product(dgu + m * n, n, int64_t(1), wu, int64_t(1), ld_w, i0, m, j0, k, n, acc, sa, sb);
    for (int r = 0; r < 4; ++r)
        for (int c = 0; c < 4; ++c) {
            const int64_t i = i0 + threadIdx.x / 16 * 4 + r, j = j0 + threadIdx.x % 16 * 4 + c;
            if (i < m && j < k) dx[i * ld_dx + j] = from_f32<T>(acc[r][c]);
        }
}

template <typename T, typename G>
__global__ void __launch_bounds__(256) glu_dw_kernel(const T* dgu, const T* x, int64_t ld_x, int64_t m, int64_t n, int64_t k, G* dwg, G* dwu, int64_t ld_dw) {
    __shared__ float sa[16][65], sb[16][65];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 64, j0 = static_cast<int64_t>(blockIdx.y) * 64;
    float acc[4][4] = {};
    tile_product(dgu + blockIdx.z * m * n, int64_t(1), n, x, int64_t(1), ld_x, i0, n, j0, k, m, acc, sa, sb);
    G* out = blockIdx.z ? dwu : dwg;
    for (int r = 0; r < 4; ++r)
        for (int c = 0; c < 4; ++c) {
            const int64_t i = i0 + threadIdx.x / 16 * 4 + r, j = j0 + threadIdx.x % 16 * 4 + c;
            if (i < n && j < k) out[i * ld_dw + j] = from_f32<G>(acc[r][c]);
        }
}

unsigned tiles(int64_t n) { return static_cast<unsigned>((n + 63) / 64); }

template <typename T, int ACT>
int forward(const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, int64_t m, int64_t n, int64_t k, void* h, int64_t ld_h,
            float* preact, cudaStream_t s) {
    glu_kernel<T, ACT><<<dim3(tiles(m), tiles(n)), 256, 0, s>>>(static_cast<const T*>(x), ld_x, static_cast<const T*>(wg),
                                                                 static_cast<const T*>(wu), ld_w, m, n, k, static_cast<T*>(h), ld_h, preact);
    note_launch();
    return check_launch();
}

template <typename T, int ACT>
int backward(const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, const float* preact, const void* dh, int64_t ld_dh,
             int64_t m, int64_t n, int64_t k, void* dx, int64_t ld_dx, void* dwg, void* dwu, int64_t ld_dw, int grad_dtype, void* ws, cudaStream_t s) {
    T* dgu = static_cast<T*>(ws);
    glu_dgu_kernel<T, ACT><<<8 * kNumSMs, 256, 0, s>>>(preact, static_cast<const T*>(dh), ld_dh, m, n, dgu);
    note_launch();
    if (dx != nullptr && m > 0 && k > 0) {
        glu_dx_kernel<T><<<dim3(tiles(m), tiles(k)), 256, 0, s>>>(dgu, static_cast<const T*>(wg), static_cast<const T*>(wu), ld_w, m, n, k, static_cast<T*>(dx), ld_dx);
        note_launch();
    }
    if (dwg != nullptr && n > 0 && k > 0) {
        const dim3 grid(tiles(n), tiles(k), 2);
        if (grad_dtype == BZ_F32)
            glu_dw_kernel<T, float><<<grid, 256, 0, s>>>(dgu, static_cast<const T*>(x), ld_x, m, n, k, static_cast<float*>(dwg), static_cast<float*>(dwu), ld_dw);
        else
            glu_dw_kernel<T, T><<<grid, 256, 0, s>>>(dgu, static_cast<const T*>(x), ld_x, m, n, k, static_cast<T*>(dwg), static_cast<T*>(dwu), ld_dw);
        note_launch();
    }
    return check_launch();
}

#define BZ_GLU_SWITCH(CALL)                                                   \
    switch (act) {                                                            \
        case BZ_ACT_SILU: return dtype == BZ_F16 ? CALL(__half, BZ_ACT_SILU) : CALL(__nv_bfloat16, BZ_ACT_SILU);                \
        case BZ_ACT_GELU_TANH: return dtype == BZ_F16 ? CALL(__half, BZ_ACT_GELU_TANH) : CALL(__nv_bfloat16, BZ_ACT_GELU_TANH); \
        case BZ_ACT_GELU: return dtype == BZ_F16 ? CALL(__half, BZ_ACT_GELU) : CALL(__nv_bfloat16, BZ_ACT_GELU);                \
        default: return dtype == BZ_F16 ? CALL(__half, BZ_ACT_RELU) : CALL(__nv_bfloat16, BZ_ACT_RELU);                         \
    }

int check(const void* x, int64_t ld_x, const void* wg, const void* wu, int64_t ld_w, int64_t m, int64_t n, int64_t k, int dtype, int act) {
    if (m < 0 || n < 0 || k < 0 || element_bytes(dtype) == 0 || act < BZ_ACT_SILU || act > BZ_ACT_RELU) return BZ_ERR_INVALID_ARG;
    const int64_t most = (int64_t(1) << 31) - 1;
    if (m > most || n > most || k > most || dtype == BZ_F32) return BZ_ERR_UNSUPPORTED;
    if ((m > 1 && ld_x < k) || (n > 1 && ld_w < k)) return BZ_ERR_INVALID_ARG;
    if ((m > 0 && k > 0 && x == nullptr) || (n > 0 && k > 0 && (wg == nullptr || wu == nullptr))) return BZ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(wg) | reinterpret_cast<uintptr_t>(wu)) & 1) return BZ_ERR_INVALID_ARG;
    return BZ_OK;
}

// Whether a tensor map can describe rows like these.
bool laid_out(const void* p, int64_t ld, int64_t rows) { return aligned16(p) && (rows <= 1 || ld % 8 == 0); }

}  // namespace

}  // namespace bz

using namespace bz;

extern "C" size_t bz_glu_workspace_bytes(int64_t m, int64_t n, int64_t k, int dtype, int backward) {
    if (m < 0 || n < 0 || k < 0 || (dtype != BZ_F16 && dtype != BZ_BF16)) return 0;
    return backward ? round_up(static_cast<size_t>(4) * m * n, 256) + 256 : 256;
}

extern "C" int bz_glu(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w, int64_t m, int64_t n, int64_t k,
                      int dtype, int act, void* h, int64_t ld_h, float* preact, void* workspace, size_t workspace_bytes, void* stream) {
    const int st = check(x, ld_x, w_gate, w_up, ld_w, m, n, k, dtype, act);
    if (st != BZ_OK) return st;
    if (m == 0 || n == 0) return BZ_OK;
    if (h == nullptr || (m > 1 && ld_h < n) || (reinterpret_cast<uintptr_t>(h) & 1) || !aligned16(preact)) return BZ_ERR_INVALID_ARG;
    if (!(laid_out(x, ld_x, m) && laid_out(w_gate, ld_w, n) && laid_out(w_up, ld_w, n)) && k > 0 &&
        (workspace == nullptr || !aligned256(workspace) || workspace_bytes < bz_glu_workspace_bytes(m, n, k, dtype, 0)))
        return BZ_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
#define BZ_CALL(T, A) forward<T, A>(x, ld_x, w_gate, w_up, ld_w, m, n, k, h, ld_h, preact, s)
    BZ_GLU_SWITCH(BZ_CALL)
#undef BZ_CALL
}

extern "C" int bz_glu_backward(const void* x, int64_t ld_x, const void* w_gate, const void* w_up, int64_t ld_w, const float* preact,
                               const void* dh, int64_t ld_dh, int64_t m, int64_t n, int64_t k, int dtype, int act, void* dx, int64_t ld_dx,
                               void* dw_gate, void* dw_up, int64_t ld_dw, int grad_dtype, void* workspace, size_t workspace_bytes,
                               void* stream) {
    const int st = check(x, ld_x, w_gate, w_up, ld_w, m, n, k, dtype, act);
    if (st != BZ_OK) return st;
    if ((grad_dtype != dtype && grad_dtype != BZ_F32) || (dw_gate == nullptr) != (dw_up == nullptr)) return BZ_ERR_INVALID_ARG;
    if (k == 0 || (m == 0 && n == 0)) return BZ_OK;
    const uintptr_t grads = reinterpret_cast<uintptr_t>(dw_gate) | reinterpret_cast<uintptr_t>(dw_up);
    if (dx == nullptr && dw_gate == nullptr) return BZ_ERR_INVALID_ARG;
    if ((m > 1 && ld_dh < n) || (dx != nullptr && m > 1 && ld_dx < k) || (dw_gate != nullptr && n > 1 && ld_dw < k)) return BZ_ERR_INVALID_ARG;
    if (m > 0 && n > 0 && (preact == nullptr || dh == nullptr)) return BZ_ERR_INVALID_ARG;
    if (!aligned16(preact) || ((reinterpret_cast<uintptr_t>(dh) | reinterpret_cast<uintptr_t>(dx)) & 1) || grads % (grad_dtype == BZ_F32 ? 4 : 2))
        return BZ_ERR_INVALID_ARG;
    if (workspace == nullptr || !aligned256(workspace) || workspace_bytes < bz_glu_workspace_bytes(m, n, k, dtype, 1)) return BZ_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
#define BZ_CALL(T, A) \
    backward<T, A>(x, ld_x, w_gate, w_up, ld_w, preact, dh, ld_dh, m, n, k, dx, ld_dx, dw_gate, dw_up, ld_dw, grad_dtype, workspace, s)
    BZ_GLU_SWITCH(BZ_CALL)
#undef BZ_CALL
}
