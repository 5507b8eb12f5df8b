// mbarrier and TMA (cp.async.bulk.tensor) primitives for the staged kernels, and the host lookup of
// the driver's tensor-map encoder.  Every wait is bounded; every load is a plain per-CTA load.
#pragma once

#include <cuda.h>

#include "bz_common.cuh"

namespace bz {

constexpr uint32_t kSpinLimit = 1u << 20;  // try_wait attempts before a wait is declared dead


__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Bounded wait for the phase with the given parity.  Returns false if the limit ran out.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity) {
    const uint32_t addr = smem_u32(bar);
    for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
        uint32_t done;
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
            "selp.u32 %0, 1, 0, p;\n"
            "}\n"
            : "=r"(done)
            : "r"(addr), "r"(parity)
            : "memory");
        if (done) return true;
    }
    return false;
}

// Orders this thread's ordinary accesses to shared memory before accesses by the asynchronous proxy (bulk copies, the
// tensor core's reads) that follow.
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// The warp's arrival for a stage that it has read with ordinary loads and that a bulk copy will refill.  The copy writes by
// the asynchronous proxy, and an arrival alone does not hold it back behind loads that are still on their way: shared loads
// queue behind misses of global ones, and one call of a million (24 rows of 2048, 5461 units) multiplied pieces of a
// later group's weights.  So each lane fences first (20.4 -> 21.5 us there, from memory; the other rings within 1 %).
__device__ __forceinline__ void release_stage(uint64_t* empty) {
    fence_async_smem();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(empty);
}

__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(smem_dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// ---- host side ----------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

template <typename F> F driver_entry(const char* name) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint(name, &p, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess)
        return reinterpret_cast<F>(p);
    (void)cudaGetLastError();
    return nullptr;
}

// The encoder needs a current context, and a thread that has made no call of the runtime has none yet: choosing the
// device that is chosen already makes its context current.  A context that the caller has made current stays.
inline void bind_context() {
    static const auto current = driver_entry<CUresult (*)(CUcontext*)>("cuCtxGetCurrent");
    CUcontext context = nullptr;
    int device;
    if (current == nullptr || current(&context) != CUDA_SUCCESS || context != nullptr) return;
    if (cudaGetDevice(&device) != cudaSuccess || cudaSetDevice(device) != cudaSuccess) (void)cudaGetLastError();
}

// Looked up once; a second thread's first call waits for it.
inline EncodeTiledFn encode_tiled() {
    static const EncodeTiledFn fn = driver_entry<EncodeTiledFn>("cuTensorMapEncodeTiled");
    if (fn != nullptr) bind_context();
    return fn;
}

}  // namespace bz
