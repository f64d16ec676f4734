// What the kernels that work on the rollout's side share (rr_products.cu, rr_cache.cu,
// rr_attend.cu): element types, dependent launches, checks of arguments.  Not part of
// the public ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "rr_internal.h"

namespace {

// ---------------------------------------------------------------------------
// 16-bit element types
// ---------------------------------------------------------------------------

struct BF16 {
    static __device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float(uint32_t(b) << 16); }
    static __device__ __forceinline__ uint16_t round(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
    static constexpr uint16_t kNaN = 0x7FC0;
};
struct F16 {
    static __device__ __forceinline__ float widen(uint16_t b) { return __half2float(__ushort_as_half(b)); }
    static __device__ __forceinline__ uint16_t round(float f) { return __half_as_ushort(__float2half_rn(f)); }
    static constexpr uint16_t kNaN = 0x7E00;
};

// Programmatic dependent launch: the next kernel on the stream may be scheduled
// while this one runs; each waits for the kernels before it to complete before it
// touches memory.
__device__ __forceinline__ void after_previous() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

inline rr_status cuda_fail(cudaError_t e, const char* what) {
    return rr_fail(RR_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

#define RR_CUDA(call)                                   \
    do {                                                \
        cudaError_t e_ = (call);                        \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call); \
    } while (0)

#define RR_TRY(call)                     \
    do {                                 \
        rr_status s_ = (call);           \
        if (s_ != RR_OK) return s_;      \
    } while (0)

// Memory of device `dev`, the current one, `align`ed.
inline rr_status check_device(int dev, const void* p, size_t align, const char* what) {
    if (!p || (uintptr_t)p % align) return rr_fail(RR_EINVAL, "%s is NULL or not %zu-byte aligned", what, align);
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return rr_fail(RR_EINVAL, "%s is not memory of this GPU", what);
    }
    if (at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev)) return RR_OK;
    return rr_fail(RR_EINVAL, "%s is not memory of this GPU", what);
}

constexpr int kMaxDevices = 16;

inline rr_status current_device(int* dev) {
    RR_CUDA(cudaGetDevice(dev));
    if (*dev < 0 || *dev >= kMaxDevices) return rr_fail(RR_EINVAL, "device %d: 0..%d", *dev, kMaxDevices - 1);
    return RR_OK;
}

// Lets a kernel have `smem` bytes of dynamic shared memory, once per kernel and device
// (`done`: its own bits, one a device).
template <class K>
cudaError_t allow_smem(K* kernel, int smem, int dev, std::atomic<uint32_t>* done) {
    if (done->load(std::memory_order_relaxed) >> dev & 1) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) done->fetch_or(1u << dev, std::memory_order_relaxed);
    return e;
}

// A launch that may be scheduled while the one before it on the stream runs.
template <class... Params, class... Args>
cudaError_t launch_after(void (*kernel)(Params...), unsigned grid, int threads, cudaStream_t stream, Args... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(unsigned(threads));
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

}  // namespace
