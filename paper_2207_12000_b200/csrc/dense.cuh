// What the operators beside the aggregation share: element types, wide accesses, launches that follow one another.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <utility>

#include "gnnpre_internal.cuh"

namespace gnnpre {

inline int64_t dtype_bytes(int32_t dtype) { return dtype == GNNPRE_F32 ? 4 : 2; }
inline bool is_dtype(int32_t dtype) { return dtype == GNNPRE_F32 || dtype == GNNPRE_BF16 || dtype == GNNPRE_F16; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// One rounding, to nearest.
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// E neighbouring elements, read and written by accesses of up to 16 bytes.
template <typename T, int E>
struct alignas(E * sizeof(T) < 16 ? E * sizeof(T) : 16) Vec {
    T v[E];
};

// Elements per access that `bytes`-aligned addresses allow, at most `most` (a power of two).
inline int elements_per_access(uintptr_t addresses, int64_t es, int most) {
    int e = most;
    while (e > 1 && addresses % (uintptr_t)(e * es) != 0) e /= 2;
    return e;
}

constexpr int kMaxDevices = 64;

// The current device's SMs; UNSUPPORTED_ARCH on a device that is not of compute capability 10.x.
int device_sms(int* out);

// Launches a kernel whose CTAs may start when those of the kernel before it on the stream have left: it waits
// (wait_previous_kernel) before it reads or writes anything that kernel touches.
template <typename... Params, typename... Args>
int launch_after(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, bool overlap, cudaStream_t st, Args&&... args) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = overlap ? 1 : 0;
    GNNPRE_CUDA(cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...));
    return GNNPRE_OK;
}

__device__ __forceinline__ void wait_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Whether [rows, width] matrices of elements of es bytes at a and b (pitches lda, ldb in elements) share a byte.  Column views of
// one wider buffer (equal pitch in bytes, disjoint columns) do not.
inline bool arrays_overlap(const void* a, int64_t rows_a, int64_t width_a, int64_t lda, int64_t es_a, const void* b, int64_t rows_b,
                           int64_t width_b, int64_t ldb, int64_t es_b) {
    if (rows_a < 1 || rows_b < 1 || width_a < 1 || width_b < 1) return false;
    const intptr_t pa = reinterpret_cast<intptr_t>(a), pb = reinterpret_cast<intptr_t>(b);
    const intptr_t wa = width_a * es_a, wb = width_b * es_b, ta = lda * es_a, tb = ldb * es_b;
    if (pa + (rows_a - 1) * ta + wa <= pb || pb + (rows_b - 1) * tb + wb <= pa) return false;
    if (ta != tb || ta < 1) return true;
    intptr_t r = (pb - pa) % ta;
    if (r < 0) r += ta;
    return r < wa || r > ta - wb;
}

}  // namespace gnnpre
