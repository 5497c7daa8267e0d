// serving.cuh -- what the paged beam-search operators (paged.cu, beam.cu,
// chunk_attention*.cu) share: argument errors, element types.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "common.cuh"
#include "kernels.cuh"
#include "mtp.h"

namespace mtp {

inline int invalid(const char* fmt, ...) {
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    return report_error(MTP_ERR_INVALID, msg);
}
inline int cuda_status(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return MTP_OK;
    char msg[256];
    snprintf(msg, sizeof(msg), "%s: %s", what, cudaGetErrorString(e));
    return report_error(MTP_ERR_CUDA, msg);
}
// The body of a C entry point: no C++ exception leaves it.
template <class F>
int guarded(F body) noexcept {
    try {
        clear_error();
        return body();
    } catch (...) {
        return MTP_ERR_CUDA;
    }
}

// Enqueue a kernel, in clusters of `cluster` CTAs.  All of these operators' kernels are launched programmatically:
// they may be placed while the kernel before them in the stream ends, and touch global memory only
// after pdl_wait, by plain loads (one that says its data never change could be moved before it).
template <class... P>
cudaError_t launch_ex(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, int cluster, P... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64 || p == 128; }

// Element types of two bytes as raw bits: to and from fp32, rounded to nearest even.
struct Bf16 {
    static __device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
};
struct F16 {
    static __device__ __forceinline__ float to_float(uint16_t x) { return __half2float(__ushort_as_half(x)); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const __half2 p = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&p);
    }
};

}  // namespace mtp
