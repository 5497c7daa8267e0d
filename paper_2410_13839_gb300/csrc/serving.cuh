// serving.cuh -- what the operators of the caller's own paged cache (paged.cu, beam.cu,
// chunk_attention*.cu, rotary.cu, key_weights*.cu, verify.cu, evict.cu) share: argument
// errors, launches, element types.
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

// Enqueue a kernel, clusters of `cluster` CTAs.  (The 48 KB that a kernel has without asking hold its static shared memory
// too: any size is asked for.)
template <class... P>
cudaError_t launch(void (*kern)(P...), int grid, int threads, size_t smem, int cluster, cudaStream_t s, P... args) {
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), smem);
    return e == cudaSuccess ? launch_ex(kern, dim3(grid), threads, smem, s, cluster, args...) : e;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64 || p == 128; }
constexpr int PG_MAX_PAGES = 1 << 22;
inline int log2_of(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7; }

inline int check_pool(const char* what, int n_pages, int layers, int layer, int n_kv_heads, int head_dim, int page_size) {
    if (n_pages < 1 || n_pages > PG_MAX_PAGES || layers < 1 || layer < 0 || layer >= layers || n_kv_heads < 1 ||
        n_kv_heads > 1024 || head_dim < 8 || head_dim > 256 || head_dim % 8 || !page_size_ok(page_size))
        return invalid("%s: invalid pool (pages %d, layers %d, layer %d, heads %d, head_dim %d, page_size %d)", what,
                       n_pages, layers, layer, n_kv_heads, head_dim, page_size);
    return MTP_OK;
}

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
