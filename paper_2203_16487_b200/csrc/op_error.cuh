// What the operators that take no handle share: errors (the message waits for specdec_last_error(NULL) on the calling thread) and launches.
#pragma once
#include <cuda_runtime.h>

#include <atomic>

#include "../../include/specdec.h"

namespace sd {
int op_fail(int code, const char* who, const char* why) noexcept;      // returns code
inline int op_bad(const char* who, const char* why) { return op_fail(SPECDEC_ERR_INVALID_ARG, who, why); }
inline int op_elem_bytes(int dtype) { return dtype == SPECDEC_DTYPE_F32 ? 4 : dtype == SPECDEC_DTYPE_BF16 || dtype == SPECDEC_DTYPE_F16 ? 2 : 0; }
inline long long op_stride(long long stride, long long extent) { return extent > 1 ? stride : 0; }     // (a dimension of 1 may come with any)
// Launches behind one another: a kernel that begins with op_begin() is set up while its predecessor in the stream still runs, and waits for it there.  What such a kernel
// reads comes by pointers without __restrict__: the compiler may fetch what those lead to ahead of the wait.
// (cluster > 1: CTAs of a cluster.)
template <typename... P, typename... A>
inline cudaError_t op_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization; at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension; at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
// Lets `Kernel` have up to `bytes` of dynamic shared memory on the current device: set once for each device, as the limit belongs to both (beyond 64 devices: every time).  A
// refusal is not kept.
template <auto* Kernel> inline cudaError_t op_allow(int bytes) {
    static std::atomic<unsigned long long> done{0};
    int d;
    if (const cudaError_t e = cudaGetDevice(&d)) return e;
    const unsigned long long bit = d < 64 ? 1ull << d : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}
#ifdef __CUDACC__
__device__ __forceinline__ void op_begin() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif
inline int op_done(const char* who, cudaError_t e) {
    if (e == cudaSuccess) return SPECDEC_OK;
    cudaGetLastError();                                   // (not left for an unrelated call to find)
    return op_fail(SPECDEC_ERR_CUDA, who, cudaGetErrorString(e));
}
}  // namespace sd
