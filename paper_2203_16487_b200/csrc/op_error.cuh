// Errors of the operators that take no handle: the message waits for specdec_last_error(NULL) on the calling thread.
#pragma once
#include <cuda_runtime.h>

#include "../../include/specdec.h"

namespace sd {
int op_fail(int code, const char* who, const char* why) noexcept;      // returns code
inline int op_bad(const char* who, const char* why) { return op_fail(SPECDEC_ERR_INVALID_ARG, who, why); }
// What became of the launches since the last call.
inline int op_launched(const char* who) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SPECDEC_OK : op_fail(SPECDEC_ERR_CUDA, who, cudaGetErrorString(e));
}
inline int op_elem_bytes(int dtype) { return dtype == SPECDEC_DTYPE_F32 ? 4 : dtype == SPECDEC_DTYPE_BF16 || dtype == SPECDEC_DTYPE_F16 ? 2 : 0; }
}  // namespace sd
