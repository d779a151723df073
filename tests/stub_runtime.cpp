// A CUDA runtime of two devices without any, for the host side of the operators as it was built (their object files are linked against this): what is set, what is
// launched, and on which device.  A launch is accepted only as the real ones are: with no more dynamic shared memory than was allowed for that kernel on that device.
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdio>
#include <map>
#include <string>
#include <utility>

#include "../include/specdec.h"

static int device = 0, refuse_once = 0, launches = 0, settings = 0, wrong = 0;
static std::map<std::pair<int, const void*>, int> allowed;
static std::string said;

namespace sd {
int op_fail(int code, const char* who, const char* why) noexcept { said = std::string(who) + ": " + why; return code; }
}

extern "C" {
void** __cudaRegisterFatBinary(void*) { static void* p; return &p; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { ++wrong; return cudaSuccess; }         // (operators launch by attributes)
cudaError_t __cudaGetKernel(cudaKernel_t* k, const void* f) { *k = (cudaKernel_t)f; return cudaSuccess; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { ++wrong; return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = device; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "refused"; }
cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute a, int v) {
    ++settings;
    if (refuse_once) { refuse_once = 0; return cudaErrorMemoryAllocation; }
    if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) allowed[{device, f}] = v;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**) {
    const auto at = allowed.find({device, f});
    if (c->dynamicSmemBytes > size_t(at == allowed.end() ? 48 * 1024 : at->second)) return cudaErrorInvalidValue;
    ++launches;
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int* n, const void*, int, size_t, unsigned) { *n = 2; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) { *n = 2; return cudaSuccess; }
static CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                       CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) { return CUDA_SUCCESS; }
cudaError_t cudaGetDriverEntryPoint(const char*, void** p, unsigned long long, cudaDriverEntryPointQueryResult* q) { *p = (void*)encode; *q = cudaDriverEntryPointSuccess; return cudaSuccess; }
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** p, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    *p = (void*)encode; *q = cudaDriverEntryPointSuccess; return cudaSuccess;
}
}

// One call of every kernel that may need more than 48 KB.  Returns those refused.
static int calls(bool print) {
    int bad = 0;
    auto is = [&](const char* what, int rc) { if (rc) { ++bad; if (print) fprintf(stderr, "device %d: %s %d (%s)\n", device, what, rc, said.c_str()); } };
    int* i = (int*)64;
    char name[64];
    is("ancestors", specdec_tree_ancestors(i, nullptr, 1, 1024, (uint32_t*)64, i, nullptr));
    for (int dtype = 0; dtype < 3; ++dtype) {
        for (int V : {30000, 50265, 60000, 131072, 262144})
            for (int rows : {1, 40, 300}) {
                sprintf(name, "sample %d %d x %d", dtype, rows, V);
                is(name, specdec_sample((void*)4096, dtype, V, rows, V, (float*)64, nullptr, nullptr, nullptr, nullptr, 1, i, nullptr, nullptr));
            }
        for (int dim : {64, 128})
            for (int page : {4, 64})
                for (int T : {1, 2, 3, 4, 20, 60, 100, 300, 1024})
                    for (int B : {1, 40, 200}) {
                        specdec_cache c = {(void*)4096, dtype, 1, 8, dim, 1 << 16, page, B, 8192 / page, 0, 1 << 24, 8 * dim * page, 8 * dim, dim, i, i, i, i, i, i};
                        specdec_tree_attention_args a = {(void*)4096, (void*)4096, 8 * dim * T, 8 * dim, dim, 8 * dim * T, 8 * dim, dim, B, T, 8, 0, i, (uint32_t*)64, 0, nullptr, 4000, 0.1f,
                                                         (void*)4096, 1ll << 40};
                        sprintf(name, "attention %d %d x %d, %d wide, pages of %d", dtype, B, T, dim, page);
                        is(name, specdec_tree_attention(&c, &a, nullptr));
                    }
    }
    return bad;
}

int main() {
    const int first = calls(true), once = settings;
    device = 1;
    const int second = calls(true);
    printf("refused_on_the_first_device %d\nrefused_on_the_second_device %d\n", first, second);
    printf("settings_repeated %d\n", settings - 2 * once);
    const int before = settings;
    device = 0; calls(false);
    printf("settings_of_known_kernels %d\n", settings - before);
    device = 2; refuse_once = 1;                          // a device that refuses once is asked again
    const int refused = calls(false), again = calls(true);
    printf("not_refused_once %d\nrefused_after_a_failure %d\n", refused != 1, again);
    printf("wrong_launches %d\nno_launches %d\n", wrong, launches == 0);
}
