// Attention of drafted trees over a cache in 4 bits: what its kernels share (contract: specdec.h, format: fp4.cuh, work: tree_attention.cuh).
#pragma once
#include <type_traits>

#include "fp4.cuh"
#include "tree_attention.cuh"

namespace sd {

struct Fp4Attn : TreeAttn {                               // k, v, s_page, s_head: the codes'
    const char* ks; const char* vs; long long c_page, c_head;                          // scales
    const float* unit_k; const float* unit_v;             // [K/V head] or null
};

// A block of 64 keys of one head as it lies in memory: keys, then values, of each the codes and their scales.
template <int D> struct Fp4Stage {
    static constexpr int CODES = TA_BLOCK * D / 2, HALF = CODES + TA_BLOCK * D / 16, BYTES = 2 * HALF;
};
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// The power of two that takes a row's largest number into [2^14, 2^15) is 2^(14 - e); 1 where there is none, or an infinite one.  Returns 14 - e.
__device__ __forceinline__ int row_shift(float top) {
    if (!(top > 0.f) || !(top < INFINITY)) return 0;
    const int e = (int)(__float_as_uint(top) >> 23) - 127;
    return 14 - max(e, -100);
}
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // -126 .. 127

bool fp4_tc_fits(int dim, int rows, int T, int group);                                    // whether the masks of a tile of 128 or 256 rows fit beside the rest (with 128 they always do)
cudaError_t fp4_tc(const Fp4Attn& a, int dtype, int rows, int grid, cudaStream_t st);                                     // tiles of 128, 256 rows

}  // namespace sd
