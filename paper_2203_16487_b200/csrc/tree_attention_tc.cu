// Attention of drafted trees over the paged cache for 16-bit types and many query rows: launches of the tcgen05 kernel (tree_attention_tc.cuh).
#include "tree_attention_tc.cuh"

namespace sd {
namespace {

template <typename T, int DP, int TILES>
__global__ void __launch_bounds__(32 * TcAttn<DP, TILES, false>::WARPS, 1) k_ta_tc(const __grid_constant__ CUtensorMap tm, TreeAttn a) { ta_tc<T, DP, TILES, false>(&tm, a); }

template <typename T, int DP, int TILES>
cudaError_t run(const CUtensorMap& tm, const TreeAttn& a, int grid, cudaStream_t st) {
    constexpr int BYTES = TcAttn<DP, TILES, false>::BYTES + 1024, MOST = BYTES + (TILES * TC_ROWS + 1) * (TILES == 2 && DP > 64 ? TA_WIDE_T / 32 : 32) * 4 + TA_MAX_B * 16;
    static_assert(MOST <= 232448 - (TILES == 1 ? 2048 : 1024), "shared memory of an SM");
    if (const cudaError_t e = op_allow<k_ta_tc<T, DP, TILES>>(MOST)) return e;
    return op_launch(k_ta_tc<T, DP, TILES>, dim3(ta_grid(a, grid, TA_SMS)), 32 * TcAttn<DP, TILES, false>::WARPS, BYTES + (TILES * TC_ROWS + 1) * a.words * 4 + (a.direct == 1 ? 0 : a.B) * 16, st, 1, tm, a);
}
template <typename T>
cudaError_t pick(const CUtensorMap& tm, const TreeAttn& a, int rows, int grid, cudaStream_t st) {
    if (a.dim > 64) return rows == 128 ? run<T, 128, 1>(tm, a, grid, st) : run<T, 128, 2>(tm, a, grid, st);
    return rows == 128 ? run<T, 64, 1>(tm, a, grid, st) : run<T, 64, 2>(tm, a, grid, st);
}

}  // namespace

cudaError_t ta_tc(const CUtensorMap& tm, const TreeAttn& a, int dtype, int rows, int grid, cudaStream_t st) {
    return dtype == SPECDEC_DTYPE_BF16 ? pick<__nv_bfloat16>(tm, a, rows, grid, st) : pick<__half>(tm, a, rows, grid, st);
}

}  // namespace sd
