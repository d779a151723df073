// Attention of drafted trees over a cache in 4 bits for many query rows: launches of the tcgen05 kernel (tree_attention_tc.cuh).
#include "tree_attention_tc.cuh"

namespace sd {
namespace {

template <typename T, int DP, int TILES>
__global__ void __launch_bounds__(32 * TcAttn<DP, TILES, true>::WARPS, 1) k_fp4_tc(Fp4Attn a) { ta_tc<T, DP, TILES, true>(nullptr, a); }

// Shared memory of a CTA: besides what the sizes fix, a mask row for each node that a tile of `rows` may have, what anyone sees, and the sequences that are cut.
constexpr int most(int tiles) { return 232448 - (tiles == 1 ? 2048 : 1024); }          // (the kernel's static part)
template <int DP, int TILES> constexpr int bytes(int T, int group, int B) {
    const int nodes = (TILES * TC_ROWS - 1) / group + 2, words = (T + 31) / 32;
    return TcAttn<DP, TILES, true>::BYTES + 1024 + ((nodes < T ? nodes : T) + 1) * words * 4 + B * 16;
}
static_assert(bytes<128, 1>(1024, 1, TA_MAX_B) <= most(1) && bytes<64, 1>(1024, 1, TA_MAX_B) <= most(1), "tiles of 128 rows take all trees");

template <typename T, int DP, int TILES>
cudaError_t run(const Fp4Attn& a, int grid, cudaStream_t st) {
    if (const cudaError_t e = op_allow<k_fp4_tc<T, DP, TILES>>(most(TILES))) return e;
    return op_launch(k_fp4_tc<T, DP, TILES>, dim3(ta_grid(a, grid, TA_SMS)), 32 * TcAttn<DP, TILES, true>::WARPS, bytes<DP, TILES>(a.T, a.group, a.direct == 1 ? 0 : a.B), st, 1, a);
}
template <typename T>
cudaError_t pick(const Fp4Attn& a, int rows, int grid, cudaStream_t st) {
    if (a.dim > 64) return rows == 128 ? run<T, 128, 1>(a, grid, st) : run<T, 128, 2>(a, grid, st);
    return rows == 128 ? run<T, 64, 1>(a, grid, st) : run<T, 64, 2>(a, grid, st);
}
}  // namespace

bool fp4_tc_fits(int dim, int rows, int T, int group) {
    return rows == 128 || (dim > 64 ? bytes<128, 2>(T, group, TA_MAX_B) : bytes<64, 2>(T, group, TA_MAX_B)) <= most(2);
}
cudaError_t fp4_tc(const Fp4Attn& a, int dtype, int rows, int grid, cudaStream_t st) {
    return dtype == SPECDEC_DTYPE_BF16 ? pick<__nv_bfloat16>(a, rows, grid, st) : pick<__half>(a, rows, grid, st);
}

}  // namespace sd
