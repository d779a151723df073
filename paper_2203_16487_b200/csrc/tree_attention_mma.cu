// Attention of drafted trees over the paged cache for 16-bit types and few query rows: keys by TMA, mma.sync (contract: specdec.h, work: tree_attention.cuh).
//
// CTA = one item: WM x WK consumer warps and one that loads.  A block of 64 keys is a stage of a ring: one TMA box a page, keys and values each in column halves of
// 128 swizzled bytes a row.  Warp (wm, wk) takes 16 rows and every WK-th block: scores (m16n8k16, fp32), running maximum and sum in registers, probabilities (rounded
// to the type; the sum keeps the unrounded ones) straight from the score registers into the second product.  The WK groups' partial outputs
// meet in shared memory at the end.
//
// Few rows: HBM bounds it, so what counts is bytes in flight (a ring of NS stages of 16 or 32 KB an SM) and that nothing but the boxes' addresses passes through
// registers on the way.  A box needs its page number: the loading warp's lanes read a block's numbers together.
#include "tree_attention.cuh"

namespace sd {
namespace {

// NS is a multiple of WK: a stage always serves the same group, which so sees every one of its phases.
template <typename T, int DP, int WM, int WK, int NS>
__global__ void __launch_bounds__(32 * (WM * WK + 1), DP > 64 ? 2 : 3) k_ta_tma(const __grid_constant__ CUtensorMap tm, TreeAttn a) {
    static_assert(NS % WK == 0, "a stage serves one group");
    constexpr int TM_WARPS = WM * WK, ROWS = 16 * WM, KT = TA_BLOCK, HALVES = DP / 64;
    constexpr int SIDE = KT * DP * 2, STAGE = 2 * SIDE;
    extern __shared__ __align__(1024) char ta_smem[];
    __shared__ __align__(8) uint64_t bars[2 * NS];
    __shared__ int abort_flag;
    char* ring = ta_smem + (1024 - (smem_u32(ta_smem) & 1023)) % 1024;
    uint32_t* any = (uint32_t*)(ring + NS * STAGE);
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t full = smem_u32(bars), empty = full + NS * 8;
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) { mbar_init(full + i * 8, 1); mbar_init(empty + i * 8, WM); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch_map(&tm);
    }
    const Item it = ta_item(a, (int*)ring);
    if (it.b < 0) return;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // ta_item's use of the ring, ahead of the boxes
    const SeqKeys s = ta_keys(a, it.b);
    const int r0 = it.tile * ROWS, all_rows = a.T * a.group, t0 = r0 / a.group;
    ta_load_masks(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
    const int k_begin = it.split * it.per * KT, k_end = min(s.keys, (int)min((long long)(it.split + 1) * it.per * KT, (long long)s.keys));
    const int blocks = max(0, (k_end - k_begin + KT - 1) / KT);

    if (warp == TM_WARPS) {                               // loads
        const int page = 1 << a.page_shift, rows = min(page, KT), n_pages = KT / rows;
        const int* table = a.table + (long long)s.seq * a.max_pages;
        auto page_of = [&](int j) {                       // this lane's page of block j: out of range where there is none
            const int key = k_begin + j * KT + lane * rows, i = key >> a.page_shift;
            int p = -1;
            if (lane < n_pages && key < k_end && i < a.max_pages) p = table[i];
            return (unsigned)p < (unsigned)a.n_pages ? p : a.n_pages;
        };
        int p = blocks ? page_of(0) : 0;
        for (int j = 0; j < blocks; ++j) {
            const int st = j % NS, key = k_begin + j * KT + lane * rows;
            const int cur = p;
            if (j + 1 < blocks) p = page_of(j + 1);
            if (j >= NS && !mbar_wait_warp(empty + st * 8, (j / NS - 1) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) break;
            const bool mine = lane < n_pages && key < k_end;
            const unsigned boxes = __popc(__ballot_sync(0xffffffffu, mine));
            if (lane == 0) mbar_expect_tx(full + st * 8, boxes * rows * 128 * HALVES * 2);
            __syncwarp();
            if (mine) {
                const uint32_t d = smem_u32(ring + st * STAGE) + lane * rows * 128;
#pragma unroll
                for (int side = 0; side < 2; ++side)
#pragma unroll
                    for (int hf = 0; hf < HALVES; ++hf)
                        ta_box(d + side * SIDE + hf * KT * 128, &tm, hf * 64, it.h, key & (page - 1), cur, side, full + st * 8);
            }
        }
        __syncthreads();
        if constexpr (WK > 1) __syncthreads();
        return;
    }

    const int wm = warp % WM, wk = warp / WM;
    const int ra = wm * 16 + (lane >> 2), rb = ra + 8;
    const int ga = r0 + ra, gb = r0 + rb, ta = ga / a.group, tb = gb / a.group;
    const bool live_a = ga < all_rows && ta < s.nodes, live_b = gb < all_rows && tb < s.nodes;
    const uint32_t* mask_a = mask + (live_a ? ta - t0 : 0) * a.words;
    const uint32_t* mask_b = mask + (live_b ? tb - t0 : 0) * a.words;
    uint32_t qf[DP / 16][4];                              // the rows as fragments, straight from memory
    {
        const char* qa = a.q + it.b * a.q_sb + ta * a.q_st + (it.h * a.group + ga % a.group) * a.q_sh + (lane & 3) * 4;
        const char* qb = a.q + it.b * a.q_sb + tb * a.q_st + (it.h * a.group + gb % a.group) * a.q_sh + (lane & 3) * 4;
        auto two = [&](const char* p) -> uint32_t {
            if (a.q_vec) return *reinterpret_cast<const uint32_t*>(p);
            return reinterpret_cast<const unsigned short*>(p)[0] | (uint32_t)reinterpret_cast<const unsigned short*>(p)[1] << 16;
        };
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk) {
            const bool lo = kk * 16 < a.dim, hi = kk * 16 + 8 < a.dim;
            qf[kk][0] = live_a && lo ? two(qa + kk * 32) : 0u;
            qf[kk][1] = live_b && lo ? two(qb + kk * 32) : 0u;
            qf[kk][2] = live_a && hi ? two(qa + kk * 32 + 16) : 0u;
            qf[kk][3] = live_b && hi ? two(qb + kk * 32 + 16) : 0u;
        }
    }
    TaRows<T, DP> rows;
    rows.clear();
    for (int j = wk; j < blocks; j += WK) {
        const int st = j % NS, k0 = k_begin + j * KT;
        if (!mbar_wait_warp(full + st * 8, (j / NS) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) break;
        const uint32_t ks = smem_u32(ring + st * STAGE), vs = ks + SIDE;
        const bool tail = k0 + KT > s.len;                // nodes, or what is behind the last key
        if (tail) {                                       // values that no query sees: whatever is in them is multiplied by 0
            for (int r = wm * (KT / WM); r < (wm + 1) * (KT / WM); ++r)
                if (k0 + r >= k_end || !ta_seen(any, s, k0 + r))
                    if (lane < DP / 8) *reinterpret_cast<uint4*>(ring + st * STAGE + SIDE + (lane >> 3) * KT * 128 + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
            if constexpr (WM == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(1 + wk), "n"(32 * WM) : "memory");
        }
        rows.block(qf, k0, s.len, a.scale, a.words, live_a ? mask_a : nullptr, live_b ? mask_b : nullptr,
                   [&](int r, int c) { return ks + (c >> 3) * KT * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4); },
                   [&](int r, int c) { return vs + (c >> 3) * KT * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4); });
        if (tail) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");         // the zeros, ahead of the stage's next boxes
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + st * 8);
    }
    rows.finish(live_a, live_b);
    __syncthreads();                                      // the ring is free
    if constexpr (WK > 1) {
        constexpr int RP = TaRows<T, DP>::RP;
        float* red = reinterpret_cast<float*>(ring);      // [WK - 1][ROWS][RP], then [WK - 1][ROWS] (maximum, sum)
        float2* red_ml = reinterpret_cast<float2*>(red + (WK - 1) * ROWS * RP);
        static_assert((WK - 1) * ROWS * (RP * 4 + 8) <= NS * STAGE, "partial outputs fit the ring");
        if (wk > 0) rows.leave(red + (wk - 1) * ROWS * RP, red_ml + (wk - 1) * ROWS, ra);
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int g = 0; g < WK - 1; ++g) rows.join(red + g * ROWS * RP, red_ml + g * ROWS, ra);
    }
    rows.store(a, it, r0, ra, ROWS);
}

template <typename T, int DP, int WM, int WK, int NS>
cudaError_t run(const CUtensorMap& tm, const TreeAttn& a, int grid, cudaStream_t st) {
    constexpr int RING = NS * 2 * TA_BLOCK * DP * 2;
    static const cudaError_t attr = cudaFuncSetAttribute(k_ta_tma<T, DP, WM, WK, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize, RING + 1024 + (16 * WM + 1) * 32 * 4);
    if (attr != cudaSuccess) return attr;
    k_ta_tma<T, DP, WM, WK, NS><<<grid, 32 * (WM * WK + 1), RING + 1024 + (16 * WM + 1) * a.words * 4, st>>>(tm, a);
    return cudaGetLastError();
}
template <typename T>
cudaError_t pick(const CUtensorMap& tm, const TreeAttn& a, int rows, int grid, cudaStream_t st) {
    if (a.dim > 64) return rows == 16 ? run<T, 128, 1, 3, 3>(tm, a, grid, st) : rows == 32 ? run<T, 128, 2, 1, 3>(tm, a, grid, st) : run<T, 128, 4, 1, 3>(tm, a, grid, st);
    return rows == 16 ? run<T, 64, 1, 4, 4>(tm, a, grid, st) : rows == 32 ? run<T, 64, 2, 2, 4>(tm, a, grid, st) : run<T, 64, 4, 1, 3>(tm, a, grid, st);
}

}  // namespace

cudaError_t ta_tma_mma(const CUtensorMap& tm, const TreeAttn& a, int dtype, int rows, int grid, cudaStream_t st) {
    return dtype == SPECDEC_DTYPE_BF16 ? pick<__nv_bfloat16>(tm, a, rows, grid, st) : pick<__half>(tm, a, rows, grid, st);
}

}  // namespace sd
