// Attention of drafted trees over the paged cache for 16-bit types and few query rows: keys by TMA, mma.sync (contract: specdec.h, work: tree_attention.cuh).
//
// CTA = WM x WK consumer warps and one that loads.  A block of 64 keys is a stage of a ring: one TMA box a page, keys and values each in column halves of
// 128 swizzled bytes a row.  Warp (wm, wk) takes 16 rows and every WK-th block: scores (m16n8k16, fp32), running maximum and sum in registers, probabilities (rounded
// to the type, as mma.sync takes them; the sum adds up the rounded ones) straight from the score registers into the second product.  The WK groups' partial outputs
// meet in shared memory at the end.
//
// Few rows: HBM bounds it, so what counts is bytes in flight (a ring of NS stages of 16 or 32 KB an SM) and that nothing but the boxes' addresses passes through
// registers on the way.  A box needs its page number: the loading warp's lanes read a block's numbers together.  2 x 1 query, 32/8 heads of 128, over 65,537 to
// 131,071 keys: 150 us with the merge, 6.5 TB/s; 8 x 1 query, 8 heads of 64, over 8000 in pages of 16: 34 us (both in a graph), 3.8 TB/s, of which start and merge are some 14.
// 64 rows over short sequences: the chain of a warp bounds it (scores, maximum, exponentials, second product: some 3000 clocks a block, 5500 more a sequence and head),
// of which 3 CTAs an SM overlap.  128 x 51 queries, 8 heads of 64, over 51 to 307 keys: 28 us in a graph, 55 TFLOP/s; 29.4 as a call among others.  (Four CTAs need 96 registers a thread, which spills
// 700 bytes; two CTAs of eight computing warps the same, 39 us.)
#include "tree_attention.cuh"

namespace sd {
namespace {

// Group wk has the stages wk, wk + WK, ... to itself and so waits for every phase of their barriers.
template <typename T, int DP, int WM, int WK, int NS>
__global__ void __launch_bounds__(32 * (WM * WK + 1), DP > 64 ? 2 : 3) k_ta_tma(const __grid_constant__ CUtensorMap tm, TreeAttn a) {
    static_assert(NS % WK == 0, "a stage serves one group");
    constexpr int TM_WARPS = WM * WK, NG = NS / WK, ROWS = 16 * WM, KT = TA_BLOCK, HALVES = DP / 64;
    constexpr int SIDE = KT * DP * 2, STAGE = 2 * SIDE;
    extern __shared__ __align__(1024) char ta_smem[];
    __shared__ __align__(8) uint64_t bars[2 * NS];
    __shared__ int abort_flag;
    char* ring = ta_smem + (1024 - (smem_u32(ta_smem) & 1023)) % 1024;
    int4* seqs = (int4*)(ring + NS * STAGE);              // [B] where sequences are cut
    uint32_t* any = (uint32_t*)(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + (a.words + 1) / 2 * 2;         // (8-byte aligned, as the partial results behind it are)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t full = smem_u32(bars), empty = full + NS * 8;
    if (warp == TM_WARPS && lane == 0) {
        for (int i = 0; i < NS; ++i) { mbar_init(full + i * 8, 1); mbar_init(empty + i * 8, WM); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch_map(&tm);
    }
    op_begin();
    TaWork work;
    work.begin(a, seqs);
    __syncthreads();

    if (warp == TM_WARPS) {                               // loads, running ahead into the next parts
        const int page = 1 << a.page_shift, box = min(page, KT), n_pages = KT / box;
        int count = 0;                                    // lane g: blocks that group g had in the parts before
        Part it, ahead;
        for (bool more = work.next(a, seqs, ahead); more;) {
            it = ahead;
            const int* table = a.table + (long long)it.s.seq * a.max_pages;
            auto page_of = [&](int j) {                   // this lane's page of block j: out of range where there is none
                const int key = it.k_begin + j * KT + lane * box, i = key >> a.page_shift;
                int p = -1;
                if (lane < n_pages && key < it.k_end && i < a.max_pages) p = table[i];
                return (unsigned)p < (unsigned)a.n_pages ? p : a.n_pages;
            };
            int p = it.blocks ? page_of(0) : 0;
            more = work.next(a, seqs, ahead);
            for (int j = 0; j < it.blocks; ++j) {
                const int g = j % WK, n = __shfl_sync(0xffffffffu, count, g) + j / WK, st = g + WK * (n % NG), key = it.k_begin + j * KT + lane * box, cur = p;
                if (j + 1 < it.blocks) p = page_of(j + 1);
                if (n >= NG && !mbar_wait_warp<true>(empty + st * 8, (n / NG - 1) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) return;
                const bool mine = lane < n_pages && key < it.k_end;
                const unsigned boxes = __popc(__ballot_sync(0xffffffffu, mine));
                if (lane == 0) mbar_expect_tx(full + st * 8, boxes * box * 128 * HALVES * 2);
                __syncwarp();
                if (mine) {
                    const uint32_t d = smem_u32(ring + st * STAGE) + lane * box * 128;
#pragma unroll
                    for (int side = 0; side < 2; ++side)
#pragma unroll
                        for (int hf = 0; hf < HALVES; ++hf)
                            ta_box(d + side * SIDE + hf * KT * 128, &tm, hf * 64, it.h, key & (page - 1), cur, side, full + st * 8);
                }
            }
            count += (it.blocks - lane + WK - 1) / WK;    // (lanes below WK)
        }
        return;
    }

    const int wm = warp % WM, wk = warp / WM, all_rows = a.T * a.group;
    auto consumers = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * TM_WARPS) : "memory"); };
    int count = 0;                                        // this group's blocks so far
    Part it, ahead;
    for (bool more = work.next(a, seqs, ahead, tid == 0); more;) {
        it = ahead;
        more = work.next(a, seqs, ahead, tid == 0);
        const SeqKeys& s = it.s;
        const int r0 = it.tile * ROWS, t0 = ta_node(a, r0);
        const int ra = wm * 16 + (lane >> 2), rb = ra + 8;
        const int ga = r0 + ra, gb = r0 + rb, ta = ta_node(a, ga), tb = ta_node(a, gb);
        const bool live_a = ga < all_rows && ta < s.nodes, live_b = gb < all_rows && tb < s.nodes;
        uint32_t qf[DP / 16][4];                          // the rows as fragments, straight from memory
        {
            const char* qa = a.q + it.b * a.q_sb + ta * a.q_st + (it.h * a.group + ga - ta * a.group) * a.q_sh + (lane & 3) * 4;
            const char* qb = a.q + it.b * a.q_sb + tb * a.q_st + (it.h * a.group + gb - tb * a.group) * a.q_sh + (lane & 3) * 4;
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
        // What the rows see, and the nodes that anyone sees.  Up to 64 nodes: in every warp's own registers (anyone: any query of the tree), so that no warp waits for
        // another; more: in shared memory.
        const bool own = a.words <= 2;
        uint32_t ma[2] = {0, 0}, mb[2] = {0, 0}, seen[2] = {0, 0};
        if (own) {
            const uint32_t* words = a.mask + it.b * a.mask_sb;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int left = s.nodes - w * 32;
                if (w >= a.words || left <= 0) break;
                const uint32_t cut = left < 32 ? (1u << left) - 1u : 0xffffffffu;
                uint32_t all = lane < s.nodes ? words[lane * a.words + w] : 0u;
                if (lane + 32 < s.nodes) all |= words[(lane + 32) * a.words + w];
                if (live_a) ma[w] = words[ta * a.words + w] & cut;
                if (live_b) mb[w] = words[tb * a.words + w] & cut;
                seen[w] = __reduce_or_sync(0xffffffffu, all) & cut;
            }
        } else {
            ta_load_masks<32 * TM_WARPS, 1>(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
        }
        const uint32_t* mask_a = mask + (live_a ? ta - t0 : 0) * a.words;
        const uint32_t* mask_b = mask + (live_b ? tb - t0 : 0) * a.words;
        auto window_a = [&](int base) { return !live_a ? 0u : own ? ta_window2(ma[0], ma[1], base) : ta_window(mask_a, a.words, base); };
        auto window_b = [&](int base) { return !live_b ? 0u : own ? ta_window2(mb[0], mb[1], base) : ta_window(mask_b, a.words, base); };
        TaRows<T, DP> rows;
        rows.clear();
        for (int j = wk; j < it.blocks; j += WK, ++count) {
            const int st = wk + WK * (count % NG), k0 = it.k_begin + j * KT;
            if (!mbar_wait_warp<true>(full + st * 8, (count / NG) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) {
                // The part is given up; but warps of the group that have not given up wait at the barriers of its blocks for this one.
                if constexpr (WM > 1)
#pragma unroll 1
                    for (; j < it.blocks; j += WK)
                        if (it.k_begin + j * KT + KT > s.len) asm volatile("bar.sync %0, %1;" ::"r"(2 + wk), "n"(32 * WM) : "memory");
                break;
            }
            const uint32_t ks = smem_u32(ring + st * STAGE), vs = ks + SIDE;
            const bool tail = k0 + KT > s.len;            // nodes, or what is behind the last key
            if (tail) {                                   // values that no query sees: whatever is in them is multiplied by 0
                ta_zero_unseen<KT / WM, HALVES>(ring + st * STAGE + SIDE, wm * (KT / WM), [&](int row) {
                    const int base = k0 + row - s.len;
                    return own ? ta_window2(seen[0], seen[1], base) : ta_window(any, a.words, base);
                });
                if constexpr (WM == 1) __syncwarp();
                else asm volatile("bar.sync %0, %1;" ::"r"(2 + wk), "n"(32 * WM) : "memory");
            }
            rows.block(qf, k0, s.len, a.scale, window_a, window_b,
                       [&](int r, int c) { return ks + (c >> 3) * KT * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4); },
                       [&](int r, int c) { return vs + (c >> 3) * KT * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4); });
            if (tail) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the zeros, ahead of the stage's next boxes
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + st * 8);
        }
        rows.finish(live_a, live_b);
        if constexpr (WK > 1) {                           // the groups' results meet in the first group
            constexpr int RP = TaRows<T, DP>::RP;
            float* red = reinterpret_cast<float*>(mask + ROWS * a.words);      // [ROWS][RP], then [ROWS] (maximum, sum): one group's at a time, so that two CTAs fit an SM
            float2* red_ml = reinterpret_cast<float2*>(red + ROWS * RP);
            for (int g = 1; g < WK; ++g) {
                if (wk == g) rows.leave(red, red_ml, ra);
                consumers();
                if (wk == 0) rows.join(red, red_ml, ra);
                if (g + 1 < WK) consumers();
            }
        }
        if (wk == 0) rows.store(a, it, r0, ra, ROWS);
        if (WK > 1 || !own) consumers();                  // masks and partial results may be overwritten
    }
}

template <typename T, int DP, int WM, int WK, int NS>
cudaError_t run(const CUtensorMap& tm, const TreeAttn& a, int grid, cudaStream_t st) {
    constexpr int ROWS = 16 * WM, RING = NS * 2 * TA_BLOCK * DP * 2, RED = (WK > 1) * ROWS * ((DP + 8) * 4 + 8);
    constexpr int MOST = RING + RED + 1024 + (ROWS + 2) * 32 * 4 + TA_MAX_B * 16;
    if (const cudaError_t e = op_allow<k_ta_tma<T, DP, WM, WK, NS>>(MOST)) return e;
    static std::atomic<int> found{0};                     // (the same on every device this code runs on)
    int per_sm = found.load(std::memory_order_relaxed);
    if (!per_sm) {
        if (const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k_ta_tma<T, DP, WM, WK, NS>, 32 * (WM * WK + 1), MOST)) return e;
        if (per_sm < 1) per_sm = 1;
        found.store(per_sm, std::memory_order_relaxed);
    }
    return op_launch(k_ta_tma<T, DP, WM, WK, NS>, dim3(ta_grid(a, grid, per_sm * TA_SMS)), 32 * (WM * WK + 1), RING + RED + 1024 + (ROWS + 2) * a.words * 4 + (a.direct == 1 ? 0 : a.B) * 16, st, 1, tm, a);
}
template <typename T>
cudaError_t pick(const CUtensorMap& tm, const TreeAttn& a, int rows, int grid, cudaStream_t st) {
    if (a.dim > 64) return rows == 16 ? run<T, 128, 1, 3, 3>(tm, a, grid, st) : run<T, 128, 2, 1, 3>(tm, a, grid, st);
    return rows == 16 ? run<T, 64, 1, 4, 4>(tm, a, grid, st) : rows == 32 ? run<T, 64, 2, 2, 2>(tm, a, grid, st) : run<T, 64, 4, 1, 3>(tm, a, grid, st);
}

}  // namespace

cudaError_t ta_tma_mma(const CUtensorMap& tm, const TreeAttn& a, int dtype, int rows, int grid, cudaStream_t st) {
    return dtype == SPECDEC_DTYPE_BF16 ? pick<__nv_bfloat16>(tm, a, rows, grid, st) : pick<__half>(tm, a, rows, grid, st);
}

}  // namespace sd
