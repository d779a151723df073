// Attention of drafted trees over the paged cache for 16-bit types and many query rows: tcgen05 (contract: specdec.h, work: tree_attention.cuh).
//
// CTA = one item, one CTA an SM.  A block is 128 keys; the scores of 128 rows against it are one accumulator in tensor memory (a row a lane), from which the
// row's thread takes maximum and exponentials; the probabilities go back into the same columns as 16-bit pairs and are the second product's A operand, the values
// its B operand as they lie ([key, column], N-major).  Two groups of four softmax warps keep the tensor pipe busy in turn:
//   TILES = 2: the groups have 128 rows each and share the blocks of a 256-row tile.
//   TILES = 1: the groups have the same 128 rows and take every second block; their results meet at the end.
// Warps: 0 loads (one TMA box a page), 1 issues the products, 4-7 and 8-11 are the groups.
//
// The running maximum is only moved (and the output, in tensor memory, rescaled) when it grows by more than 2^8: until then probabilities up to 2^8 are relative to
// the old one, which changes neither the quotient nor its relative precision.
//
// Per block and 128 rows the tensor pipe takes 8 D clocks (D = 128: 1024) and the exponentials 1024 (16 a clock and SM), so neither can hide the other wholly: with two groups
// the pair takes about the sum of a group's two parts.
#include <type_traits>

#include "tree_attention.cuh"

namespace sd {
namespace {

constexpr int TC_KT = 128, TC_ROWS = 128, TC_WARPS = 12;

__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t acc) {     // A in tensor memory
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
// N-major operand: rows (K) of 64 N-elements (128 bytes, swizzled); the next 64 N-elements `lead` bytes on, the next 8 rows 1024.
__device__ __forceinline__ uint64_t umma_desc_n_sw128(uint32_t smem_addr, uint32_t lead) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFF) >> 4);
    d |= (uint64_t)(lead >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int DP, int TILES> struct TcAttn {
    static constexpr int NS = DP > 64 ? 2 : 4;                                         // blocks of keys and of values in flight
    static constexpr int Q = TC_ROWS * DP * 2, SIDE = TC_KT * DP * 2;
    static constexpr int BYTES = TILES * Q + 2 * NS * SIDE;
};

template <typename T, int DP, int TILES>
__global__ void __launch_bounds__(32 * TC_WARPS, 1) k_ta_tc(const __grid_constant__ CUtensorMap tm, TreeAttn a) {
    using Cfg = TcAttn<DP, TILES>;
    constexpr int NS = Cfg::NS, SIDE = Cfg::SIDE, HALVES = DP / 64, KT = TC_KT, ROWS = TILES * TC_ROWS;
    constexpr uint32_t IDESC = (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(TC_ROWS >> 4) << 24);
    constexpr uint32_t IDESC_S = IDESC | ((uint32_t)(KT >> 3) << 17), IDESC_O = IDESC | (1u << 16) | ((uint32_t)(DP >> 3) << 17);   // O: B is N-major
    extern __shared__ __align__(1024) char tc_smem[];
    __shared__ __align__(8) uint64_t bars[4 * NS + 6];
    __shared__ int abort_flag;
    __shared__ uint32_t tmem_base;
    char* qs = tc_smem + (1024 - (smem_u32(tc_smem) & 1023)) % 1024;
    char* kring = qs + TILES * Cfg::Q;
    char* vring = kring + NS * SIDE;
    uint32_t* any = (uint32_t*)(vring + NS * SIDE);
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t kfull = smem_u32(bars), kempty = kfull + NS * 8, vfull = kempty + NS * 8, vempty = vfull + NS * 8;
    const uint32_t sfull = vempty + NS * 8, pready = sfull + 16, ofin = pready + 16;
    if (tid == 0) {
        for (int i = 0; i < 4 * NS; ++i) mbar_init(kfull + i * 8, 1);
        for (int g = 0; g < 2; ++g) { mbar_init(sfull + g * 8, 1); mbar_init(pready + g * 8, 4); mbar_init(ofin + g * 8, 1); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch_map(&tm);
    }
    const Item it = ta_item(a, (int*)kring);
    if (it.b < 0) return;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // ta_item's use of the ring, ahead of the boxes
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;                      // columns: scores 0, scores 1 (128 each), outputs 0, 1 (DP each)
    const SeqKeys s = ta_keys(a, it.b);
    const int k_begin = it.split * it.per * TA_BLOCK, k_end = (int)min((long long)(it.split + 1) * it.per * TA_BLOCK, (long long)s.keys);
    const int blocks = max(0, (k_end - k_begin + KT - 1) / KT);
    auto steps = [&](int g) { return TILES == 2 ? blocks : (blocks + 1 - g) / 2; };    // of group g; its i-th is block_of(g, i)
    auto block_of = [&](int g, int i) { return TILES == 2 ? i : 2 * i + g; };

    if (warp == 0) {                                      // loads
        const int page = 1 << a.page_shift, box = min(page, TA_BLOCK), n_boxes = KT / box;
        const int* table = a.table + (long long)s.seq * a.max_pages;
        auto page_of = [&](int j) {                       // this lane's page of block j: out of range where there is none
            const int key = k_begin + j * KT + lane * box, i = key >> a.page_shift;
            int p = -1;
            if (lane < n_boxes && key < k_end && i < a.max_pages) p = table[i];
            return (unsigned)p < (unsigned)a.n_pages ? p : a.n_pages;
        };
        int p = blocks ? page_of(0) : 0;
        bool ok = true;
        for (int j = 0; j < blocks && ok; ++j) {
            const int st = j % NS, key = k_begin + j * KT + lane * box, cur = p;
            if (j + 1 < blocks) p = page_of(j + 1);
            const bool mine = lane < n_boxes && key < k_end;
            const unsigned boxes = __popc(__ballot_sync(0xffffffffu, mine));
#pragma unroll
            for (int side = 0; side < 2 && ok; ++side) {
                const uint32_t full = (side ? vfull : kfull) + st * 8, empty = (side ? vempty : kempty) + st * 8;
                if (j >= NS) ok = mbar_wait_warp(empty, (j / NS - 1) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(full, boxes * box * 128 * HALVES);
                __syncwarp();
                if (mine) {
                    const uint32_t d = smem_u32((side ? vring : kring) + st * SIDE) + lane * box * 128;
#pragma unroll
                    for (int hf = 0; hf < HALVES; ++hf) ta_box(d + hf * KT * 128, &tm, hf * 64, it.h, key & (page - 1), cur, side, full);
                }
            }
        }
    } else if (warp >= 4) {                               // the queries, and what they see
        const int t = tid - 128, r0 = it.tile * ROWS, all_rows = a.T * a.group;
        for (int i = t; i < ROWS * (DP / 8); i += 256) {
            const int r = i / (DP / 8), c = i % (DP / 8), gr = r0 + r, node = ta_node(a, gr);
            uint4 x = make_uint4(0, 0, 0, 0);
            if (gr < all_rows && node < s.nodes && c * 8 < a.dim) {
                const char* p = a.q + it.b * a.q_sb + node * a.q_st + (it.h * a.group + gr - node * a.group) * a.q_sh + c * 16;
                if (a.q_vec) x = *reinterpret_cast<const uint4*>(p);
                else {
                    const unsigned short* e = reinterpret_cast<const unsigned short*>(p);
                    x = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                }
            }
            *reinterpret_cast<uint4*>(qs + (r / TC_ROWS) * Cfg::Q + (c >> 3) * TC_ROWS * 128 + (r % TC_ROWS) * 128 + (((c & 7) ^ (r & 7)) << 4)) = x;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        // (the mask rows: by these 256 threads, which count from 128)
        auto sync = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
        for (int w = t; w < a.words; w += 256) any[w] = 0;
        sync();
        const int t0 = ta_node(a, r0), t1 = min(ta_node(a, min(r0 + ROWS, all_rows) - 1), a.T - 1);
        for (int i = t; i < (t1 - t0 + 1) * a.words; i += 256) {
            const int node = t0 + i / a.words, w = i % a.words, left = s.nodes - w * 32;
            uint32_t m = node < s.nodes ? a.mask[it.b * a.mask_sb + (long long)node * a.words + w] : 0u;
            if (left < 32) m &= left <= 0 ? 0u : (1u << left) - 1u;
            mask[i] = m;
            if (m) atomicOr(any + w, m);
        }
    }
    // the queries are there (the loads run meanwhile)
    if (warp == 1 || warp >= 4) asm volatile("bar.sync 2, 288;" ::: "memory");

    if (warp == 1) {                                      // products
        bool ok = true;
        const int most = max(steps(0), steps(1));
        auto second = [&](int g, int i) {                 // output += probabilities x values
            const int j = block_of(g, i), st = j % NS;
            ok = ok && mbar_wait_warp(pready + g * 8, i & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT) &&
                 mbar_wait_warp(vfull + st * 8, (j / NS) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t v = umma_desc_n_sw128(smem_u32(vring + st * SIDE), KT * 128);
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk)      // 16 keys: 2048 bytes of values, 8 columns of probabilities
                    umma_ts(tmem + 256 + g * DP, tmem + g * 128 + kk * 8, v + kk * 128, IDESC_O, i || kk ? 1u : 0u);
                if (TILES == 1 || g == 1) umma_commit(vempty + st * 8);
                if (i + 1 == steps(g)) umma_commit(ofin + g * 8);
            }
        };
        for (int i = 0; i <= most && ok; ++i)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                if (!ok) break;
                if (i > 0 && i <= steps(g)) second(g, i - 1);
                if (!ok || i >= steps(g)) continue;
                const int j = block_of(g, i), st = j % NS;
                ok = mbar_wait_warp(kfull + st * 8, (j / NS) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk) {
                        const uint64_t q = umma_desc_k_sw128(smem_u32(qs + (TILES == 2 ? g : 0) * Cfg::Q) + (kk / 4) * TC_ROWS * 128) + (kk % 4) * 2;
                        const uint64_t k = umma_desc_k_sw128(smem_u32(kring + st * SIDE) + (kk / 4) * KT * 128) + (kk % 4) * 2;
                        umma_bf16(tmem + g * 128, q, k, IDESC_S, kk ? 1u : 0u);
                    }
                    umma_commit(sfull + g * 8);
                    if (TILES == 1 || g == 1) umma_commit(kempty + st * 8);
                }
            }
    } else if (warp >= 4) {                               // softmax: one row a thread
        const int g = (warp - 4) >> 2, r = (TILES == 2 ? g * TC_ROWS : 0) + (warp & 3) * 32 + lane, r0 = it.tile * ROWS, gr = r0 + r;
        const int node = ta_node(a, gr), n = steps(g);
        const bool live = gr < a.T * a.group && node < s.nodes;
        const uint32_t* row = mask + (live ? (node - ta_node(a, r0)) * a.words : 0);
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;                  // this warp's lanes: 32 (warp % 4) in bits 16..31
        const uint32_t ts = tmem + g * 128 + lanes, to = tmem + 256 + g * DP + lanes;
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int j = block_of(g, i), k0 = k_begin + j * KT;
            ok = mbar_wait_warp(sfull + g * 8, i & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
            if (!ok) break;
            tc_fence_after();
            const bool tail = k0 + KT > s.len;
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < KT / 32; ++c) {
                float x[32];
                tmem_ld32(ts + c * 32, x);
                if (tail) {
                    const uint32_t w = live ? ta_window(row, a.words, k0 + c * 32 - s.len) : 0u;
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = w >> e & 1 ? x[e] : -INFINITY;
                }
                float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                for (int e = 0; e < 32; e += 4) { t0 = fmaxf(t0, fmaxf(x[e], x[e + 1])); t1 = fmaxf(t1, fmaxf(x[e + 2], x[e + 3])); }
                top = fmaxf(top, fmaxf(t0, t1));
            }
            top *= a.scale;
            const bool grow = top > (m == -INFINITY ? m : m + 8.f);
            if (__any_sync(0xffffffffu, grow)) {
                const float f = grow ? ta_exp2(m - top) : 1.f;              // (m = -inf: 0)
                if (grow) m = top;
                l *= f;
                if (i > 0) {
#pragma unroll
                    for (int c = 0; c < DP / 16; ++c) {
                        float x[16];
                        uint32_t y[16];
                        tmem_ld<16>(to + c * 16, x);
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(f == 0.f ? 0.f : x[e] * f);
                        tmem_st16(to + c * 16, y);
                    }
                    tmem_st_wait();
                }
            }
            const float z = m == -INFINITY ? 0.f : m;
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int c = 0; c < KT / 32; ++c) {
                float x[32];
                uint32_t y[16];
                tmem_ld32(ts + c * 32, x);
                if (tail) {
                    const uint32_t w = live ? ta_window(row, a.words, k0 + c * 32 - s.len) : 0u;
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = w >> e & 1 ? x[e] : -INFINITY;
                }
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float u = ta_exp2(fmaf(x[e], a.scale, -z)), v = ta_exp2(fmaf(x[e + 1], a.scale, -z));
                    l0 += u; l1 += v;
                    y[e / 2] = Half<T>::pack(u, v);
                }
                tmem_st16(ts + c * 16, y);                // over scores that have been read
            }
            l += l0 + l1;
            if (tail && (TILES == 1 || g == 0)) {         // values that no query sees: whatever is in them is multiplied by 0
                const int st = j % NS;
                ok = mbar_wait_warp(vfull + st * 8, (j / NS) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
                if (!ok) break;
                // (each of the group's warps a quarter of the rows)
                const uint32_t seen = ta_window(any, a.words, k0 + (warp & 3) * 32 - s.len);
                for (int q = lane; q < 32 * 8 * HALVES; q += 32) {
                    const int rr = q / 8 % 32, hf = q / 256;
                    if (!(seen >> rr & 1)) *reinterpret_cast<uint4*>(vring + st * SIDE + hf * KT * 128 + ((warp & 3) * 32 + rr) * 128 + (q & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(pready + g * 8);
        }
        if (ok && n) ok = mbar_wait_warp(ofin + g * 8, 0, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
        tc_fence_after();
        if (!live) { m = -INFINITY; l = 0.f; }
        if (l == 0.f) m = -INFINITY;
        float f = l == 0.f ? 0.f : 1.f, f1 = 0.f;         // shares of this group's output and, TILES = 1, of the other's
        const float* red = reinterpret_cast<const float*>(kring) + (warp & 3) * 32 + lane;             // [DP + 2][128]: columns, maximum, sum
        if constexpr (TILES == 1) {                       // the second group's results through the ring, once the products have read it
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (g == 1) {
                float* to_red = const_cast<float*>(red);
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) {
                    float x[32];
                    if (n) tmem_ld32(to + c * 32, x);
#pragma unroll
                    for (int e = 0; e < 32; ++e) to_red[(c * 32 + e) * 128] = n && l != 0.f ? x[e] : 0.f;
                }
                to_red[DP * 128] = m; to_red[(DP + 1) * 128] = l;
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (g == 0) {
                const float m1 = red[DP * 128], l1 = red[(DP + 1) * 128], mm = fmaxf(m, m1), z = mm == -INFINITY ? 0.f : mm;
                f = ta_exp2(m - z); f1 = ta_exp2(m1 - z);
                l = l * f + l1 * f1;
                m = mm;
            }
        }
        if (TILES == 2 || g == 0) {
            const bool real = gr < a.T * a.group;
            const float inv = it.splits > 1 ? 1.f : l > 0.f || l != l ? 1.f / l : 0.f;
            char* p = a.out + it.b * a.o_sb + node * a.o_st + (it.h * a.group + gr - node * a.group) * a.o_sh;
            const long long slot = (long long)blockIdx.x * ROWS + r;
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                float x[32];
                if (n) tmem_ld32(to + c * 32, x);
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    float y = n && f != 0.f ? x[e] * f : 0.f;
                    if constexpr (TILES == 1) y = fmaf(red[(c * 32 + e) * 128], f1, y);
                    x[e] = y * inv;
                }
                if (!real) continue;
                if (it.splits == 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        if (c * 32 + e >= a.dim) break;
                        uint32_t y[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) y[q] = Half<T>::pack(x[e + 2 * q], x[e + 2 * q + 1]);
                        if (a.out_vec) *reinterpret_cast<uint4*>(p + (c * 32 + e) * 2) = make_uint4(y[0], y[1], y[2], y[3]);
                        else
#pragma unroll
                            for (int q = 0; q < 8; ++q) reinterpret_cast<unsigned short*>(p + (c * 32 + e) * 2)[q] = (unsigned short)(y[q / 2] >> (q & 1) * 16);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        if (c * 32 + e < a.dim) *reinterpret_cast<float4*>(a.part + slot * a.dim + c * 32 + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                }
            }
            if (real && it.splits > 1) a.part_ml[slot] = make_float2(m, l);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

template <typename T, int DP, int TILES>
cudaError_t run(const CUtensorMap& tm, const TreeAttn& a, int grid, cudaStream_t st) {
    constexpr int BYTES = TcAttn<DP, TILES>::BYTES + 1024, MOST = BYTES + (TILES * TC_ROWS + 1) * 32 * 4;
    static_assert(MOST <= 232448 - 1024, "shared memory of an SM");
    static const cudaError_t attr = cudaFuncSetAttribute(k_ta_tc<T, DP, TILES>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
    if (attr != cudaSuccess) return attr;
    k_ta_tc<T, DP, TILES><<<grid, 32 * TC_WARPS, BYTES + (TILES * TC_ROWS + 1) * a.words * 4, st>>>(tm, a);
    return cudaGetLastError();
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
