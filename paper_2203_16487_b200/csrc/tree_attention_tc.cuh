// Attention of drafted trees over the paged cache for many query rows: tcgen05 (contract: specdec.h, work: tree_attention.cuh).  The cache is of 16-bit types, or in 4 bits (FP4, format: fp4.cuh).
//
// One CTA an SM.  A block is 128 keys; the scores of 128 rows against it are one accumulator in tensor memory (a row a lane), which the row's thread takes into
// registers for maximum and exponentials; the probabilities go back into the same columns as 16-bit pairs and are the second product's A operand
// (of B's type, as tcgen05.mma wants it; the sum adds up the rounded ones), the values its B operand as they lie ([key, column], N-major).  Two groups of four softmax warps keep the tensor pipe busy in turn:
//   TILES = 2: the groups have 128 rows each and share the blocks of a 256-row tile.
//   TILES = 1: the groups have the same 128 rows and take every second block; their results meet at the end.
// Warps: 0 loads (one TMA box a page), 1 issues the products, 4-7 and 8-11 are the groups.  4 bits: bulk copies of a page's codes and scales, and four more warps, 12-15, that turn half
// a block at a time (keys, then values) into fp16 where the boxes would have landed.
//
// A group's chain is scores (512 clocks at D = 128), maximum, exponentials (1024: 16 a clock and SM), second product (512, its first half under the second half of the
// exponentials), and its scores' columns are taken by the probabilities until that is done.  Blocks of 64 keys leave room for both, so that
// the next scores can be under way meanwhile, but each issue of products costs some 200 clocks beside their own: 256 rows took 5760 clocks for 128 keys instead of 3700.
//
// 8 x 64 queries, 32/8 heads of 128, over 8191 to 16,385 keys: 121 us with the merge (8 us) in a burst, 866 TFLOP/s, the tensor pipe 50 % active; 145 us as a call among others, at
// lower clocks.  The same over 4 bits: 145 us, whose unpacking warps keep up; the tensor pipe 32 %.  (A quarter of the exponentials as polynomials on the fused multiply-adds: 130 us; it is the chain, not their rate.)
//
// The running maximum is only moved (and the output, in tensor memory, rescaled) when it grows by more than 2^8: until then probabilities up to 2^8 are relative to
// the old one, which changes neither the quotient nor its relative precision: a dominating one is not exactly 1 any more, but its rounding is in the sum as well.
#pragma once
#include <type_traits>

#include "fp4_attention.cuh"

namespace sd {
namespace {

constexpr int TC_KT = 128, TC_ROWS = 128;

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
// Two fp32 at a time.
__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int DP, int TILES, bool FP4> struct TcAttn {
    static constexpr int WARPS = FP4 ? 16 : 12, NS = DP > 64 ? 2 : 4;                  // blocks of keys and of values in flight
    static constexpr int Q = TC_ROWS * DP * 2, SIDE = TC_KT * DP * 2;
    // 4 bits: half a block (keys or values) as it lies in memory, codes and scales; how many of them are in flight; the factor of each row's scores
    static constexpr int CODES = TC_KT * DP / 2, RAW = CODES + TC_KT * DP / 16, NR = FP4 ? (DP > 64 ? 3 : 6) : 0, FACTORS = FP4 ? TILES * TC_ROWS * 4 : 0;
    static constexpr int BYTES = TILES * Q + 2 * NS * SIDE + NR * RAW + FACTORS;
};

// Args: TreeAttn, or Fp4Attn (FP4).  T: the type of queries and outputs.  FP4: the operands of both products are fp16.
template <typename T, int DP, int TILES, bool FP4, typename Args>
__device__ __forceinline__ void ta_tc(const CUtensorMap* tm, const Args& a) {
    using Cfg = TcAttn<DP, TILES, FP4>;
    using P = std::conditional_t<FP4, __half, T>;         // of the products' operands
    constexpr int NS = Cfg::NS, SIDE = Cfg::SIDE, HALVES = DP / 64, KT = TC_KT, ROWS = TILES * TC_ROWS;
    constexpr float P_SHIFT = FP4 ? 7.f : 0.f;            // probabilities are 2^7 times their value: fp16 ends at 2^-24
    constexpr uint32_t IDESC = (1u << 4) | (std::is_same<P, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(TC_ROWS >> 4) << 24);
    constexpr uint32_t IDESC_S = IDESC | ((uint32_t)(KT >> 3) << 17), IDESC_O = IDESC | (1u << 16) | ((uint32_t)(DP >> 3) << 17);   // O: B is N-major
    extern __shared__ __align__(1024) char tc_smem[];
    constexpr int NR = Cfg::NR, RAW = Cfg::RAW, CONVERTERS = FP4 ? 4 : 1;
    __shared__ __align__(8) uint64_t bars[4 * NS + 8 + 2 * NR];
    __shared__ int abort_flag;
    __shared__ uint32_t tmem_base;
    __shared__ float2 other[TILES == 1 ? TC_ROWS : 1];    // maximum and sum of the second group's rows
    char* qs = tc_smem + (1024 - (smem_u32(tc_smem) & 1023)) % 1024;
    char* kring = qs + TILES * Cfg::Q;
    char* vring = kring + NS * SIDE;
    char* raw = vring + NS * SIDE;
    float* factor = (float*)(raw + NR * RAW);
    int4* seqs = (int4*)(raw + NR * RAW + Cfg::FACTORS);  // [B] where sequences are cut
    uint32_t* any = (uint32_t*)(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t kfull = smem_u32(bars), kempty = kfull + NS * 8, vfull = kempty + NS * 8, vempty = vfull + NS * 8;
    const uint32_t sfull = vempty + NS * 8, pready = sfull + 16, ofin = pready + 32;            // of group g: + 8 g; pready: of a half, + 16 g + 8 half
    const uint32_t rfull = ofin + 16, rempty = rfull + NR * 8;
    if (tid == 0) {
        for (int i = 0; i < 4 * NS; ++i) mbar_init(kfull + i * 8, (i / NS) % 2 == 0 ? CONVERTERS : 1);
        for (int i = 0; i < NR; ++i) { mbar_init(rfull + i * 8, 1); mbar_init(rempty + i * 8, CONVERTERS); }
        for (int g = 0; g < 2; ++g) { mbar_init(sfull + g * 8, 1); mbar_init(pready + g * 16, 4); mbar_init(pready + g * 16 + 8, 4); mbar_init(ofin + g * 8, 1); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if constexpr (!FP4) tma_prefetch_map(tm);
    }
    op_begin();
    TaWork work;
    work.begin(a, seqs);
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;                      // columns: scores of the groups (128 each), outputs from 256 (DP each)
    // steps of group g in a part of `blocks` blocks of 128 keys; its i-th is block_of(g, i)
    auto steps = [](int blocks, int g) { return TILES == 2 ? blocks : (blocks + 1 - g) / 2; };
    auto block_of = [](int g, int i) { return TILES == 2 ? i : 2 * i + g; };
    auto wait = [&](uint32_t bar, int n) { return mbar_wait_warp<true>(bar, n & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT); };     // for its completion number n
    Part it;
    int done = 0;                                         // blocks of the parts before: block j is in stage (done + j) % NS
    bool ok = true;

    // 384 threads have 168 registers each: the first warpgroup passes on what the softmax groups need (128 x 104 + 256 x 200 = 384 x 168).  4 bits: 512 threads have 128, and
    // two warpgroups do (256 x 56 + 256 x 200 = 512 x 128)
    if (FP4 && warp >= 12) {                              // keys and values from 4 bits to fp16, running ahead into the next parts
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if constexpr (FP4) {
            // a lane takes 32 channels of a key: 16 bytes of codes, two scales, four pieces out; lanes of a store in eight different columns of banks
            constexpr int PER = DP / 32, ITEMS = KT * PER / 128;
            const int quarter = lane % PER, row0 = (warp - 12) * (32 / PER) + lane / PER, turn = DP > 64 ? quarter & 2 : 0;
            int h = 0;                                    // half blocks so far
            for (; ok && work.next(a, seqs, it); done += it.blocks)
                for (int j = 0; j < it.blocks && ok; ++j) {
                    const int n = done + j, st = n % NS;
#pragma unroll 1
                    for (int side = 0; side < 2; ++side, ++h) {
                        const int slot = h % NR;
                        ok = wait(rfull + slot * 8, h / NR);
                        if (n >= NS) ok = ok && wait((side ? vempty : kempty) + st * 8, n / NS - 1);
                        if (!ok) break;
                        const char* from = raw + slot * RAW;
                        char* to = (side ? vring : kring) + st * SIDE;
#pragma unroll
                        for (int i = 0; i < ITEMS; ++i) {
                            const int r = row0 + i * (128 / PER);
                            const uint4 v = *reinterpret_cast<const uint4*>(from + r * (DP / 2) + quarter * 16);
                            const uint32_t s = fp4_scales2(*reinterpret_cast<const unsigned short*>(from + Cfg::CODES + r * (DP / 16) + quarter * 2));
                            const uint32_t s2[2] = {__byte_perm(s, s, 0x1010), __byte_perm(s, s, 0x3232)}, w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int q = e ^ turn, c = quarter * 4 + q;
                                const uint32_t x = turn ? w[e ^ 2] : w[e], sc = s2[(e >> 1) ^ (turn >> 1)];
                                uint32_t o[4];
                                fp4_unpack8(x, o);
                                *reinterpret_cast<uint4*>(to + (c >> 3) * KT * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(h2_mul(o[0], sc), h2_mul(o[1], sc), h2_mul(o[2], sc), h2_mul(o[3], sc));
                            }
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");             // ahead of the products that read them
                        __syncwarp();
                        if (lane == 0) { mbar_arrive((side ? vfull : kfull) + st * 8); mbar_arrive(rempty + slot * 8); }
                    }
                }
        }
    } else if (warp < 4) {
    if constexpr (FP4) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (FP4 && warp == 0) {                               // loads, running ahead into the next parts
        if constexpr (FP4) {
        const int page = 1 << a.page_shift, box = min(page, KT), n_boxes = KT / box;
        int h = 0;                                        // half blocks so far
        for (; ok && work.next(a, seqs, it);) {
            const int* table = a.table + (long long)it.s.seq * a.max_pages;
            auto page_of = [&](int j) {                   // this lane's page of block j: -1 where there is none
                const int key = it.k_begin + j * KT + lane * box, i = key >> a.page_shift;
                int p = -1;
                if (lane < n_boxes && key < it.k_end && i < a.max_pages) p = table[i];
                return (unsigned)p < (unsigned)a.n_pages ? p : -1;
            };
            int p = it.blocks ? page_of(0) : 0;
            for (int j = 0; j < it.blocks && ok; ++j) {
                const int key = it.k_begin + j * KT + lane * box, cur = p;
                if (j + 1 < it.blocks) p = page_of(j + 1);
                const bool mine = lane < n_boxes && key < it.k_end;
                const unsigned boxes = __popc(__ballot_sync(0xffffffffu, mine && cur >= 0));
                const int first = key & (page - 1);
                const long long codes = cur * a.s_page + it.h * a.s_head + first * (DP / 2), scales = cur * a.c_page + it.h * a.c_head + first * (DP / 16);
#pragma unroll 1
                for (int side = 0; side < 2; ++side, ++h) {
                    const int slot = h % NR;
                    if (h >= NR) ok = ok && wait(rempty + slot * 8, h / NR - 1);
                    if (!ok) break;
                    char* to = raw + slot * RAW;
                    if (mine && cur < 0) {                // a page that is none: zeros, ahead of what the slot's next block brings
                        for (int i = 0; i < box * DP / 16; i += 16) *reinterpret_cast<uint4*>(to + Cfg::CODES + lane * box * (DP / 16) + i) = make_uint4(0, 0, 0, 0);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    if (lane == 0) mbar_expect_tx(rfull + slot * 8, boxes * box * (DP / 2 + DP / 16));
                    __syncwarp();
                    if (mine && cur >= 0) {
                        bulk_copy(smem_u32(to) + lane * box * (DP / 2), (side ? a.v : a.k) + codes, box * (DP / 2), rfull + slot * 8);
                        bulk_copy(smem_u32(to) + Cfg::CODES + lane * box * (DP / 16), (side ? a.vs : a.ks) + scales, box * (DP / 16), rfull + slot * 8);
                    }
                }
            }
        }
        }
    } else if (warp == 0) {                               // loads, running ahead into the next parts
        const int page = 1 << a.page_shift, box = min(page, TA_BLOCK), n_boxes = KT / box;
        for (; ok && work.next(a, seqs, it); done += it.blocks) {
            const int* table = a.table + (long long)it.s.seq * a.max_pages;
            auto page_of = [&](int j) {                   // this lane's page of block j: out of range where there is none
                const int key = it.k_begin + j * KT + lane * box, i = key >> a.page_shift;
                int p = -1;
                if (lane < n_boxes && key < it.k_end && i < a.max_pages) p = table[i];
                return (unsigned)p < (unsigned)a.n_pages ? p : a.n_pages;
            };
            int p = it.blocks ? page_of(0) : 0;
            for (int j = 0; j < it.blocks && ok; ++j) {
                const int n = done + j, st = n % NS, key = it.k_begin + j * KT + lane * box, cur = p;
                if (j + 1 < it.blocks) p = page_of(j + 1);
                const bool mine = lane < n_boxes && key < it.k_end;
                const unsigned boxes = __popc(__ballot_sync(0xffffffffu, mine));
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    const uint32_t full = (side ? vfull : kfull) + st * 8, empty = (side ? vempty : kempty) + st * 8;
                    if (n >= NS) ok = ok && wait(empty, n / NS - 1);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(full, boxes * box * 128 * HALVES);
                    __syncwarp();
                    if (mine) {
                        const uint32_t d = smem_u32((side ? vring : kring) + st * SIDE) + lane * box * 128;
#pragma unroll
                        for (int hf = 0; hf < HALVES; ++hf) ta_box(d + hf * KT * 128, tm, hf * 64, it.h, key & (page - 1), cur, side, full);
                    }
                }
            }
        }
    } else if (warp == 1) {                               // products
        int taken[2] = {0, 0};                            // steps of the groups in the parts before
        for (; work.next(a, seqs, it); done += it.blocks, taken[0] += steps(it.blocks, 0), taken[1] += steps(it.blocks, 1)) {
            asm volatile("bar.sync 2, 288;" ::: "memory");            // the queries are there, the last outputs have been read
            tc_fence_after();
            const int n0 = steps(it.blocks, 0), n1 = steps(it.blocks, 1);
            auto first = [&](int g, int i) {              // scores = queries x keys
                const int n = done + block_of(g, i), st = n % NS;
                ok = ok && wait(kfull + st * 8, n / NS);
                if (!ok) return;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < DP / 16; ++kk) {
                        const uint64_t q = umma_desc_k_sw128(smem_u32(qs + (TILES == 2 ? g : 0) * Cfg::Q) + (kk / 4) * TC_ROWS * 128) + (kk % 4) * 2;
                        const uint64_t k = umma_desc_k_sw128(smem_u32(kring + st * SIDE) + (kk / 4) * KT * 128) + (kk % 4) * 2;
                        umma_bf16(tmem + g * KT, q, k, IDESC_S, kk ? 1u : 0u);
                    }
                    umma_commit(sfull + g * 8);
                    if (TILES == 1 || g == 1) umma_commit(kempty + st * 8);
                }
            };
            auto second = [&](int g, int i, bool last) {  // output += probabilities x values, 64 keys at a time
                const int n = done + block_of(g, i), st = n % NS;
                ok = ok && wait(vfull + st * 8, n / NS);
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    ok = ok && wait(pready + g * 16 + hf * 8, taken[g] + i);
                    if (!ok) return;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t v = umma_desc_n_sw128(smem_u32(vring + st * SIDE), KT * 128);
#pragma unroll
                        for (int kk = hf * 4; kk < hf * 4 + 4; ++kk)           // 16 keys: 2048 bytes of values, 8 columns of probabilities
                            umma_ts(tmem + 256 + g * DP, tmem + g * KT + kk * 8, v + kk * 128, IDESC_O, i || kk ? 1u : 0u);
                        if (hf == 1) {
                            if (TILES == 1 || g == 1) umma_commit(vempty + st * 8);
                            if (last) umma_commit(ofin + g * 8);
                        }
                    }
                }
            };
            for (int i = 0; i <= n0 && ok; ++i)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int n = g ? n1 : n0;
                    if (i > 0 && i <= n) second(g, i - 1, i == n);
                    if (i < n) first(g, i);               // (behind the second product, which reads the probabilities in its columns)
                }
        }
    }
    } else {                                              // softmax: one row a thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int g = (warp - 4) >> 2, t = tid - 128, all_rows = a.T * a.group;
        int taken = 0, outputs = 0;                       // this group's steps and outputs in the parts before
        auto softmax_warps = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
        while (work.next(a, seqs, it, t == 0)) {
        const SeqKeys& s = it.s;
        const int r0 = it.tile * ROWS;
        // the queries: thread t takes piece t % PIECES of every (256 / PIECES)-th row
        constexpr int PIECES = DP / 8;
        const int qc = t % PIECES;
        char* q_to = qs + (qc >> 3) * TC_ROWS * 128;
        const char* q_from = a.q + it.b * a.q_sb + it.h * a.group * a.q_sh + qc * 16;
        if constexpr (FP4 && !std::is_same<T, __half>::value) {       // as fp16, each row scaled by a power of two
#pragma unroll 2
            for (int r = t / PIECES; r < ROWS; r += 256 / PIECES) {
                const int gr = r0 + r, node = ta_node(a, gr);
                uint32_t w[4] = {0, 0, 0, 0};
                if (gr < all_rows && node < s.nodes) {
                    const char* p = q_from + node * a.q_st + (gr - node * a.group) * a.q_sh;
                    if (a.q_vec) { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
                    else
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const unsigned short*>(p)[2 * i] | (uint32_t)reinterpret_cast<const unsigned short*>(p)[2 * i + 1] << 16;
                }
                float x[8], top = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) { x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); top = fmaxf(top, fabsf(x[i])); }
#pragma unroll
                for (int of = 1; of < PIECES; of <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, of));
                const int shift = row_shift(top);
                const float f = power2(shift);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = Half<__half>::pack(x[2 * i] * f, x[2 * i + 1] * f);
                *reinterpret_cast<uint4*>(q_to + (r / TC_ROWS) * Cfg::Q + (r % TC_ROWS) * 128 + (((qc & 7) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                if (qc == 0) factor[r] = power2(-shift);
            }
        } else
#pragma unroll 4
        for (int r = t / PIECES; r < ROWS; r += 256 / PIECES) {
            const int gr = r0 + r, node = ta_node(a, gr);
            const bool real = gr < all_rows && node < s.nodes && qc * 8 < a.dim;
            const char* p = q_from + (real ? node * a.q_st + (gr - node * a.group) * a.q_sh : 0);
            char* to = q_to + (r / TC_ROWS) * Cfg::Q + (r % TC_ROWS) * 128 + (((qc & 7) ^ (r & 7)) << 4);
            if (a.q_vec) ta_copy16(smem_u32(to), real ? p : a.q, real);
            else {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (real) {
                    const unsigned short* e = reinterpret_cast<const unsigned short*>(p);
                    x = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                }
                *reinterpret_cast<uint4*>(to) = x;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        for (int w = t; w < a.words; w += 256) any[w] = 0;            // what they see (as ta_load_masks, by the threads from 128 on)
        softmax_warps();
        const int t0n = ta_node(a, r0), t1n = min(ta_node(a, min(r0 + ROWS, all_rows) - 1), a.T - 1);
        for (int i = t; i < (t1n - t0n + 1) * a.words; i += 256) {
            const int node = t0n + i / a.words, w = i % a.words, left = s.nodes - w * 32;
            uint32_t m = node < s.nodes ? a.mask[it.b * a.mask_sb + (long long)node * a.words + w] : 0u;
            if (left < 32) m &= left <= 0 ? 0u : (1u << left) - 1u;
            mask[i] = m;
            if (m) atomicOr(any + w, m);
        }
        asm volatile("cp.async.wait_all;\n\tfence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        asm volatile("bar.sync 2, 288;" ::: "memory");

        const int r = (TILES == 2 ? g * TC_ROWS : 0) + (warp & 3) * 32 + lane, gr = r0 + r, node = ta_node(a, gr), n = steps(it.blocks, g);
        const bool live = gr < a.T * a.group && node < s.nodes;
        const uint32_t* row = mask + (live ? (node - t0n) * a.words : 0);
        float scale = a.scale, unit = 1.f;
        if constexpr (FP4) {
            if (a.unit_k) { scale *= a.unit_k[it.h]; unit = a.unit_v[it.h]; }
            if constexpr (!std::is_same<T, __half>::value) scale *= factor[r];
        }
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;                  // this warp's lanes: 32 (warp % 4) in bits 16..31
        const uint32_t ts = tmem + g * KT + lanes, to = tmem + 256 + g * DP + lanes;
        // Fused with the subtraction of its maximum, a product leaves what the maximum's rounding has cut off, and the difference to the shift is rounded too: nothing to speak of, but from 2^20 on either may be
        // more than the probabilities' type has room for.
        //   16 bits: such a maximum becomes 0, by taking the score that it came from off all of the row's scores, this block's and, `moved`, the later ones'.
        //   4 bits: the products are rounded as the maximum was, which is taken off before the shift is put on.
        // (8 x 64 queries over 8191 to 16385 keys without either 144.2 and 145.4 us, so 144.2 and 145.9; the first way over 4 bits 153, the second over 16 146.6.)
        constexpr bool MOVES = !FP4;
        auto beyond = [](float y) { return fabsf(y) > 1048576.f && fabsf(y) < INFINITY; };
        float m = -INFINITY, l = 0.f, from = 0.f;
        bool moved = false;                               // whether a row of the warp has a number taken off its scores
        auto take_off = [](uint32_t (&x)[KT / 32][32], float y) {
#pragma unroll
            for (int e = 0; e < KT; ++e) x[e / 32][e % 32] = __float_as_uint(__fsub_rn(__uint_as_float(x[e / 32][e % 32]), y));
        };
        for (int i = 0; i < n; ++i) {
            const int j = block_of(g, i), k0 = it.k_begin + j * KT;
            ok = ok && wait(sfull + g * 8, taken + i);    // (and with it the last second product, which was issued before)
            if (!ok) break;
            tc_fence_after();
            uint32_t x[KT / 32][32];                      // the row's scores
#pragma unroll
            for (int c = 0; c < KT / 32; ++c) tmem_ld_issue<32>(ts + c * 32, x[c]);
#pragma unroll
            for (int c = 0; c < KT / 32; ++c) tmem_ld_done<32>(x[c]);
            const bool tail = k0 + KT > s.len;
            if (tail || moved) {                          // (one branch: two take 1 % longer)
                if (moved) take_off(x, from);
                if (tail) {
#pragma unroll
                for (int c = 0; c < KT / 32; ++c) {
                    const uint32_t w = live ? ta_window(row, a.words, k0 + c * 32 - s.len) : 0u;
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[c][e] = w >> e & 1 ? x[c][e] : 0xff800000u;
                }
                if (TILES == 1 || g == 0) {               // values that no query sees: whatever is in them is multiplied by 0
                    const int st = (done + j) % NS;
                    ok = wait(vfull + st * 8, (done + j) / NS);
                    if (!ok) break;
                    const uint32_t seen = ta_window(any, a.words, k0 + (warp & 3) * 32 - s.len);      // each of the group's warps a quarter of the rows
                    for (int q = lane; q < 32 * 8 * HALVES; q += 32) {
                        const int rr = q / 8 % 32, hf = q / 256;
                        if (!(seen >> rr & 1)) *reinterpret_cast<uint4*>(vring + st * SIDE + hf * KT * 128 + ((warp & 3) * 32 + rr) * 128 + (q & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                }
            }
            float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < KT; e += 2)
                t4[e / 2 % 4] = fmaxf(t4[e / 2 % 4], fmaxf(__uint_as_float(x[e / 32][e % 32]), __uint_as_float(x[e / 32][e % 32 + 1])));
            const float most = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])), top = most * scale;
            // (4 bits: not top > m + 8, which for a large m is rounded up to the next number behind it; nothing seen so far: infinite)
            const bool grow = MOVES ? top > (m == -INFINITY ? m : m + 8.f) : top - m > 8.f;
            if (__any_sync(0xffffffffu, grow)) {
                const float f = grow ? ta_exp2(m - top) : 1.f;              // (m = -inf: 0)
                if (grow) m = top;
                l *= f;
                if (MOVES && __any_sync(0xffffffffu, beyond(m))) {
                    const float y = beyond(m) ? most : 0.f;             // (a maximum beyond is of this block: older ones are 0 by now)
                    take_off(x, y);
                    from += y;
                    if (beyond(m)) m = 0.f;
                    moved = true;
                }
                if (i > 0) {
#pragma unroll 1
                    for (int c = 0; c < DP / 16; ++c) {
                        uint32_t y[16];
                        tmem_ld_issue<16>(to + c * 16, y);
                        tmem_ld_done<16>(y);
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(f == 0.f ? 0.f : __uint_as_float(y[e]) * f);
                        tmem_st16(to + c * 16, y);
                    }
                }
            }
            const float y0 = m == -INFINITY ? 0.f : m;
            float times = scale, plus = P_SHIFT - y0;
            if (!MOVES && __any_sync(0xffffffffu, beyond(y0))) {
#pragma unroll
                for (int e = 0; e < KT; ++e) x[e / 32][e % 32] = __float_as_uint(__fmul_rn(__uint_as_float(x[e / 32][e % 32]), scale));
                take_off(x, y0);
                times = 1.f; plus = P_SHIFT;
            }
            float sum[4] = {0.f, 0.f, 0.f, 0.f};          // of the rounded probabilities
            const uint64_t scale2 = pair2(times, times), z2 = pair2(plus, plus);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
                for (int c = hf * 2; c < hf * 2 + 2; ++c) {
                    uint32_t y[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint64_t d = fma2(pair2(__uint_as_float(x[c][2 * e]), __uint_as_float(x[c][2 * e + 1])), scale2, z2);
                        const float u = ta_exp2(__uint_as_float((uint32_t)d)), v = ta_exp2(__uint_as_float((uint32_t)(d >> 32)));
                        y[e] = Half<P>::pack(u, v);
                        sum[e & 3] = Half<P>::add(sum[e & 3], y[e]);
                    }
                    tmem_st16(ts + c * 16, y);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready + g * 16 + hf * 8);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        if (ok && n) ok = wait(ofin + g * 8, outputs++);
        taken += n;
        done += it.blocks;
        tc_fence_after();
        if (moved) m = fmaf(from, scale, m);
        if (!live) { m = -INFINITY; l = 0.f; }
        if (l == 0.f) m = -INFINITY;
        float f = l == 0.f ? 0.f : 1.f, f1 = 0.f;         // shares of this group's output and, TILES = 1, of the other's
        const int rr = (warp & 3) * 32 + lane, n1 = steps(it.blocks, 1);
        if constexpr (TILES == 1) {                       // both outputs are in this lane's tensor memory: the first group adds them up
            if (g == 1) { other[rr] = make_float2(m, l); tc_fence_before(); }      // (what the second group has waited for, the first reads)
            softmax_warps();
            if (g == 0) {
                tc_fence_after();
                const float m1 = other[rr].x, l1 = other[rr].y, mm = fmaxf(m, m1), z = mm == -INFINITY ? 0.f : mm;
                f = ta_exp2(m - z); f1 = ta_exp2(m1 - z);
                l = l * f + l1 * f1;
                m = mm;
            }
        }
        if (TILES == 2 || g == 0) {
            // through this group's queries' place in shared memory, 128 rows of 128 bytes at a time, so that rows leave in whole lines
            const float inv = !it.whole ? unit : l > 0.f || l != l ? unit / l : 0.f;
            constexpr int BUFFERS = Cfg::Q / (TC_ROWS * 128);                            // 2 (one is filled while the other leaves), or 1
            char* stage = qs + (TILES == 2 ? g : 0) * Cfg::Q;
            auto group_sync = [&] { asm volatile("bar.sync %0, 128;" ::"r"(3 + g) : "memory"); };
            auto columns = [&](int c, float* x) {         // 32 columns of this thread's row
                if (n) tmem_ld32(to + c * 32, x);
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = n && f != 0.f ? x[e] * f : 0.f;
                if (TILES == 1 && n1) {
                    float x1[32];
                    tmem_ld32(to + DP + c * 32, x1);
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = f1 != 0.f ? fmaf(x1[e], f1, x[e]) : x[e];
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] *= inv;
            };
            const int per = it.whole ? 64 : 32;           // columns of 128 bytes
            for (int c0 = 0; c0 < a.dim; c0 += per) {
                if (BUFFERS == 2) stage = qs + (TILES == 2 ? g : 0) * Cfg::Q + (c0 / per & 1) * TC_ROWS * 128;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    if (hf && !it.whole) break;
                    float x[32];
                    columns(c0 / 32 + hf, x);
                    if (it.whole) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<uint4*>(stage + rr * 128 + (((hf * 4 + q) ^ (rr & 7)) << 4)) =
                                make_uint4(Half<T>::pack(x[8 * q], x[8 * q + 1]), Half<T>::pack(x[8 * q + 2], x[8 * q + 3]), Half<T>::pack(x[8 * q + 4], x[8 * q + 5]),
                                           Half<T>::pack(x[8 * q + 6], x[8 * q + 7]));
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q) *reinterpret_cast<float4*>(stage + rr * 128 + ((q ^ (rr & 7)) << 4)) = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                    }
                }
                group_sync();
#pragma unroll
                for (int k = 0; k < 8; ++k) {             // a warp: its 32 rows, four at a time
                    const int row_in = (warp & 3) * 32 + k * 4 + (lane >> 3), piece = lane & 7, r_out = r - rr + row_in, g_out = r0 + r_out;
                    const int col = c0 + piece * (per / 8);
                    if (g_out >= all_rows || col >= a.dim) continue;
                    const uint4 y = *reinterpret_cast<const uint4*>(stage + row_in * 128 + ((piece ^ (row_in & 7)) << 4));
                    if (it.whole) {
                        const int nd = ta_node(a, g_out);
                        char* p = a.out + it.b * a.o_sb + nd * a.o_st + (it.h * a.group + g_out - nd * a.group) * a.o_sh + col * 2;
                        if (a.out_vec) *reinterpret_cast<uint4*>(p) = y;
                        else {
                            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int q = 0; q < 8; ++q) reinterpret_cast<unsigned short*>(p)[q] = (unsigned short)(w[q / 2] >> (q & 1) * 16);
                        }
                    } else {
                        *reinterpret_cast<uint4*>(a.part + (it.slot * ROWS + r_out) * a.dim + col) = y;
                    }
                }
                if (BUFFERS == 1) group_sync();
            }
            if (gr < all_rows && !it.whole) a.part_ml[it.slot * ROWS + r] = make_float2(m, l);
        }
        softmax_warps();                                  // queries and masks may be overwritten
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

}  // namespace
}  // namespace sd
