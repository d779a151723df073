// Attention of drafted trees over the caller's paged cache (contract: specdec.h): entry point, warp-level kernels, merge of split keys.
//
// out = sum_j p_j v_j over the keys a query sees, p = softmax(scale q . k).  One pass over the keys with the running maximum m and sum l of
// 2^(s - m): s in units of log2, sums and outputs in fp32, rescaled where m grows.  All query heads of a K/V head share its keys, so a row tile
// mixes nodes and heads; few rows: the keys of a sequence are split over CTAs, whose partial outputs k_ta_merge joins.
#include "barriers.cuh"
#include "tree_attention.cuh"

namespace sd {
namespace {

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
template <typename T> struct Half;
template <> struct Half<__nv_bfloat16> {
    static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <> struct Half<__half> {
    static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

// The mask rows of a tile's queries (cut at n_nodes), and any[w]: the nodes that one of them sees.  rows: query rows r0 ..; `words` a row.
__device__ void load_masks(const TreeAttn& a, int b, int r0, int rows, int nodes, uint32_t* mask, uint32_t* any) {
    for (int w = threadIdx.x; w < a.words; w += blockDim.x) any[w] = 0;
    __syncthreads();
    const int t0 = r0 / a.group, t1 = min((r0 + rows - 1) / a.group, a.T - 1);
    for (int i = threadIdx.x; i < (t1 - t0 + 1) * a.words; i += blockDim.x) {
        const int t = t0 + i / a.words, w = i % a.words;
        uint32_t m = t < nodes ? a.mask[b * a.mask_sb + (long long)t * a.words + w] : 0u;
        const int left = nodes - w * 32;
        if (left < 32) m &= left <= 0 ? 0u : (1u << left) - 1u;
        mask[i] = m;
        if (m) atomicOr(any + w, m);
    }
    __syncthreads();
}

// ------------------------------------------------------------------ 16-bit types: mma.sync
// CTA = (split, row tile, K/V head, sequence); WM x WK warps: 16 rows each, the WK key groups take every WK-th block of keys and merge at the end.  Each group
// walks its blocks through a ring of NS cp.async stages of its own.  Rows of DP elements, 16-byte pieces XORed with the row's low three bits.
template <typename T, int DP, int WM, int WK, int KT, int NS>
__global__ void __launch_bounds__(32 * WM * WK) k_ta_mma(TreeAttn a) {
    constexpr int ROWS = 16 * WM, PITCH = DP * 2, PIECES = DP / 8, GT = 32 * WM, STAGE = 2 * KT * PITCH;
    constexpr int NK = KT / 8, ND = DP / 8;
    extern __shared__ __align__(128) char sm[];
    char* ring = sm;                                      // [WK][NS][K, V][KT][PITCH]; at first the queries, at last the groups' partial outputs
    uint32_t* any = (uint32_t*)(sm + WK * NS * STAGE);
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % WM, wk = warp / WM, gt = tid % GT;
    const int split = blockIdx.x % a.splits, tile = blockIdx.x / a.splits, h = blockIdx.y, b = blockIdx.z;
    const int r0 = tile * ROWS, all_rows = a.T * a.group;
    const SeqKeys s = ta_keys(a, b);
    int per;
    const int used = ta_used(a, s.keys, per);
    if (split >= max(used, 1)) return;
    const int t0 = r0 / a.group;
    load_masks(a, b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);

    // queries: rows through shared memory into fragments
    {
        for (int i = tid; i < ROWS * PIECES; i += 32 * WM * WK) {
            const int r = i / PIECES, c = i % PIECES, gr = r0 + r;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (gr < all_rows && c * 8 < a.dim) {
                const char* p = a.q + b * a.q_sb + (gr / a.group) * a.q_st + (h * a.group + gr % a.group) * a.q_sh + c * 16;
                if (a.q_vec) x = *reinterpret_cast<const uint4*>(p);
                else {
                    const unsigned short* e = reinterpret_cast<const unsigned short*>(p);
                    x = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                }
            }
            *reinterpret_cast<uint4*>(ring + r * PITCH + ((c ^ (r & 7)) << 4)) = x;
        }
    }
    __syncthreads();
    uint32_t qf[DP / 16][4];
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) {
        const int r = wm * 16 + (lane & 15), c = kk * 2 + (lane >> 4);
        ldsm4(smem_u32(ring + r * PITCH + ((c ^ (r & 7)) << 4)), qf[kk]);
    }
    __syncthreads();

    const char* kbase = a.k + h * a.s_head;
    const char* vbase = a.v + h * a.s_head;
    char* my_ring = ring + wk * NS * STAGE;
    if (a.dim < DP) {                                     // pieces beyond the head: zero once, never written again
        for (int i = gt; i < NS * 2 * KT * PIECES; i += GT) {
            const int r = (i / PIECES) % KT, c = i % PIECES;
            if (c * 8 >= a.dim) *reinterpret_cast<uint4*>(my_ring + (i / PIECES) * PITCH + ((c ^ (r & 7)) << 4)) = make_uint4(0, 0, 0, 0);
        }
    }
    const int k_begin = split * per * TA_BLOCK, k_end = min(s.keys, (split + 1) * per * TA_BLOCK);
    const int blocks = (max(k_end - k_begin, 0) + KT - 1) / KT, mine = (blocks - wk + WK - 1) / WK;
    const int real_pieces = a.dim / 8;
    auto load = [&](int j) {                              // the group's j-th block
        if (j < mine) {
            const int k0 = k_begin + (j * WK + wk) * KT;
            char* st = my_ring + (j % NS) * STAGE;
            for (int i = gt; i < KT * PIECES; i += GT) {
                const int r = i / PIECES, c = i % PIECES, key = k0 + r;
                if (c >= real_pieces) continue;
                bool real = key < k_end;
                if (real && key >= s.len) real = any[(key - s.len) >> 5] >> ((key - s.len) & 31) & 1;
                const int pi = key >> a.page_shift;
                int page = -1;
                if (real && pi < a.max_pages) page = a.table[(long long)s.seq * a.max_pages + pi];
                real = real && (unsigned)page < (unsigned)a.n_pages;
                const long long off = real ? page * a.s_page + (key & ((1 << a.page_shift) - 1)) * a.s_token + c * 16 : 0;
                const uint32_t d = smem_u32(st + r * PITCH + ((c ^ (r & 7)) << 4));
                ta_copy16(d, kbase + off, real);
                ta_copy16(d + KT * PITCH, vbase + off, real);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto group_sync = [&]() {
        if constexpr (WM == 1) __syncwarp();
        else if constexpr (WK == 1) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + wk), "n"(GT) : "memory");
    };
    const int ra = wm * 16 + (lane >> 2), rb = ra + 8;
    const int ta = (r0 + ra) / a.group, tb = (r0 + rb) / a.group;
    const bool live_a = r0 + ra < all_rows && ta < s.nodes, live_b = r0 + rb < all_rows && tb < s.nodes;
    const uint32_t* mask_a = mask + (live_a ? ta - t0 : 0) * a.words;
    const uint32_t* mask_b = mask + (live_b ? tb - t0 : 0) * a.words;
    float o[ND][4];
#pragma unroll
    for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float ma = -INFINITY, mb = -INFINITY, la = 0.f, lb = 0.f;
    group_sync();
    for (int j = 0; j < NS - 1; ++j) load(j);
    for (int j = 0; j < mine; ++j) {
        asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
        group_sync();
        load(j + NS - 1);
        const uint32_t ks = smem_u32(my_ring + (j % NS) * STAGE), vs = ks + KT * PITCH;
        const int k0 = k_begin + (j * WK + wk) * KT;
        float sc[NK][4];
#pragma unroll
        for (int i = 0; i < NK; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
#pragma unroll
            for (int n = 0; n < KT / 16; ++n) {
                const int r = n * 16 + (lane & 7) + ((lane >> 4) << 3), c = kk * 2 + ((lane >> 3) & 1);
                uint32_t kf[4];
                ldsm4(ks + r * PITCH + ((c ^ (r & 7)) << 4), kf);
                Half<T>::mma(sc[2 * n], qf[kk], kf[0], kf[1]);
                Half<T>::mma(sc[2 * n + 1], qf[kk], kf[2], kf[3]);
            }
        if (k0 + KT > s.len) {                            // a block with nodes, or behind the last key
#pragma unroll
            for (int n = 0; n < KT / 32; ++n) {
                const int base = k0 + n * 32 - s.len;
                uint32_t wa = live_a ? ta_window(mask_a, a.words, base) : 0u, wb = live_b ? ta_window(mask_b, a.words, base) : 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int bit = i * 8 + (lane & 3) * 2;
                    float* c = sc[n * 4 + i];
                    if (!(wa >> bit & 1)) c[0] = -INFINITY;
                    if (!(wa >> bit & 2)) c[1] = -INFINITY;
                    if (!(wb >> bit & 1)) c[2] = -INFINITY;
                    if (!(wb >> bit & 2)) c[3] = -INFINITY;
                }
            }
        }
        float na = ma, nb = mb;
#pragma unroll
        for (int i = 0; i < NK; ++i) { na = fmaxf(na, fmaxf(sc[i][0], sc[i][1]) * a.scale); nb = fmaxf(nb, fmaxf(sc[i][2], sc[i][3]) * a.scale); }
        na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 1)); na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 2));
        nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 1)); nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 2));
        const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
        const float fa = ta_exp2(ma - za), fb = ta_exp2(mb - zb);
        ma = na; mb = nb;
        la *= fa; lb *= fb;
#pragma unroll
        for (int i = 0; i < ND; ++i) { o[i][0] *= fa; o[i][1] *= fa; o[i][2] *= fb; o[i][3] *= fb; }
#pragma unroll
        for (int n = 0; n < KT / 16; ++n) {
            uint32_t pf[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float* c = sc[2 * n + e];
                c[0] = ta_exp2(fmaf(c[0], a.scale, -za)); c[1] = ta_exp2(fmaf(c[1], a.scale, -za));
                c[2] = ta_exp2(fmaf(c[2], a.scale, -zb)); c[3] = ta_exp2(fmaf(c[3], a.scale, -zb));
                la += c[0] + c[1]; lb += c[2] + c[3];
                pf[2 * e] = Half<T>::pack(c[0], c[1]);
                pf[2 * e + 1] = Half<T>::pack(c[2], c[3]);
            }
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                const int r = n * 16 + (lane & 15), c = d * 2 + (lane >> 4);
                uint32_t vf[4];
                ldsm4_t(vs + r * PITCH + ((c ^ (r & 7)) << 4), vf);
                Half<T>::mma(o[2 * d], pf, vf[0], vf[1]);
                Half<T>::mma(o[2 * d + 1], pf, vf[2], vf[3]);
            }
        }
    }
    la += __shfl_xor_sync(0xffffffffu, la, 1); la += __shfl_xor_sync(0xffffffffu, la, 2);
    lb += __shfl_xor_sync(0xffffffffu, lb, 1); lb += __shfl_xor_sync(0xffffffffu, lb, 2);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // a query behind the nodes has taken the committed keys of blocks without a mask; one that sees nothing has multiplied values by 0
    if (!live_a) la = 0.f;
    if (!live_b) lb = 0.f;
    if (la == 0.f) { ma = -INFINITY;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = 0.f;
    }
    if (lb == 0.f) { mb = -INFINITY;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i][2] = o[i][3] = 0.f;
    }
    if constexpr (WK > 1) {                               // the groups' partial outputs meet in the first group
        constexpr int RP = DP + 8;
        float* red = reinterpret_cast<float*>(ring);      // [WK - 1][ROWS][RP], then [WK - 1][ROWS] (maximum, sum)
        float2* red_ml = reinterpret_cast<float2*>(red + (WK - 1) * ROWS * RP);
        static_assert((WK - 1) * ROWS * (RP * 4 + 8) <= WK * NS * STAGE, "partial outputs fit the ring");
        __syncthreads();
        if (wk > 0) {
            float* pa = red + ((wk - 1) * ROWS + ra) * RP + (lane & 3) * 2;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                *reinterpret_cast<float2*>(pa + i * 8) = make_float2(o[i][0], o[i][1]);
                *reinterpret_cast<float2*>(pa + 8 * RP + i * 8) = make_float2(o[i][2], o[i][3]);
            }
            if ((lane & 3) == 0) { red_ml[(wk - 1) * ROWS + ra] = make_float2(ma, la); red_ml[(wk - 1) * ROWS + rb] = make_float2(mb, lb); }
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int g = 0; g < WK - 1; ++g) {
            const float2 xa = red_ml[g * ROWS + ra], xb = red_ml[g * ROWS + rb];
            const float na = fmaxf(ma, xa.x), nb = fmaxf(mb, xb.x);
            const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
            const float fa = ta_exp2(ma - za), fb = ta_exp2(mb - zb), ga = ta_exp2(xa.x - za), gb = ta_exp2(xb.x - zb);
            ma = na; mb = nb;
            la = la * fa + xa.y * ga; lb = lb * fb + xb.y * gb;
            const float* pa = red + (g * ROWS + ra) * RP + (lane & 3) * 2;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const float2 u = *reinterpret_cast<const float2*>(pa + i * 8), w = *reinterpret_cast<const float2*>(pa + 8 * RP + i * 8);
                o[i][0] = o[i][0] * fa + u.x * ga; o[i][1] = o[i][1] * fa + u.y * ga;
                o[i][2] = o[i][2] * fb + w.x * gb; o[i][3] = o[i][3] * fb + w.y * gb;
            }
        }
    }
    if (used <= 1) {
        const float ia = la > 0.f || la != la ? 1.f / la : 0.f, ib = lb > 0.f || lb != lb ? 1.f / lb : 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int gr = r0 + (e ? rb : ra);
            if (gr >= all_rows) continue;
            char* p = a.out + b * a.o_sb + (gr / a.group) * a.o_st + (h * a.group + gr % a.group) * a.o_sh + (lane & 3) * 4;
            const float inv = e ? ib : ia;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                if (i * 8 >= a.dim) break;
                const uint32_t x = Half<T>::pack(o[i][2 * e] * inv, o[i][2 * e + 1] * inv);
                if (a.out_vec) *reinterpret_cast<uint32_t*>(p + i * 16) = x;
                else { reinterpret_cast<unsigned short*>(p + i * 16)[0] = (unsigned short)x; reinterpret_cast<unsigned short*>(p + i * 16)[1] = (unsigned short)(x >> 16); }
            }
        }
    } else {
        const long long slot = ((((long long)b * a.kv_heads + h) * a.tiles + tile) * a.splits + split) * ROWS;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = e ? rb : ra;
            float* p = a.part + (slot + r) * a.dim + (lane & 3) * 2;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                if (i * 8 >= a.dim) break;
                *reinterpret_cast<float2*>(p + i * 8) = make_float2(o[i][2 * e], o[i][2 * e + 1]);
            }
            if ((lane & 3) == 0) a.part_ml[slot + r] = make_float2(e ? mb : ma, e ? lb : la);
        }
    }
}

// ------------------------------------------------------------------ fp32: FFMA
// CTA of 128 threads = 16 rows x a split's blocks of 64 keys; keys and values pass through shared memory, scores between the two products too.
constexpr int TF_ROWS = 16, TF_KT = 64;
template <int DP>
__global__ void __launch_bounds__(128) k_ta_f32(TreeAttn a) {
    constexpr int KP = DP + 4, SP = TF_KT + 4;
    extern __shared__ __align__(128) char sm[];
    float* q = reinterpret_cast<float*>(sm);              // [16][KP]
    float* kt = q + TF_ROWS * KP;                         // [64][KP]
    float* vt = kt + TF_KT * KP;
    float* sc = vt + TF_KT * KP;                          // [16][SP]
    float* row_f = sc + TF_ROWS * SP;                     // [16] rescale, [16] maximum, [16] sum
    uint32_t* any = reinterpret_cast<uint32_t*>(row_f + 48);
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int split = blockIdx.x % a.splits, tile = blockIdx.x / a.splits, h = blockIdx.y, b = blockIdx.z;
    const int r0 = tile * TF_ROWS, all_rows = a.T * a.group;
    const SeqKeys s = ta_keys(a, b);
    int per;
    const int used = ta_used(a, s.keys, per);
    if (split >= max(used, 1)) return;
    load_masks(a, b, r0, min(TF_ROWS, all_rows - r0), s.nodes, mask, any);
    for (int i = tid; i < TF_ROWS * DP; i += 128) {
        const int r = i / DP, d = i % DP, gr = r0 + r;
        float x = 0.f;
        if (gr < all_rows && d < a.dim) x = *reinterpret_cast<const float*>(a.q + b * a.q_sb + (gr / a.group) * a.q_st + (h * a.group + gr % a.group) * a.q_sh + d * 4);
        q[r * KP + d] = x;
    }
    if (tid < 16) { row_f[16 + tid] = -INFINITY; row_f[32 + tid] = 0.f; }
    const int t0 = r0 / a.group;
    const int k_begin = split * per * TA_BLOCK, k_end = min(s.keys, (split + 1) * per * TA_BLOCK);
    constexpr int DC = DP / 4, RG = 128 / DC, RR = TF_ROWS / RG;           // output: DC column groups of 4, RG row groups of RR rows
    const int oc = tid % DC, og = tid / DC;
    float4 o[RR];
#pragma unroll
    for (int i = 0; i < RR; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = k_begin; k0 < k_end; k0 += TF_KT) {
        __syncthreads();
        for (int i = tid; i < TF_KT * (DP / 4); i += 128) {
            const int r = i / (DP / 4), c = i % (DP / 4), key = k0 + r;
            bool real = key < k_end && c * 4 < a.dim;
            if (real && key >= s.len) real = any[(key - s.len) >> 5] >> ((key - s.len) & 31) & 1;
            const int pi = key >> a.page_shift;
            int page = -1;
            if (real && pi < a.max_pages) page = a.table[(long long)s.seq * a.max_pages + pi];
            real = real && (unsigned)page < (unsigned)a.n_pages;
            const long long off = real ? page * a.s_page + (key & ((1 << a.page_shift) - 1)) * a.s_token + c * 16 + h * a.s_head : 0;
            ta_copy16(smem_u32(kt + r * KP + c * 4), a.k + off, real);
            ta_copy16(smem_u32(vt + r * KP + c * 4), a.v + off, real);
        }
        asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        {   // scores: key tid % 64, eight rows
            const int key = tid & 63, rr = (tid >> 6) * 8;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
            for (int d = 0; d < a.dim; d += 4) {
                const float4 kv = *reinterpret_cast<const float4*>(kt + key * KP + d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float4 qv = *reinterpret_cast<const float4*>(q + (rr + i) * KP + d);
                    x[i] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, x[i]))));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int gr = r0 + rr + i, t = gr / a.group, base = k0 + (key & 32) - s.len;
                const bool live = gr < all_rows && t < s.nodes;
                const uint32_t w = live ? ta_window(mask + (t - t0) * a.words, a.words, base) : 0u;
                sc[(rr + i) * SP + key] = (w >> (key & 31) & 1) && k0 + key < k_end ? x[i] * a.scale : -INFINITY;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {                     // running maximum and sum: four rows a warp
            const int r = warp * 4 + i;
            const float x = sc[r * SP + lane], y = sc[r * SP + lane + 32], m0 = row_f[16 + r];
            float m = fmaxf(x, y);
#pragma unroll
            for (int of = 16; of; of >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, of));
            m = fmaxf(m, m0);
            const float z = m == -INFINITY ? 0.f : m, p = exp2f(x - z), u = exp2f(y - z);
            sc[r * SP + lane] = p; sc[r * SP + lane + 32] = u;
            float l = p + u;
#pragma unroll
            for (int of = 16; of; of >>= 1) l += __shfl_xor_sync(0xffffffffu, l, of);
            if (lane == 0) { const float f = exp2f(m0 - z); row_f[r] = f; row_f[16 + r] = m; row_f[32 + r] = row_f[32 + r] * f + l; }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RR; ++i) { const float f = row_f[og * RR + i]; o[i].x *= f; o[i].y *= f; o[i].z *= f; o[i].w *= f; }
        const int kn = min(TF_KT, k_end - k0);
        for (int key = 0; key < kn; ++key) {
            const float4 v = *reinterpret_cast<const float4*>(vt + key * KP + oc * 4);
#pragma unroll
            for (int i = 0; i < RR; ++i) {
                const float p = sc[(og * RR + i) * SP + key];
                o[i].x = fmaf(p, v.x, o[i].x); o[i].y = fmaf(p, v.y, o[i].y); o[i].z = fmaf(p, v.z, o[i].z); o[i].w = fmaf(p, v.w, o[i].w);
            }
        }
    }
    __syncthreads();
    const long long slot = ((((long long)b * a.kv_heads + h) * a.tiles + tile) * a.splits + split) * TF_ROWS;
#pragma unroll
    for (int i = 0; i < RR; ++i) {
        const int r = og * RR + i, gr = r0 + r;
        if (gr >= all_rows || oc * 4 >= a.dim) continue;
        const float l = row_f[32 + r];
        if (l == 0.f) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);               // sees nothing: values times 0
        if (used <= 1) {
            const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
            float* p = reinterpret_cast<float*>(a.out + b * a.o_sb + (gr / a.group) * a.o_st + (h * a.group + gr % a.group) * a.o_sh) + oc * 4;
            if (a.out_vec) *reinterpret_cast<float4*>(p) = make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv);
            else { p[0] = o[i].x * inv; p[1] = o[i].y * inv; p[2] = o[i].z * inv; p[3] = o[i].w * inv; }
        } else {
            *reinterpret_cast<float4*>(a.part + (slot + r) * a.dim + oc * 4) = o[i];
            if (oc == 0) a.part_ml[slot + r] = make_float2(row_f[16 + r], l);
        }
    }
}

// ------------------------------------------------------------------ merge
template <typename T> __device__ __forceinline__ void put(char* p, float x);
template <> __device__ __forceinline__ void put<float>(char* p, float x) { *reinterpret_cast<float*>(p) = x; }
template <> __device__ __forceinline__ void put<__nv_bfloat16>(char* p, float x) { *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ void put<__half>(char* p, float x) { *reinterpret_cast<__half*>(p) = __float2half_rn(x); }

// One warp a query row: the splits' outputs, each rescaled to the largest maximum.
template <typename T>
__global__ void __launch_bounds__(128) k_ta_merge(TreeAttn a, int rows_per_tile) {
    const int gr = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31, h = blockIdx.y, b = blockIdx.z;
    if (gr >= a.T * a.group) return;
    int per;
    const int used = ta_used(a, ta_keys(a, b).keys, per);
    if (used <= 1) return;
    const int tile = gr / rows_per_tile, r = gr % rows_per_tile;
    const long long slot0 = (((long long)b * a.kv_heads + h) * a.tiles + tile) * a.splits * rows_per_tile + r;
    float m = -INFINITY;
    for (int s = lane; s < used; s += 32) m = fmaxf(m, a.part_ml[slot0 + (long long)s * rows_per_tile].x);
#pragma unroll
    for (int of = 16; of; of >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, of));
    const float z = m == -INFINITY ? 0.f : m;
    float o[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
    for (int s = 0; s < used; ++s) {
        const long long slot = slot0 + (long long)s * rows_per_tile;
        const float2 ml = a.part_ml[slot];
        const float f = exp2f(ml.x - z);
        l += ml.y * f;
#pragma unroll
        for (int i = 0; i < 4; ++i) if (lane + 32 * i < a.dim) o[i] = fmaf(a.part[slot * a.dim + lane + 32 * i], f, o[i]);
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    char* p = a.out + b * a.o_sb + (gr / a.group) * a.o_st + (h * a.group + gr % a.group) * a.o_sh;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (lane + 32 * i < a.dim) put<T>(p + (lane + 32 * i) * sizeof(T), o[i] * inv);
}

// ------------------------------------------------------------------ host
struct Plan { int rows, tiles, splits, min_blocks; };     // rows of a tile; see TreeAttn
Plan plan(int B, int T, int n_q_heads, int n_kv_heads, int dtype, long long max_keys) {
    const int all = T * (n_q_heads / n_kv_heads);
    Plan p;
    p.rows = dtype == SPECDEC_DTYPE_F32 ? TF_ROWS : all <= 16 ? 16 : all <= 32 ? 32 : 64;
    p.tiles = (all + p.rows - 1) / p.rows;
    const long long ctas = (long long)B * n_kv_heads * p.tiles, blocks = (max_keys + TA_BLOCK - 1) / TA_BLOCK;
    long long s = (4 * 148 + ctas - 1) / ctas;            // about four CTAs an SM
    p.min_blocks = 2;
    s = s < blocks / p.min_blocks ? s : blocks / p.min_blocks;
    p.splits = (int)(s < 1 ? 1 : s > 128 ? 128 : s);
    return p;
}
long long part_bytes(const Plan& p, int B, int n_kv_heads, int head_dim) {
    return p.splits <= 1 ? 0 : (long long)B * n_kv_heads * p.tiles * p.splits * p.rows * (head_dim * 4 + 8);
}

template <typename T, int DP, int WM, int WK, int KT, int NS>
cudaError_t run_mma(const TreeAttn& a, cudaStream_t st) {
    const size_t smem = (size_t)WK * NS * 2 * KT * DP * 2 + (size_t)(16 * WM + 1) * a.words * 4;
    const cudaError_t e = cudaFuncSetAttribute(k_ta_mma<T, DP, WM, WK, KT, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
    if (e != cudaSuccess) return e;
    k_ta_mma<T, DP, WM, WK, KT, NS><<<dim3(a.tiles * a.splits, a.kv_heads, a.B), 32 * WM * WK, smem, st>>>(a);
    return cudaGetLastError();
}
template <typename T, int DP>
cudaError_t run_half(const TreeAttn& a, int rows, cudaStream_t st) {
    if (rows == 16) return run_mma<T, DP, 1, 4, 32, 3>(a, st);
    if (rows == 32) return run_mma<T, DP, 2, 2, 32, 3>(a, st);
    return run_mma<T, DP, 4, 1, 64, 3>(a, st);
}
template <int DP>
cudaError_t run_f32(const TreeAttn& a, cudaStream_t st) {
    const size_t smem = ((size_t)(TF_ROWS + 2 * TF_KT) * (DP + 4) + TF_ROWS * (TF_KT + 4) + 48) * 4 + (size_t)(TF_ROWS + 1) * a.words * 4;
    const cudaError_t e = cudaFuncSetAttribute(k_ta_f32<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
    if (e != cudaSuccess) return e;
    k_ta_f32<DP><<<dim3(a.tiles * a.splits, a.kv_heads, a.B), 128, smem, st>>>(a);
    return cudaGetLastError();
}
template <typename T>
cudaError_t run_merge(const TreeAttn& a, int rows, cudaStream_t st) {
    k_ta_merge<T><<<dim3((a.T * a.group + 3) / 4, a.kv_heads, a.B), 128, 0, st>>>(a, rows);
    return cudaGetLastError();
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_tree_attention_workspace(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int dtype, int max_length) {
    if (B < 0 || T < 1 || T > 1024 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || head_dim < 8 || head_dim > 128 || head_dim % 8 ||
        !op_elem_bytes(dtype) || max_length < 0)
        return op_bad("tree_attention_workspace", "sizes that tree_attention does not take");
    if (B == 0) return 0;
    return part_bytes(plan(B, T, n_q_heads, n_kv_heads, dtype, (long long)max_length + T), B, n_kv_heads, head_dim);
}

int specdec_tree_attention(const specdec_cache* c, const specdec_tree_attention_args* g, void* stream) {
    const char* who = "tree_attention";
    if (!c || !g || !c->d_kv || !c->d_table || !c->d_length || (g->B && (!g->d_q || !g->d_out || !g->d_seqs || !g->d_mask))) return op_bad(who, "a pointer is NULL");
    const int e = op_elem_bytes(c->dtype);
    if (!e) return op_bad(who, "unknown dtype");
    if (g->B < 0 || g->B > 65535 || g->T < 1 || c->n_layers < 1 || g->layer < 0 || g->layer >= c->n_layers || c->n_heads < 1 || c->n_heads > 65535 ||
        g->n_q_heads < 1 || g->n_q_heads % c->n_heads || c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1 || g->max_length < 0)
        return op_bad(who, "a size is out of range, or the query heads are no multiple of the K/V heads");
    if (c->page_tokens < 1 || (c->page_tokens & (c->page_tokens - 1))) return op_bad(who, "page_tokens is not a power of two");
    if ((long long)c->max_pages * c->page_tokens > 0x7fffffffLL - 65536) return op_bad(who, "a sequence could pass 2^31 tokens");
    if (g->T > 1024) return op_fail(SPECDEC_ERR_CAPACITY, who, "trees have at most 1024 nodes");
    if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return op_fail(SPECDEC_ERR_UNSUPPORTED, who, "head_dim is no multiple of 8 up to 128");
    const long long st[5] = {c->stride_layer, c->stride_side, c->stride_page, c->stride_token, c->stride_head};
    for (long long s : st) if (s < 0 || s * e % 16) return op_bad(who, "a stride of the cache is negative or not a multiple of 16 bytes");
    if ((uintptr_t)c->d_kv % 16 || (uintptr_t)g->d_q % e || (uintptr_t)g->d_out % e) return op_bad(who, "d_kv is not 16-byte aligned, or q or out not to its type");
    if (!(g->scale > 0.f) || g->scale > 3e38f) return op_bad(who, "scale is not a positive number");
    if (g->B == 0) return SPECDEC_OK;
    TreeAttn a;
    a.q = (const char*)g->d_q; a.out = (char*)g->d_out;
    a.k = (const char*)c->d_kv + g->layer * c->stride_layer * e; a.v = a.k + c->stride_side * e;
    a.q_sb = g->q_stride_b * e; a.q_st = g->q_stride_t * e; a.q_sh = g->q_stride_h * e;
    a.o_sb = g->out_stride_b * e; a.o_st = g->out_stride_t * e; a.o_sh = g->out_stride_h * e;
    a.s_page = c->stride_page * e; a.s_token = c->stride_token * e; a.s_head = c->stride_head * e;
    a.table = c->d_table; a.length = c->d_length; a.held = c->d_held; a.seqs = g->d_seqs; a.n_nodes = g->d_n_nodes;
    a.mask = g->d_mask; a.mask_sb = g->mask_stride_b;
    a.n_pages = c->n_pages; a.n_seqs = c->n_seqs; a.max_pages = c->max_pages; a.page_shift = __builtin_ctz(c->page_tokens);
    const long long cap = (long long)c->max_pages * c->page_tokens;
    a.max_length = (int)(g->max_length && g->max_length < cap ? g->max_length : cap);
    a.T = g->T; a.words = (g->T + 31) / 32; a.group = g->n_q_heads / c->n_heads; a.kv_heads = c->n_heads; a.dim = c->head_dim; a.B = g->B;
    if ((long long)a.T * a.group > 1 << 20) return op_fail(SPECDEC_ERR_CAPACITY, who, "nodes times query heads of a K/V head pass 2^20");
    a.scale = g->scale * 1.4426950408889634f;
    a.q_vec = (((uintptr_t)g->d_q | a.q_sb | a.q_st | a.q_sh) & 15) == 0;
    a.out_vec = (((uintptr_t)g->d_out | a.o_sb | a.o_st | a.o_sh) & 15) == 0;
    const Plan p = plan(a.B, a.T, g->n_q_heads, c->n_heads, c->dtype, (long long)a.max_length + a.T);
    a.tiles = p.tiles; a.splits = p.splits; a.min_blocks = p.min_blocks;
    const long long need = part_bytes(p, a.B, c->n_heads, c->head_dim);
    if (need && (!g->d_workspace || (uintptr_t)g->d_workspace % 16 || g->workspace_bytes < need))
        return op_fail(SPECDEC_ERR_CAPACITY, who, "the workspace is smaller than specdec_tree_attention_workspace says, or not 16-byte aligned");
    a.part = (float*)g->d_workspace;
    a.part_ml = need ? (float2*)(a.part + (long long)a.B * a.kv_heads * a.tiles * a.splits * p.rows * a.dim) : nullptr;
    const cudaStream_t s = (cudaStream_t)stream;
    const bool wide = a.dim > 64;
    cudaError_t rc;
    if (c->dtype == SPECDEC_DTYPE_F32) rc = wide ? run_f32<128>(a, s) : run_f32<64>(a, s);
    else if (c->dtype == SPECDEC_DTYPE_BF16) rc = wide ? run_half<__nv_bfloat16, 128>(a, p.rows, s) : run_half<__nv_bfloat16, 64>(a, p.rows, s);
    else rc = wide ? run_half<__half, 128>(a, p.rows, s) : run_half<__half, 64>(a, p.rows, s);
    if (rc == cudaSuccess && need)
        rc = c->dtype == SPECDEC_DTYPE_F32 ? run_merge<float>(a, p.rows, s) : c->dtype == SPECDEC_DTYPE_BF16 ? run_merge<__nv_bfloat16>(a, p.rows, s) : run_merge<__half>(a, p.rows, s);
    return rc == cudaSuccess ? SPECDEC_OK : op_fail(SPECDEC_ERR_CUDA, who, cudaGetErrorString(rc));
}

}  // extern "C"
