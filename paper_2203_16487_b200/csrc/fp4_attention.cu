// Attention of drafted trees over a cache in 4 bits, few query rows: entry point, plan, mma.sync (contract: specdec.h, work: tree_attention.cuh).
//
// CTA = WM x WK consumer warps and one that loads.  A block of 64 keys is a stage of a ring: a bulk copy each of a page's codes and scales.  Warp (wm, wk) takes 16 rows and every WK-th block.
// Codes become fp16 in the registers of the lane whose fragment they are part of: values are exact, and nothing of 16 bits passes through shared memory, whose bandwidth
// (128 bytes a clock) is what a tile of fp16 in between would run into first (32 KB written and read for every 9 KB from HBM).
//
// Which channel and key stand where in a fragment is free as long as both operands agree:
//   scores (m16n8k16, B = keys): a lane's channels are D / 4 that follow one another, so that its codes of a key are one load (8 or 16 bytes); the queries are loaded the same way.
//   output (B = values): a lane's keys are those of its score columns, its columns D / 8 channels that follow one another; two keys' codes are paired by nibbles
//     (a shift and a select for four pairs), converted, and multiplied by the two keys' scales.
// Column c of eight keys is key c ^ (c >> 1 & 1) (D = 128) or c ^ (c >> 2 & 1) (D = 64): lanes that load together then hit different banks, or two lanes one.
//
// Probabilities are fp16, 2^15 times their value: a weight 2^-29 of the largest is still a normal number, so that a hundred thousand small ones add up.
#include "fp4_attention.cuh"

namespace sd {
namespace {

constexpr float P_SHIFT = 15.f;
// Two numbers as fp16, and what the rounding left.
__device__ __forceinline__ uint32_t half_pair(float x, float y) { return Half<__half>::pack(x, y); }
__device__ __forceinline__ uint32_t rest_pair(float x, float y, uint32_t h) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return Half<__half>::pack(x - f.x, y - f.y);
}

// Sixteen query rows of a warp: lane (g, t) = (lane / 4, lane % 4) holds rows g and g + 8, and of the output the channels D / 4 * t ...
template <typename T, int D> struct Fp4Rows {
    static constexpr bool WIDE = sizeof(T) == 4;          // fp32: queries and probabilities in two parts
    static constexpr int KK = D / 16, ND = D / 8, NK = TA_BLOCK / 8, PARTS = WIDE ? 2 : 1;
    uint32_t q[PARTS][KK][4];
    float o[ND][4], ma, mb, la, lb, sa, sb;               // s: scale of the row's scores
    // Row `e` (0: g, 1: g + 8) from its channels at p; times: what its scores are multiplied by.
    __device__ __forceinline__ void query(int e, const char* p, bool live, bool vec, float times) {
        float x[D / 4];
        constexpr int N = D / 4;
        if (!live) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = 0.f;
        } else if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float* f = reinterpret_cast<const float*>(p) + i;
                const float4 v = vec ? *reinterpret_cast<const float4*>(f) : make_float4(f[0], f[1], f[2], f[3]);
                x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 8) {
                const unsigned short* f = reinterpret_cast<const unsigned short*>(p) + i;
                uint4 v;
                if (vec) v = *reinterpret_cast<const uint4*>(f);
                else v = make_uint4(f[0] | f[1] << 16, f[2] | f[3] << 16, f[4] | f[5] << 16, f[6] | f[7] << 16);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (std::is_same<T, __half>::value) {
                        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(w + j));
                        x[i + 2 * j] = h.x; x[i + 2 * j + 1] = h.y;
                    } else {
                        x[i + 2 * j] = __uint_as_float(w[j] << 16); x[i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                    }
                }
            }
        }
        int shift = 0;
        if constexpr (!std::is_same<T, __half>::value) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(x[i]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1)); top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            shift = row_shift(top);
            const float f = power2(shift);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] *= f;
        }
        (e ? sb : sa) = times * power2(-shift);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float u = x[4 * kk + 2 * i], w = x[4 * kk + 2 * i + 1];
                q[0][kk][e + 2 * i] = half_pair(u, w);
                if constexpr (WIDE) q[PARTS - 1][kk][e + 2 * i] = rest_pair(u, w, q[0][kk][e + 2 * i]);
            }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        ma = mb = -INFINITY; la = lb = 0.f;
    }
    static __device__ __forceinline__ int key_of(int c) { return D == 128 ? c ^ (c >> 1 & 1) : c ^ (c >> 2 & 1); }
    // One block at st; window_a, window_b(base): what the rows see of 32 keys, asked where the block holds nodes or ends behind the last key
    template <typename WA, typename WB>
    __device__ __forceinline__ void block(const char* st, bool tail, int base0, WA window_a, WB window_b) {
        using Stage = Fp4Stage<D>;
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, x = D == 128 ? t & 1 : t >> 1;      // x: whether this lane's two columns are exchanged
        float sc[NK][4];
        const char* kc = st + key_of(g) * (D / 2) + t * (D / 8);
        const char* kq = st + Stage::KS + key_of(g) * (D / 16) + t * (D / 64);
#pragma unroll
        for (int n = 0; n < NK; ++n) {
            uint32_t w[D / 32], s2[2];
            if constexpr (D == 128) {
                const uint4 v = *reinterpret_cast<const uint4*>(kc + n * 8 * (D / 2));
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                const uint32_t s = fp4_scales2(*reinterpret_cast<const unsigned short*>(kq + n * 8 * (D / 16)));
                s2[0] = __byte_perm(s, s, 0x1010); s2[1] = __byte_perm(s, s, 0x3232);
            } else {
                const uint2 v = *reinterpret_cast<const uint2*>(kc + n * 8 * (D / 2));
                w[0] = v.x; w[1] = v.y;
                const uint32_t s = *reinterpret_cast<const unsigned char*>(kq + n * 8 * (D / 16));
                s2[0] = s2[1] = fp4_scales2(s | s << 8);
            }
            sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                uint32_t k[4];
                fp4_unpack8(w[i], k);
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = h2_mul(k[j], s2[D == 128 ? i >> 1 : 0]);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    Half<__half>::mma(sc[n], q[p][2 * i], k[0], k[1]);
                    Half<__half>::mma(sc[n], q[p][2 * i + 1], k[2], k[3]);
                }
            }
        }
        if (tail) {
#pragma unroll
            for (int n = 0; n < TA_BLOCK / 32; ++n) {
                const uint32_t wa = window_a(base0 + n * 32), wb = window_b(base0 + n * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int b0 = i * 8 + 2 * t + x, b1 = b0 ^ 1;
                    float* c = sc[n * 4 + i];
                    if (!(wa >> b0 & 1)) c[0] = -INFINITY;
                    if (!(wa >> b1 & 1)) c[1] = -INFINITY;
                    if (!(wb >> b0 & 1)) c[2] = -INFINITY;
                    if (!(wb >> b1 & 1)) c[3] = -INFINITY;
                }
            }
        }
        // (scaled ahead of the maximum: fused with its subtraction, a product's own rounding would be left where scores are beyond 2^27)
        float na = -INFINITY, nb = -INFINITY;
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            sc[i][0] *= sa; sc[i][1] *= sa; sc[i][2] *= sb; sc[i][3] *= sb;
            na = fmaxf(na, fmaxf(sc[i][0], sc[i][1])); nb = fmaxf(nb, fmaxf(sc[i][2], sc[i][3]));
        }
        na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 1)); na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 2));
        nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 1)); nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 2));
        na = fmaxf(ma, na); nb = fmaxf(mb, nb);
        const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
        if (__any_sync(0xffffffffu, na != ma || nb != mb)) {
            const float fa = ta_exp2(ma - za), fb = ta_exp2(mb - zb);
            la *= fa; lb *= fb;
#pragma unroll
            for (int i = 0; i < ND; ++i) { o[i][0] *= fa; o[i][1] *= fa; o[i][2] *= fb; o[i][3] *= fb; }
        }
        ma = na; mb = nb;
        const char* vc = st + Stage::V + (2 * t) * (D / 2) + g * (D / 16);
        const char* vq = st + Stage::VS + (2 * t) * (D / 16) + g * (D / 16) / 8;
#pragma unroll
        for (int n = 0; n < TA_BLOCK / 16; ++n) {
            uint32_t pf[PARTS][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float* c = sc[2 * n + e];
                c[0] = ta_exp2(c[0] - za + P_SHIFT); c[1] = ta_exp2(c[1] - za + P_SHIFT);
                c[2] = ta_exp2(c[2] - zb + P_SHIFT); c[3] = ta_exp2(c[3] - zb + P_SHIFT);
                pf[0][2 * e] = half_pair(c[0], c[1]);
                pf[0][2 * e + 1] = half_pair(c[2], c[3]);
                if constexpr (WIDE) {
                    pf[PARTS - 1][2 * e] = rest_pair(c[0], c[1], pf[0][2 * e]);
                    pf[PARTS - 1][2 * e + 1] = rest_pair(c[2], c[3], pf[0][2 * e + 1]);
                    la += c[0] + c[1]; lb += c[2] + c[3];
                } else {                                  // (the sum adds up the rounded ones: the weights add up to 1)
                    la = Half<__half>::add(la, pf[0][2 * e]); lb = Half<__half>::add(lb, pf[0][2 * e + 1]);
                }
            }
            // keys 2 t + x and 2 t + 1 - x of each eight
            uint32_t w[2][2][D / 64], s2[2];              // [eight][key][word]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r0 = n * 16 + e * 8 + x, r1 = n * 16 + e * 8 + 1 - x;
                if constexpr (D == 128) {
                    const uint2 u = *reinterpret_cast<const uint2*>(vc + r0 * (D / 2)), v = *reinterpret_cast<const uint2*>(vc + r1 * (D / 2));
                    w[e][0][0] = u.x; w[e][0][1] = u.y; w[e][1][0] = v.x; w[e][1][1] = v.y;
                } else {
                    w[e][0][0] = *reinterpret_cast<const uint32_t*>(vc + r0 * (D / 2)); w[e][1][0] = *reinterpret_cast<const uint32_t*>(vc + r1 * (D / 2));
                }
                s2[e] = fp4_scales2(*reinterpret_cast<const unsigned char*>(vq + r0 * (D / 16)) | (uint32_t)*reinterpret_cast<const unsigned char*>(vq + r1 * (D / 16)) << 8);
            }
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {            // eight channels
                uint32_t b[2][2][4];                      // [eight keys][even, odd channels][pair]
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t u = w[e][0][i], v = w[e][1][i];
                    fp4_unpack8((u & 0x0f0f0f0fu) | (v << 4 & 0xf0f0f0f0u), b[e][0]);
                    fp4_unpack8((u >> 4 & 0x0f0f0f0fu) | (v & 0xf0f0f0f0u), b[e][1]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { b[e][0][j] = h2_mul(b[e][0][j], s2[e]); b[e][1][j] = h2_mul(b[e][1][j], s2[e]); }
                }
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int j = 0; j < 8; ++j) Half<__half>::mma(o[8 * i + j], pf[p], b[0][j & 1][j >> 1], b[1][j & 1][j >> 1]);
            }
        }
    }
    // The lanes' sums together.  A query behind the nodes has taken the committed keys of blocks without a mask; one that sees nothing has multiplied values by 0.
    __device__ __forceinline__ void finish(bool live_a, bool live_b, float unit) {
        la += __shfl_xor_sync(0xffffffffu, la, 1); la += __shfl_xor_sync(0xffffffffu, la, 2);
        lb += __shfl_xor_sync(0xffffffffu, lb, 1); lb += __shfl_xor_sync(0xffffffffu, lb, 2);
        const bool none_a = !live_a || la == 0.f, none_b = !live_b || lb == 0.f;
        if (none_a) { ma = -INFINITY; la = 0.f; }
        if (none_b) { mb = -INFINITY; lb = 0.f; }
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            o[i][0] = none_a ? 0.f : o[i][0] * unit; o[i][1] = none_a ? 0.f : o[i][1] * unit;
            o[i][2] = none_b ? 0.f : o[i][2] * unit; o[i][3] = none_b ? 0.f : o[i][3] * unit;
        }
    }
    // This lane's D / 4 channels of row e, in order.
    __device__ __forceinline__ float channel(int e, int i) const { return i < ND ? o[i][2 * e] : o[i - ND][2 * e + 1]; }
    // Partial results in shared memory: rows of RP floats, and (maximum, sum) of each.
    static constexpr int RP = D + 4;
    __device__ __forceinline__ void leave(float* red, float2* red_ml, int ra) const {
        const int t = threadIdx.x & 3;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float* p = red + (ra + 8 * e) * RP + t * (D / 4);
#pragma unroll
            for (int i = 0; i < D / 4; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(channel(e, i), channel(e, i + 1), channel(e, i + 2), channel(e, i + 3));
            if (t == 0) red_ml[ra + 8 * e] = make_float2(e ? mb : ma, e ? lb : la);
        }
    }
    __device__ __forceinline__ void join(const float* red, const float2* red_ml, int ra) {
        const float2 xa = red_ml[ra], xb = red_ml[ra + 8];
        const float na = fmaxf(ma, xa.x), nb = fmaxf(mb, xb.x);
        const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
        const float fa = ta_exp2(ma - za), fb = ta_exp2(mb - zb), ea = ta_exp2(xa.x - za), eb = ta_exp2(xb.x - zb);
        ma = na; mb = nb;
        la = la * fa + xa.y * ea; lb = lb * fb + xb.y * eb;
        const float* pa = red + ra * RP + (threadIdx.x & 3) * (D / 4);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            o[i][0] = o[i][0] * fa + pa[i] * ea; o[i][1] = o[i][1] * fa + pa[ND + i] * ea;
            o[i][2] = o[i][2] * fb + pa[8 * RP + i] * eb; o[i][3] = o[i][3] * fb + pa[8 * RP + ND + i] * eb;
        }
    }
    // Rows ra and ra + 8 of a tile of `rows` that begins at query row r0: the output, or the part's partial results.
    __device__ __forceinline__ void store(const TreeAttn& a, const Part& it, int r0, int ra, int rows) const {
        const int t = threadIdx.x & 3;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = ra + 8 * e, gr = r0 + r;
            const float l = e ? lb : la;
            if (gr >= a.T * a.group) continue;
            if (!it.whole) {
                const long long slot = it.slot * rows + r;
                float* p = a.part + slot * D + t * (D / 4);
#pragma unroll
                for (int i = 0; i < D / 4; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(channel(e, i), channel(e, i + 1), channel(e, i + 2), channel(e, i + 3));
                if (t == 0) a.part_ml[slot] = make_float2(e ? mb : ma, l);
                continue;
            }
            const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
            const int node = ta_node(a, gr);
            char* p = a.out + it.b * a.o_sb + node * a.o_st + (it.h * a.group + gr - node * a.group) * a.o_sh + t * (D / 4) * (int)sizeof(T);
            if constexpr (WIDE) {
#pragma unroll
                for (int i = 0; i < D / 4; i += 4) {
                    const float4 v = make_float4(channel(e, i) * inv, channel(e, i + 1) * inv, channel(e, i + 2) * inv, channel(e, i + 3) * inv);
                    float* f = reinterpret_cast<float*>(p) + i;
                    if (a.out_vec) *reinterpret_cast<float4*>(f) = v;
                    else { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 4; i += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = Half<T>::pack(channel(e, i + 2 * j) * inv, channel(e, i + 2 * j + 1) * inv);
                    unsigned short* f = reinterpret_cast<unsigned short*>(p) + i;
                    if (a.out_vec) *reinterpret_cast<uint4*>(f) = make_uint4(w[0], w[1], w[2], w[3]);
                    else
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] = (unsigned short)(w[j / 2] >> (j & 1) * 16);
                }
            }
        }
    }
};

// Group wk has the stages wk, wk + WK, ... to itself and so waits for every phase of their barriers.
template <typename T, int D, int WM, int WK, int NS, int PER_SM>
__global__ void __launch_bounds__(32 * (WM * WK + 1), PER_SM) k_fp4_mma(Fp4Attn a) {
    static_assert(NS % WK == 0, "a stage serves one group");
    using Stage = Fp4Stage<D>;
    constexpr int WARPS = WM * WK, NG = NS / WK, ROWS = 16 * WM, KT = TA_BLOCK, STAGE = Stage::BYTES;
    extern __shared__ __align__(128) char fp4_smem[];
    __shared__ __align__(8) uint64_t bars[2 * NS];
    __shared__ int abort_flag;
    char* ring = fp4_smem;
    int4* seqs = (int4*)(ring + NS * STAGE);              // [B] where sequences are cut
    uint32_t* any = (uint32_t*)(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + (a.words + 3) / 4 * 4;         // (16-byte aligned, as the partial results behind it are)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t full = smem_u32(bars), empty = full + NS * 8;
    if (warp == WARPS && lane == 0) {
        for (int i = 0; i < NS; ++i) { mbar_init(full + i * 8, 1); mbar_init(empty + i * 8, WM); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    op_begin();
    TaWork work;
    work.begin(a, seqs);
    __syncthreads();

    if (warp == WARPS) {                                  // loads, running ahead into the next parts
        const int page = 1 << a.page_shift, box = min(page, KT), n_pages = KT / box;
        int count = 0;                                    // lane g: blocks that group g had in the parts before
        Part it, ahead;
        for (bool more = work.next(a, seqs, ahead); more;) {
            it = ahead;
            const int* table = a.table + (long long)it.s.seq * a.max_pages;
            auto page_of = [&](int j) {                   // this lane's page of block j: -1 where there is none
                const int key = it.k_begin + j * KT + lane * box, i = key >> a.page_shift;
                int p = -1;
                if (lane < n_pages && key < it.k_end && i < a.max_pages) p = table[i];
                return (unsigned)p < (unsigned)a.n_pages ? p : -1;
            };
            int p = it.blocks ? page_of(0) : 0;
            more = work.next(a, seqs, ahead);
            for (int j = 0; j < it.blocks; ++j) {
                const int g = j % WK, n = __shfl_sync(0xffffffffu, count, g) + j / WK, st = g + WK * (n % NG), key = it.k_begin + j * KT + lane * box, cur = p;
                if (j + 1 < it.blocks) p = page_of(j + 1);
                if (n >= NG && !mbar_wait_warp<true>(empty + st * 8, (n / NG - 1) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) return;
                char* to = ring + st * STAGE;
                const bool mine = lane < n_pages && key < it.k_end;
                if (mine && cur < 0)                      // a page that is none: zeros
                    for (int i = 0; i < box * D / 16; i += 16) {
                        *reinterpret_cast<uint4*>(to + Stage::KS + lane * box * (D / 16) + i) = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4*>(to + Stage::VS + lane * box * (D / 16) + i) = make_uint4(0, 0, 0, 0);
                    }
                const unsigned boxes = __popc(__ballot_sync(0xffffffffu, mine && cur >= 0));
                if (lane == 0) mbar_expect_tx(full + st * 8, boxes * box * (D + D / 8));
                __syncwarp();
                if (mine && cur >= 0) {
                    const int first = key & (page - 1);
                    const long long codes = cur * a.s_page + it.h * a.s_head + first * (D / 2), scales = cur * a.c_page + it.h * a.c_head + first * (D / 16);
                    const uint32_t d = smem_u32(to) + lane * box * (D / 2), s = smem_u32(to) + Stage::KS + lane * box * (D / 16), bar = full + st * 8;
                    bulk_copy(d, a.k + codes, box * (D / 2), bar);
                    bulk_copy(s, a.ks + scales, box * (D / 16), bar);
                    bulk_copy(d + Stage::V, a.v + codes, box * (D / 2), bar);
                    bulk_copy(s + Stage::SCALES, a.vs + scales, box * (D / 16), bar);
                }
            }
            count += (it.blocks - lane + WK - 1) / WK;    // (lanes below WK)
        }
        return;
    }

    const int wm = warp % WM, wk = warp / WM, all_rows = a.T * a.group;
    auto consumers = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); };
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
        Fp4Rows<T, D> rows;
        {
            const float times = a.unit_k ? a.scale * a.unit_k[it.h] : a.scale;
            const int c = (lane & 3) * (D / 4) * (int)sizeof(T);
            rows.query(0, a.q + it.b * a.q_sb + ta * a.q_st + (it.h * a.group + ga - ta * a.group) * a.q_sh + c, live_a, a.q_vec, times);
            rows.query(1, a.q + it.b * a.q_sb + tb * a.q_st + (it.h * a.group + gb - tb * a.group) * a.q_sh + c, live_b, a.q_vec, times);
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
            ta_load_masks<32 * WARPS, 1>(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
        }
        const uint32_t* mask_a = mask + (live_a ? ta - t0 : 0) * a.words;
        const uint32_t* mask_b = mask + (live_b ? tb - t0 : 0) * a.words;
        auto window_a = [&](int base) { return !live_a ? 0u : own ? ta_window2(ma[0], ma[1], base) : ta_window(mask_a, a.words, base); };
        auto window_b = [&](int base) { return !live_b ? 0u : own ? ta_window2(mb[0], mb[1], base) : ta_window(mask_b, a.words, base); };
        rows.clear();
        for (int j = wk; j < it.blocks; j += WK, ++count) {
            const int st = wk + WK * (count % NG), k0 = it.k_begin + j * KT;
            if (!mbar_wait_warp<true>(full + st * 8, (count / NG) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) break;
            char* at = ring + st * STAGE;
            const bool tail = k0 + KT > s.len;            // nodes, or what is behind the last key
            if (tail) {                                   // scales of values that no query sees: whatever they are, such values are multiplied by 0
                for (int r = wm * (KT / WM) + lane; r < (wm + 1) * (KT / WM); r += 32) {
                    const int base = k0 + (r & ~31) - s.len;
                    const uint32_t w = own ? ta_window2(seen[0], seen[1], base) : ta_window(any, a.words, base);
                    if (!(w >> (r & 31) & 1)) {
                        if constexpr (D == 128) *reinterpret_cast<uint2*>(at + Stage::VS + r * 8) = make_uint2(0, 0);
                        else *reinterpret_cast<uint32_t*>(at + Stage::VS + r * 4) = 0;
                    }
                }
                if constexpr (WM == 1) __syncwarp();
                else asm volatile("bar.sync %0, %1;" ::"r"(2 + wk), "n"(32 * WM) : "memory");
            }
            rows.block(at, tail, k0 - s.len, window_a, window_b);
            if (tail) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the zeros, ahead of the stage's next copies
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + st * 8);
        }
        rows.finish(live_a, live_b, a.unit_v ? a.unit_v[it.h] : 1.f);
        if constexpr (WK > 1) {                           // the groups' results meet in the first group
            constexpr int RP = Fp4Rows<T, D>::RP;
            float* red = reinterpret_cast<float*>(mask + (ROWS * a.words + 3) / 4 * 4);      // [ROWS][RP], then [ROWS] (maximum, sum): one group's at a time, so that more CTAs fit an SM
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

// ------------------------------------------------------------------ host
struct Plan { int rows, tiles, per_sm, direct, ctas, unit, min_blocks; long long grid, slots; };       // see TreeAttn; slots of partial results
constexpr int per_sm_of(int dtype, int dim, int rows) { return rows >= 128 ? 1 : dim == 128 || dtype == SPECDEC_DTYPE_F32 ? 2 : 3; }
Plan plan(int B, int T, int n_q_heads, int n_kv_heads, int dtype, int head_dim, long long max_keys) {
    const int all = T * (n_q_heads / n_kv_heads);
    Plan p;
    const int most_mma = head_dim > 64 ? 32 : 64;
    p.rows = all <= 16 ? 16 : all <= 32 ? 32 : all <= most_mma || dtype == SPECDEC_DTYPE_F32 ? 64 : all <= 128 || !fp4_tc_fits(head_dim, 256, T, n_q_heads / n_kv_heads) ? 128 : 256;
    p.tiles = (all + p.rows - 1) / p.rows;
    p.unit = p.rows >= 128 ? 128 : TA_BLOCK;
    p.min_blocks = 4;
    const long long columns = (long long)n_kv_heads * p.tiles, whole = B * columns, blocks = (max_keys + p.unit - 1) / p.unit;
    p.per_sm = per_sm_of(dtype, head_dim, p.rows);
    const int at_once = TA_SMS * p.per_sm;
    // Whole sequences take their rounds of CTAs times the longest's blocks, stretches an equal share of all blocks and the merge.
    p.direct = (whole + at_once - 1) / at_once * blocks <= whole * blocks / at_once + 8 || B > TA_MAX_B;
    if (p.direct && whole > at_once && 2 * columns <= at_once && B <= TA_MAX_B && p.rows >= 64 && blocks >= 4) p.direct = 2;
    p.ctas = (int)(at_once / columns < 1 ? 1 : at_once / columns);
    const long long most = (B * blocks + p.min_blocks - 1) / p.min_blocks;                // stretches at most
    if (p.ctas > most) p.ctas = (int)most;
    p.grid = p.direct ? whole : p.ctas * columns;
    p.slots = p.direct ? 0 : (p.ctas + B) * columns;
    return p;
}
// Bytes: partial outputs, then (maximum, sum), then where a tile's parts are.
long long part_floats(const Plan& p, int head_dim) { return p.slots * p.rows * head_dim; }
long long workspace(const Plan& p, int B, int n_kv_heads, int head_dim) {
    return p.direct ? 0 : part_floats(p, head_dim) * 4 + p.slots * p.rows * 8 + (long long)B * n_kv_heads * p.tiles * 8;
}

template <typename T, int D, int WM, int WK, int NS, int PER_SM>
cudaError_t run(const Fp4Attn& a, int grid, cudaStream_t st) {
    constexpr int ROWS = 16 * WM, RED = (WK > 1) * ROWS * (Fp4Rows<T, D>::RP * 4 + 8);
    auto bytes = [](int words, int B) { return NS * Fp4Stage<D>::BYTES + RED + ((words + 3) / 4 + (ROWS * words + 3) / 4) * 16 + B * 16; };
    static_assert(NS * Fp4Stage<D>::BYTES + RED + (ROWS + 1) * 128 + TA_MAX_B * 16 + 1024 <= 232448 / PER_SM, "shared memory of an SM");
    if (const cudaError_t e = op_allow<k_fp4_mma<T, D, WM, WK, NS, PER_SM>>(bytes(32, TA_MAX_B))) return e;
    return op_launch(k_fp4_mma<T, D, WM, WK, NS, PER_SM>, dim3(ta_grid(a, grid, PER_SM * TA_SMS)), 32 * (WM * WK + 1), bytes(a.words, a.direct == 1 ? 0 : a.B), st, 1, a);
}
template <typename T>
cudaError_t pick(const Fp4Attn& a, int rows, int grid, cudaStream_t st) {
    constexpr int P = sizeof(T) == 4 ? 2 : 3;
    if (a.dim > 64) return rows == 16 ? run<T, 128, 1, 3, 9, 2>(a, grid, st) : rows == 32 ? run<T, 128, 2, 2, 8, 2>(a, grid, st) : run<T, 128, 4, 1, 6, 2>(a, grid, st);
    return rows == 16 ? run<T, 64, 1, 4, 8, P>(a, grid, st) : rows == 32 ? run<T, 64, 2, 2, 8, P>(a, grid, st) : run<T, 64, 4, 1, 6, P>(a, grid, st);
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_packed_attention_workspace(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int dtype, int page_tokens, int max_length) {
    if (B < 0 || T < 1 || T > 1024 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128) || !op_elem_bytes(dtype) ||
        page_tokens < FP4_MIN_PAGE || max_length < 0)
        return op_bad("packed_attention_workspace", "sizes that packed_attention does not take");
    if (B == 0) return 0;
    // Unknown lengths: the longest.  Sequences are cut into the more parts the longer they are, and never where they need not be cut however long they are.
    return workspace(plan(B, T, n_q_heads, n_kv_heads, dtype, head_dim, (max_length ? max_length : 0x7fffffffLL) + T), B, n_kv_heads, head_dim);
}

int specdec_packed_attention(const specdec_packed_cache* f, const specdec_tree_attention_args* g, int dtype, void* stream) {
    const char* who = "packed_attention";
    if (const char* why = fp4_why_not(f)) return op_bad(who, why);
    const specdec_cache* c = &f->codes;
    if (!g || (g->B && (!g->d_q || !g->d_out || !g->d_seqs || !g->d_mask))) return op_bad(who, "a pointer is NULL");
    const int e = op_elem_bytes(dtype);
    if (!e) return op_bad(who, "unknown dtype");
    if (g->B < 0 || g->B > 65535 || g->T < 1 || g->layer < 0 || g->layer >= c->n_layers || c->n_heads > 65535 || g->n_q_heads < 1 || g->n_q_heads % c->n_heads || g->max_length < 0)
        return op_bad(who, "a size is out of range, or the query heads are no multiple of the K/V heads");
    if (g->T > 1024) return op_fail(SPECDEC_ERR_CAPACITY, who, "trees have at most 1024 nodes");
    if ((uintptr_t)g->d_q % e || (uintptr_t)g->d_out % e) return op_bad(who, "q or out is not aligned to its type");
    if (!(g->scale > 0.f) || g->scale > 3e38f) return op_bad(who, "scale is not a positive number");
    if (g->B == 0) return SPECDEC_OK;
    Fp4Attn a;
    a.q = (const char*)g->d_q; a.out = (char*)g->d_out;
    a.s_page = op_stride(c->stride_page, c->n_pages); a.s_head = op_stride(c->stride_head, c->n_heads); a.s_token = c->head_dim / 2;
    a.c_page = op_stride(f->scale_stride_page, c->n_pages); a.c_head = op_stride(f->scale_stride_head, c->n_heads);
    a.k = (const char*)c->d_kv + g->layer * op_stride(c->stride_layer, c->n_layers); a.v = a.k + c->stride_side;
    a.ks = (const char*)f->d_scales + g->layer * op_stride(f->scale_stride_layer, c->n_layers); a.vs = a.ks + f->scale_stride_side;
    a.unit_k = f->d_unit ? f->d_unit + (long long)g->layer * 2 * c->n_heads : nullptr; a.unit_v = f->d_unit ? a.unit_k + c->n_heads : nullptr;
    a.q_sb = op_stride(g->q_stride_b, g->B) * e; a.q_st = op_stride(g->q_stride_t, g->T) * e; a.q_sh = op_stride(g->q_stride_h, g->n_q_heads) * e;
    a.o_sb = op_stride(g->out_stride_b, g->B) * e; a.o_st = op_stride(g->out_stride_t, g->T) * e; a.o_sh = op_stride(g->out_stride_h, g->n_q_heads) * e;
    a.table = c->d_table; a.length = c->d_length; a.status = c->d_status; a.seqs = g->d_seqs; a.n_nodes = g->d_n_nodes;
    a.mask = g->d_mask; a.mask_sb = g->mask_stride_b;
    a.n_pages = c->n_pages; a.n_seqs = c->n_seqs; a.max_pages = c->max_pages; a.page_shift = __builtin_ctz(c->page_tokens);
    const long long cap = (long long)c->max_pages * c->page_tokens;
    a.max_length = (int)(g->max_length && g->max_length < cap ? g->max_length : cap);
    a.T = g->T; a.words = (g->T + 31) / 32; a.group = g->n_q_heads / c->n_heads; a.kv_heads = c->n_heads; a.dim = c->head_dim; a.B = g->B;
    a.group_mul = a.group > 1 ? (uint32_t)(0x100000000ULL / a.group + 1) : 0;
    if ((long long)a.T * a.group * a.group > 0x7fffffffLL || a.T * a.group > 1 << 20) return op_fail(SPECDEC_ERR_CAPACITY, who, "too many query heads for each K/V head");
    a.scale = g->scale * 1.4426950408889634f;
    a.q_vec = (((uintptr_t)g->d_q | a.q_sb | a.q_st | a.q_sh) & 15) == 0;
    a.out_vec = (((uintptr_t)g->d_out | a.o_sb | a.o_st | a.o_sh) & 15) == 0;
    const Plan p = plan(a.B, a.T, g->n_q_heads, c->n_heads, dtype, a.dim, (long long)a.max_length + a.T);
    if (p.grid > 0x7fffffff || p.slots > 0x7fffffff || (long long)a.B * a.kv_heads * a.T * a.group > 0x7fffffff - 65536) return op_fail(SPECDEC_ERR_CAPACITY, who, "too many sequences, heads and nodes for one launch");
    a.tiles = p.tiles; a.direct = p.direct; a.ctas = p.ctas; a.unit = p.unit; a.min_blocks = p.min_blocks;
    const long long need = workspace(p, a.B, c->n_heads, c->head_dim);
    if (need && (!g->d_workspace || (uintptr_t)g->d_workspace % 16 || g->workspace_bytes < need))
        return op_fail(SPECDEC_ERR_CAPACITY, who, "the workspace is smaller than specdec_packed_attention_workspace says, or not 16-byte aligned");
    a.part = (float*)g->d_workspace;
    a.part_ml = (float2*)(a.part + part_floats(p, a.dim));
    a.where = (int2*)(a.part_ml + p.slots * p.rows);
    const cudaStream_t s = (cudaStream_t)stream;
    const int grid = (int)p.grid;
    cudaError_t rc = p.rows >= 128 ? fp4_tc(a, dtype, p.rows, grid, s) : dtype == SPECDEC_DTYPE_F32 ? pick<float>(a, p.rows, grid, s) : dtype == SPECDEC_DTYPE_BF16 ? pick<__nv_bfloat16>(a, p.rows, grid, s) : pick<__half>(a, p.rows, grid, s);
    if (rc == cudaSuccess && need) rc = ta_merge(a, dtype, p.rows, s);
    return op_done(who, rc);
}

}  // extern "C"
