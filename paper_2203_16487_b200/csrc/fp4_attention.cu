// Attention of drafted trees over a cache in 4 bits, few query rows: entry point, plan, mma.sync (contract: specdec.h, work: tree_attention.cuh).
//
// CTA = WM x WK consumer warps and one that loads.  A block of 64 keys is a stage of a ring: a bulk copy each of a page's codes and scales.  Warp (wm, wk) takes 8 NT rows and every WK-th block.
// Codes become fp16 in the registers of the lane whose fragment they are part of: values are exact, and nothing of 16 bits passes through shared memory, whose bandwidth
// (128 bytes a clock) is what a tile of fp16 in between would run into first (32 KB written and read for every 9 KB from HBM).
//
// The cache is the A operand of both products (m16n8k16: sixteen keys or channels), queries and probabilities are B, so that rows come in eights: a group of four query heads wastes half of a
// fragment, not three quarters.  What is unpacked once serves NT products.  Which channel and key stand where in a fragment is free as long as both operands agree:
//   scores: a lane's channels are D / 4 that follow one another, so that its codes of a key are one load (8 or 16 bytes); the queries are loaded the same way.
//   output: a lane's keys are those of the probabilities' columns (the scores, transposed in eights by movmatrix), its channels D / 8 that follow one another; two keys' codes are paired by
//     nibbles (a shift and a select for four pairs), converted, and multiplied by the two keys' scales.
// Row c of eight keys is key c ^ (c >> 1 & 1) (D = 128) or c ^ (c >> 2 & 1) (D = 64): lanes that load values together then hit different banks, or two lanes one.
//
// Probabilities are fp16, 2^15 times their value: a weight 2^-29 of the largest is still a normal number, so that a hundred thousand small ones add up.  Their sum is one more product, with ones:
// of the rounded ones, so that the weights add up to 1.
//
// What bounds it is instructions: 4 x 1 query, 32/8 heads of 128, over 65,537 to 131,071 keys (544 MB) 124 us with the merge, 4.4 TB/s; its loads alone 100, its products alone 103; issue 55 %.
// (Over 16 bits two such sequences, 978 MB, take 151.)
#include "fp4_attention.cuh"

namespace sd {
namespace {

constexpr float P_SHIFT = 15.f;
__device__ __forceinline__ uint32_t half_pair(float x, float y) { return Half<__half>::pack(x, y); }
__device__ __forceinline__ uint32_t rest_pair(float x, float y, uint32_t h) {             // what the rounding has left
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return Half<__half>::pack(x - f.x, y - f.y);
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {                               // of 8 x 8 numbers, lane (g, t) has [g][2 t], [g][2 t + 1]
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// 8 NT query rows of a warp, lane (g, t) = (lane / 4, lane % 4).  It loads row g of each eight, and has scores and outputs of rows 2 t and 2 t + 1: of the output the channels D / 8 * g ...
template <typename T, int D, int NT> struct Fp4Rows {
    static constexpr bool WIDE = sizeof(T) == 4;          // fp32: queries and probabilities in two parts
    static constexpr int KK = D / 16, MD = D / 16, MK = TA_BLOCK / 16, PARTS = WIDE ? 2 : 1;
    uint32_t q[PARTS][NT][KK][2];
    float o[NT][MD][4], l[NT][4], m[NT][2], s[NT][2];     // l: sums in [0], [1]; s: scale of the row's scores
    // Eight rows: row g from this lane's channels at p; times: what scores are multiplied by.
    __device__ __forceinline__ void query(int n, const char* p, bool live, bool vec, float times) {
        constexpr int N = D / 4;
        float x[N];
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
        const float mine = times * power2(-shift);
        s[n][0] = __shfl_sync(0xffffffffu, mine, (threadIdx.x & 3) * 8); s[n][1] = __shfl_sync(0xffffffffu, mine, (threadIdx.x & 3) * 8 + 4);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float u = x[4 * kk + 2 * i], w = x[4 * kk + 2 * i + 1];
                q[0][n][kk][i] = half_pair(u, w);
                if constexpr (WIDE) q[PARTS - 1][n][kk][i] = rest_pair(u, w, q[0][n][kk][i]);
            }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < MD; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
            l[n][0] = l[n][1] = l[n][2] = l[n][3] = 0.f;
            m[n][0] = m[n][1] = -INFINITY;
        }
    }
    static __device__ __forceinline__ int key_of(int c) { return D == 128 ? c ^ (c >> 1 & 1) : c ^ (c >> 2 & 1); }
    // One block at st; window(n, e, base): what row 2 t + e of the n-th eight sees of 32 keys, asked where the block holds nodes or ends behind the last key
    template <typename W>
    __device__ __forceinline__ void block(const char* st, bool tail, int base0, W window) {
        using Stage = Fp4Stage<D>;
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, x = D == 128 ? t & 1 : t >> 1;      // x: whether keys 2 t and 2 t + 1 are exchanged
        float sc[NT][MK][4];
        const char* kc = st + key_of(g) * (D / 2) + t * (D / 8);
        const char* kq = st + Stage::CODES + key_of(g) * (D / 16) + t * (D / 64);
#pragma unroll
        for (int i = 0; i < MK; ++i) {
            uint32_t w[2][D / 32], s2[2][2];              // [key g, g + 8 of sixteen]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const char* c = kc + (i * 16 + e * 8) * (D / 2);
                const char* z = kq + (i * 16 + e * 8) * (D / 16);
                if constexpr (D == 128) {
                    const uint4 v = *reinterpret_cast<const uint4*>(c);
                    w[e][0] = v.x; w[e][1] = v.y; w[e][2] = v.z; w[e][3] = v.w;
                    const uint32_t f = fp4_scales2(*reinterpret_cast<const unsigned short*>(z));
                    s2[e][0] = __byte_perm(f, f, 0x1010); s2[e][1] = __byte_perm(f, f, 0x3232);
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(c);
                    w[e][0] = v.x; w[e][1] = v.y;
                    const uint32_t f = *reinterpret_cast<const unsigned char*>(z);
                    s2[e][0] = s2[e][1] = fp4_scales2(f | f << 8);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[n][i][0] = sc[n][i][1] = sc[n][i][2] = sc[n][i][3] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                uint32_t k[2][4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    fp4_unpack8(w[e][j], k[e]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) k[e][u] = h2_mul(k[e][u], s2[e][D == 128 ? j >> 1 : 0]);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t f[4] = {k[0][2 * h], k[1][2 * h], k[0][2 * h + 1], k[1][2 * h + 1]};
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
#pragma unroll
                        for (int n = 0; n < NT; ++n) Half<__half>::mma(sc[n][i], f, q[p][n][2 * j + h][0], q[p][n][2 * j + h][1]);
                }
            }
        }
        if (tail) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t w = window(n, e, base0 + h * 32) >> key_of(g);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if (!(w >> (i * 16) & 1)) sc[n][2 * h + i][e] = -INFINITY;
                            if (!(w >> (i * 16 + 8) & 1)) sc[n][2 * h + i][2 + e] = -INFINITY;
                        }
                    }
        }
        // (all rows' maxima side by side, and one vote for all: the lanes' exchanges are what a block waits for)
        float top[NT][2], f[NT][2];
        bool huge = false, grown = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[n][e] = -INFINITY;
#pragma unroll
                for (int i = 0; i < MK; ++i) top[n][e] = fmaxf(top[n][e], fmaxf(sc[n][i][e], sc[n][i][2 + e]));
            }
#pragma unroll
        for (int of = 4; of < 32; of <<= 1)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) top[n][e] = fmaxf(top[n][e], __shfl_xor_sync(0xffffffffu, top[n][e], of));
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                f[n][e] = s[n][e];
                top[n][e] = fmaxf(m[n][e], top[n][e] * f[n][e]);
                huge |= fabsf(top[n][e]) > 1048576.f && fabsf(top[n][e]) < INFINITY;
                grown |= top[n][e] != m[n][e];
            }
        // 2^(score * f + z) = 2^P_SHIFT * 2^(score - maximum).  Fused, the products leave what the maximum's rounding has cut off, and z is rounded too: nothing to speak of, but where scores are huge either
        // is more than fp16 has room for above 2^P_SHIFT.  There the products are rounded as the maximum was, which is taken off before the shift is put on.
        float z[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) z[n][e] = P_SHIFT - (top[n][e] == -INFINITY ? 0.f : top[n][e]);
        if (__any_sync(0xffffffffu, huge)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float y = top[n][e] == -INFINITY ? 0.f : top[n][e];
#pragma unroll
                    for (int i = 0; i < MK; ++i) { sc[n][i][e] = __fsub_rn(__fmul_rn(sc[n][i][e], f[n][e]), y); sc[n][i][2 + e] = __fsub_rn(__fmul_rn(sc[n][i][2 + e], f[n][e]), y); }
                    f[n][e] = 1.f; z[n][e] = P_SHIFT;
                }
        }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float fa = ta_exp2(m[n][0] - (top[n][0] == -INFINITY ? 0.f : top[n][0])), fb = ta_exp2(m[n][1] - (top[n][1] == -INFINITY ? 0.f : top[n][1]));
                l[n][0] *= fa; l[n][1] *= fb;
#pragma unroll
                for (int i = 0; i < MD; ++i) { o[n][i][0] *= fa; o[n][i][1] *= fb; o[n][i][2] *= fa; o[n][i][3] *= fb; }
                m[n][0] = top[n][0]; m[n][1] = top[n][1];
            }
        }
        uint32_t pf[PARTS][NT][MK][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int i = 0; i < MK; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float u = ta_exp2(fmaf(sc[n][i][2 * h], f[n][0], z[n][0])), v = ta_exp2(fmaf(sc[n][i][2 * h + 1], f[n][1], z[n][1]));
                    const uint32_t y = half_pair(u, v);
                    pf[0][n][i][h] = transpose8(y);
                    if constexpr (WIDE) pf[PARTS - 1][n][i][h] = transpose8(rest_pair(u, v, y));
                }
        }
        const char* vc = st + Stage::HALF + (2 * t) * (D / 2) + g * (D / 16);
        const char* vq = st + Stage::HALF + Stage::CODES + (2 * t) * (D / 16) + g * (D / 16) / 8;
#pragma unroll
        for (int i = 0; i < MK; ++i) {
            // keys 2 t + x and 2 t + 1 - x of each eight
            uint32_t w[2][2][D / 64], s2[2];              // [eight][key][word]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r0 = i * 16 + e * 8 + x, r1 = i * 16 + e * 8 + 1 - x;
                if constexpr (D == 128) {
                    const uint2 u = *reinterpret_cast<const uint2*>(vc + r0 * (D / 2)), v = *reinterpret_cast<const uint2*>(vc + r1 * (D / 2));
                    w[e][0][0] = u.x; w[e][0][1] = u.y; w[e][1][0] = v.x; w[e][1][1] = v.y;
                } else {
                    w[e][0][0] = *reinterpret_cast<const uint32_t*>(vc + r0 * (D / 2)); w[e][1][0] = *reinterpret_cast<const uint32_t*>(vc + r1 * (D / 2));
                }
                s2[e] = fp4_scales2(*reinterpret_cast<const unsigned char*>(vq + r0 * (D / 16)) | (uint32_t)*reinterpret_cast<const unsigned char*>(vq + r1 * (D / 16)) << 8);
            }
            const uint32_t ones[4] = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int n = 0; n < NT; ++n) Half<__half>::mma(l[n], ones, pf[p][n][i][0], pf[p][n][i][1]);
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {            // eight channels
                uint32_t b[2][2][4];                      // [eight keys][even, odd channels][pair]
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t u = w[e][0][j], v = w[e][1][j];
                    fp4_unpack8((u & 0x0f0f0f0fu) | (v << 4 & 0xf0f0f0f0u), b[e][0]);
                    fp4_unpack8((u >> 4 & 0x0f0f0f0fu) | (v & 0xf0f0f0f0u), b[e][1]);
#pragma unroll
                    for (int h = 0; h < 4; ++h) { b[e][0][h] = h2_mul(b[e][0][h], s2[e]); b[e][1][h] = h2_mul(b[e][1][h], s2[e]); }
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) {             // channels 2 h and 2 h + 1 of them
                    const uint32_t f[4] = {b[0][0][h], b[0][1][h], b[1][0][h], b[1][1][h]};
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
#pragma unroll
                        for (int n = 0; n < NT; ++n) Half<__half>::mma(o[n][4 * j + h], f, pf[p][n][i][0], pf[p][n][i][1]);
                }
            }
        }
    }
    // A query behind the nodes has taken the committed keys of blocks without a mask; one that sees nothing has multiplied values by 0.
    template <typename L>
    __device__ __forceinline__ void finish(L live, float unit) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool none = !live(n, e) || l[n][e] == 0.f;
                if (none) { m[n][e] = -INFINITY; l[n][e] = 0.f; }
#pragma unroll
                for (int i = 0; i < MD; ++i) { o[n][i][e] = none ? 0.f : o[n][i][e] * unit; o[n][i][2 + e] = none ? 0.f : o[n][i][2 + e] * unit; }
            }
    }
    // This lane's D / 8 channels of a row, in order.
    __device__ __forceinline__ float channel(int n, int e, int i) const { return o[n][i / 2][(i & 1) * 2 + e]; }
    // Partial results in shared memory: rows of RP floats from row r0 on, and (maximum, sum) of each.
    [[maybe_unused]] static constexpr int RP = D + 4;
    __device__ __forceinline__ void leave(float* red, float2* red_ml, int r0) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = r0 + n * 8 + 2 * t + e;
                float* p = red + r * RP + g * (D / 8);
#pragma unroll
                for (int i = 0; i < D / 8; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(channel(n, e, i), channel(n, e, i + 1), channel(n, e, i + 2), channel(n, e, i + 3));
                if (g == 0) red_ml[r] = make_float2(m[n][e], l[n][e]);
            }
    }
    __device__ __forceinline__ void join(const float* red, const float2* red_ml, int r0) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = r0 + n * 8 + 2 * t + e;
                const float2 y = red_ml[r];
                const float top = fmaxf(m[n][e], y.x), z = top == -INFINITY ? 0.f : top, f = ta_exp2(m[n][e] - z), h = ta_exp2(y.x - z);
                m[n][e] = top; l[n][e] = l[n][e] * f + y.y * h;
                const float* p = red + r * RP + g * (D / 8);
#pragma unroll
                for (int i = 0; i < MD; ++i) { o[n][i][e] = o[n][i][e] * f + p[2 * i] * h; o[n][i][2 + e] = o[n][i][2 + e] * f + p[2 * i + 1] * h; }
            }
    }
    // Rows w0 ... of a tile of `rows` that begins at query row r0: the output, or the part's partial results.
    __device__ __forceinline__ void store(const TreeAttn& a, const Part& it, int r0, int w0, int rows) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        constexpr int N = D / 8;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = w0 + n * 8 + 2 * t + e, gr = r0 + r;
                if (gr >= a.T * a.group) continue;
                if (!it.whole) {
                    const long long slot = it.slot * rows + r;
                    float* p = a.part + slot * D + g * N;
#pragma unroll
                    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(channel(n, e, i), channel(n, e, i + 1), channel(n, e, i + 2), channel(n, e, i + 3));
                    if (g == 0) a.part_ml[slot] = make_float2(m[n][e], l[n][e]);
                    continue;
                }
                const float inv = l[n][e] > 0.f || l[n][e] != l[n][e] ? 1.f / l[n][e] : 0.f;
                const int node = ta_node(a, gr);
                char* p = a.out + it.b * a.o_sb + node * a.o_st + (it.h * a.group + gr - node * a.group) * a.o_sh + g * N * (int)sizeof(T);
                if constexpr (WIDE) {
#pragma unroll
                    for (int i = 0; i < N; i += 4) {
                        const float4 v = make_float4(channel(n, e, i) * inv, channel(n, e, i + 1) * inv, channel(n, e, i + 2) * inv, channel(n, e, i + 3) * inv);
                        float* f = reinterpret_cast<float*>(p) + i;
                        if (a.out_vec) *reinterpret_cast<float4*>(f) = v;
                        else { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; i += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = Half<T>::pack(channel(n, e, i + 2 * j) * inv, channel(n, e, i + 2 * j + 1) * inv);
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

// The loading warp: blocks of the CTA's parts in order, running ahead into the next parts.  Block j of a part goes to group j % WK, which has the stages j % WK, j % WK + WK, ... to itself.
template <int D, int WK, int NS>
__device__ __forceinline__ void fp4_load(const Fp4Attn& a, TaWork work, const int4* seqs, char* ring, uint32_t full, uint32_t empty, int* abort_flag) {
    using Stage = Fp4Stage<D>;
    constexpr int KT = TA_BLOCK, NG = NS / WK, STAGE = Stage::BYTES;
    const int lane = threadIdx.x & 31;
    const int page = 1 << a.page_shift, box = min(page, KT), n_pages = KT / box;
    // What a lane copies of a block: lane / 4-th page's codes of keys, of values, scales of keys, of values
    const int page_of = lane >> 2;
    const bool scales = lane & 2, values = lane & 1;
    const char* base = scales ? (values ? a.vs : a.ks) : values ? a.v : a.k;
    const long long s_page = scales ? a.c_page : a.s_page, s_head = scales ? a.c_head : a.s_head;
    const int size = box * (scales ? D / 16 : D / 2), at = (scales ? Stage::CODES : 0) + (values ? Stage::HALF : 0) + page_of * size;
    int count = 0;                                    // lane g: blocks that group g had in the parts before
    Part it, ahead;
    // This lane's page of the 32 from the b0-th of a part on; -1 where there is none.  Asked for 32 at a time and well ahead: a lookup a block, waited for, is 0.7 us a block.
    auto pages_of = [&](const Part& part, int b0) {
        const int key = part.k_begin + (b0 + lane) * box, i = key >> a.page_shift;
        int p = -1;
        if (key < part.k_end && i < a.max_pages) p = a.table[(long long)part.s.seq * a.max_pages + i];
        return (unsigned)p < (unsigned)a.n_pages ? p : -1;
    };
    bool more = work.next(a, seqs, ahead);
    int first = more ? pages_of(ahead, 0) : 0;
    while (more) {
        it = ahead;
        int now = first, then = pages_of(it, 32);
        more = work.next(a, seqs, ahead);
        if (more) first = pages_of(ahead, 0);
        for (int j = 0; j < it.blocks; ++j) {
            const int g = j % WK, n = __shfl_sync(0xffffffffu, count, g) + j / WK, st = g + WK * (n % NG), b0 = j * n_pages, key = it.k_begin + (b0 + page_of) * box;
            if (b0 && b0 % 32 == 0) { now = then; then = pages_of(it, b0 + 32); }
            const int cur = __shfl_sync(0xffffffffu, now, (b0 + page_of) % 32);
            if (n >= NG && !mbar_wait_warp<true>(empty + st * 8, (n / NG - 1) & 1, abort_flag, a.status, SPECDEC_CACHE_TIMEOUT)) return;
            char* to = ring + st * STAGE + at;
            const bool mine = lane < 4 * n_pages && key < it.k_end, real = mine && cur >= 0;
            if (mine && cur < 0 && scales) {          // a page that is none: zeros, ahead of what the stage's next block brings
                for (int i = 0; i < size; i += 16) *reinterpret_cast<uint4*>(to + i) = make_uint4(0, 0, 0, 0);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            __syncwarp();
            const unsigned pieces = __popc(__ballot_sync(0xffffffffu, real));          // four a page
            if (lane == 0) mbar_expect_tx(full + st * 8, pieces / 4 * box * (D + D / 8));
            __syncwarp();
            if (real) bulk_copy(smem_u32(to), base + cur * s_page + it.h * s_head + (key & (page - 1)) * (scales ? D / 16 : D / 2), size, full + st * 8);
        }
        count += (it.blocks - lane + WK - 1) / WK;    // (lanes below WK)
    }
}

// Group wk has the stages wk, wk + WK, ... to itself and so waits for every phase of their barriers.
template <typename T, int D, int NT, int WM, int WK, int NS, int PER_SM>
__global__ void __launch_bounds__(32 * (WM * WK + 1), PER_SM) k_fp4_mma(Fp4Attn a) {
    static_assert(NS % WK == 0, "a stage serves one group");
    using Stage = Fp4Stage<D>;
    constexpr int WARPS = WM * WK, NG = NS / WK, ROWS = 8 * NT * WM, KT = TA_BLOCK, STAGE = Stage::BYTES;
    extern __shared__ __align__(128) char fp4_smem[];
    __shared__ __align__(8) uint64_t bars[2 * NS];
    __shared__ int abort_flag, left_in[WK];               // stage that holds a group's partial results
    char* ring = fp4_smem;
    int4* seqs = (int4*)(ring + NS * STAGE);              // [B] where sequences are cut
    uint32_t* any = (uint32_t*)(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + a.words;
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

    if (warp == WARPS) { fp4_load<D, WK, NS>(a, work, seqs, ring, full, empty, &abort_flag); return; }

    const int wm = warp % WM, wk = warp / WM, all_rows = a.T * a.group;
    auto consumers = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); };
    int count = 0;                                        // this group's blocks so far
    Part it, ahead;
    for (bool more = work.next(a, seqs, ahead, tid == 0); more;) {
        it = ahead;
        more = work.next(a, seqs, ahead, tid == 0);
        const SeqKeys& s = it.s;
        const int r0 = it.tile * ROWS, t0 = ta_node(a, r0), w0 = wm * 8 * NT;
        Fp4Rows<T, D, NT> rows;
        auto live = [&](int n, int e) {                   // this lane's rows
            const int gr = r0 + w0 + n * 8 + 2 * (lane & 3) + e;
            return gr < all_rows && ta_node(a, gr) < s.nodes;
        };
        // The nodes that anyone sees, asked for ahead of the queries.  Up to 64 nodes: in every warp's own registers (anyone: any query of the tree), so that no warp waits for another; more:
        // in shared memory.
        const bool own = a.words <= 2;
        const uint32_t* words = a.mask + it.b * a.mask_sb;
        uint32_t seen[2] = {0, 0};
        if (own) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (w < a.words && lane < s.nodes) seen[w] = words[lane * a.words + w];
                if (w < a.words && lane + 32 < s.nodes) seen[w] |= words[(lane + 32) * a.words + w];
            }
        }
        auto query_at = [&](const Part& part, int n) {
            const int gr = part.tile * ROWS + w0 + n * 8 + (lane >> 2), node = ta_node(a, gr);
            return a.q + part.b * a.q_sb + node * a.q_st + (part.h * a.group + gr - node * a.group) * a.q_sh + (lane & 3) * (D / 4) * (int)sizeof(T);
        };
        auto query_live = [&](const Part& part, int n) { const int gr = part.tile * ROWS + w0 + n * 8 + (lane >> 2); return gr < all_rows && ta_node(a, gr) < part.s.nodes; };
        const float times = a.unit_k ? a.scale * a.unit_k[it.h] : a.scale;
#pragma unroll
        for (int n = 0; n < NT; ++n) rows.query(n, query_at(it, n), query_live(it, n), a.q_vec, times);
        if (more)                                         // the next part's queries, on their way to the second-level cache
#pragma unroll
            for (int n = 0; n < NT; ++n) if (query_live(ahead, n)) asm volatile("prefetch.global.L2 [%0];" ::"l"(query_at(ahead, n)));
        if (own) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int left = s.nodes - w * 32;
                seen[w] = __reduce_or_sync(0xffffffffu, seen[w]) & (left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u);
            }
        } else {
            ta_load_masks<32 * WARPS, 1>(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
        }
        auto window = [&](int n, int e, int base) {       // (a row's own words: from the first-level cache, where they are from a moment ago; in registers they cost more)
            if (!live(n, e)) return 0u;
            const int node = ta_node(a, r0 + w0 + n * 8 + 2 * (lane & 3) + e);
            return own ? ta_window2(words[node * a.words] & seen[0], a.words > 1 ? words[node * a.words + 1] & seen[1] : 0u, base) : ta_window(mask + (node - t0) * a.words, a.words, base);
        };
        rows.clear();
        int left = -1;
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
            char* at = ring + st * STAGE;
            const bool tail = k0 + KT > s.len;            // nodes, or what is behind the last key
            if (tail) {                                   // scales of values that no query sees: whatever they are, such values are multiplied by 0
                for (int r = wm * (KT / WM) + lane; r < (wm + 1) * (KT / WM); r += 32) {
                    const int base = k0 + (r & ~31) - s.len;
                    const uint32_t w = own ? ta_window2(seen[0], seen[1], base) : ta_window(any, a.words, base);
                    if (!(w >> (r & 31) & 1)) {
                        if constexpr (D == 128) *reinterpret_cast<uint2*>(at + Stage::HALF + Stage::CODES + r * 8) = make_uint2(0, 0);
                        else *reinterpret_cast<uint32_t*>(at + Stage::HALF + Stage::CODES + r * 4) = 0;
                    }
                }
                if constexpr (WM == 1) __syncwarp();
                else asm volatile("bar.sync %0, %1;" ::"r"(2 + wk), "n"(32 * WM) : "memory");
            }
            rows.block(at, tail, k0 - s.len, window);
            if (tail) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the zeros, ahead of the stage's next copies
            __syncwarp();
            if (WK > 1 && wk > 0 && j + WK >= it.blocks) left = st;                    // (the group's last block here: its place is taken by the partial results)
            else if (lane == 0) mbar_arrive(empty + st * 8);
        }
        rows.finish(live, a.unit_v ? a.unit_v[it.h] : 1.f);
        if constexpr (WK > 1) {                           // the groups' results meet in the first group: [ROWS][RP] floats, then [ROWS] (maximum, sum), in a stage of each group
            constexpr int RP = Fp4Rows<T, D, NT>::RP;
            static_assert(ROWS * (RP * 4 + 8) <= STAGE, "a stage holds a group's partial results");
            if (wk > 0) {
                if (WM > 1) asm volatile("bar.sync %0, %1;" ::"r"(2 + wk), "n"(32 * WM) : "memory");       // (the group's other warps may still read it)
                if (left >= 0) { float* red = reinterpret_cast<float*>(ring + left * STAGE); rows.leave(red, reinterpret_cast<float2*>(red + ROWS * RP), w0); }
                if (wm == 0 && lane == 0) left_in[wk] = left;
            }
            consumers();
            if (wk == 0)
                for (int g = 1; g < WK; ++g)
                    if (left_in[g] >= 0) { const float* red = reinterpret_cast<const float*>(ring + left_in[g] * STAGE); rows.join(red, reinterpret_cast<const float2*>(red + ROWS * RP), w0); }
        }
        if (wk == 0) rows.store(a, it, r0, w0, ROWS);
        if (WK > 1 || !own) consumers();                  // masks and partial results may be overwritten
        if (WK > 1 && left >= 0) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + left * 8);
        }
    }
}

// ------------------------------------------------------------------ 33 to 64 rows of 64-wide heads
// Four warps of sixteen rows over the same blocks would each unpack all of a block (128 x 51 queries over 51 to 307 keys 39 us against 30); here each unpacks a quarter, into a tile of fp16 in shared memory,
// and the products read that (ldmatrix; rows of 128 bytes, 16-byte pieces XORed with the row's low three bits).  Two tiles: a warp that has met the others at a block's barrier knows that the tile
// of the block before has been read.
template <typename T> struct Fp4Tile : TaRows<T, 64> {
    using Base = TaRows<T, 64>;
    using Base::o; using Base::ma; using Base::mb; using Base::la; using Base::lb;
    static constexpr int NK = TA_BLOCK / 8, ND = 8;
    // As TaRows::block, but operands are fp16, rows have scales of their own, and probabilities are 2^15 times their value.
    template <typename W>
    __device__ __forceinline__ void tile(const uint32_t (*qf)[4], uint32_t ks, uint32_t vs, bool tail, int base0, float sa, float sb, W window) {
        const int lane = threadIdx.x & 31;
        auto at = [](uint32_t side, int r, int c) { return side + r * 128 + ((c ^ (r & 7)) << 4); };
        float sc[NK][4];
#pragma unroll
        for (int i = 0; i < NK; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int n = 0; n < TA_BLOCK / 16; ++n) {
                uint32_t x[4];
                ta_ldsm4(at(ks, n * 16 + (lane & 7) + ((lane >> 4) << 3), kk * 2 + ((lane >> 3) & 1)), x);
                Half<__half>::mma(sc[2 * n], qf[kk], x[0], x[1]);
                Half<__half>::mma(sc[2 * n + 1], qf[kk], x[2], x[3]);
            }
        if (tail) {
#pragma unroll
            for (int n = 0; n < TA_BLOCK / 32; ++n) {
                const uint32_t wa = window(0, base0 + n * 32), wb = window(1, base0 + n * 32);
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
        float na = -INFINITY, nb = -INFINITY;
#pragma unroll
        for (int i = 0; i < NK; ++i) { na = fmaxf(na, fmaxf(sc[i][0], sc[i][1])); nb = fmaxf(nb, fmaxf(sc[i][2], sc[i][3])); }
        na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 1)); nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 1));
        na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 2)); nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 2));
        na = fmaxf(ma, na * sa); nb = fmaxf(mb, nb * sb);
        const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
        float ua = P_SHIFT - za, ub = P_SHIFT - zb;
        auto huge = [](float x) { return fabsf(x) > 1048576.f && fabsf(x) < INFINITY; };
        if (__any_sync(0xffffffffu, huge(na) || huge(nb))) {            // (as in Fp4Rows)
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                sc[i][0] = __fsub_rn(__fmul_rn(sc[i][0], sa), za); sc[i][1] = __fsub_rn(__fmul_rn(sc[i][1], sa), za);
                sc[i][2] = __fsub_rn(__fmul_rn(sc[i][2], sb), zb); sc[i][3] = __fsub_rn(__fmul_rn(sc[i][3], sb), zb);
            }
            sa = sb = 1.f;
            ua = ub = P_SHIFT;
        }
        const float fa = ta_exp2(ma - za), fb = ta_exp2(mb - zb);
        ma = na; mb = nb;
        la *= fa; lb *= fb;
#pragma unroll
        for (int i = 0; i < ND; ++i) { o[i][0] *= fa; o[i][1] *= fa; o[i][2] *= fb; o[i][3] *= fb; }
#pragma unroll
        for (int n = 0; n < TA_BLOCK / 16; ++n) {
            uint32_t pf[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float* c = sc[2 * n + e];
                c[0] = ta_exp2(fmaf(c[0], sa, ua)); c[1] = ta_exp2(fmaf(c[1], sa, ua));
                c[2] = ta_exp2(fmaf(c[2], sb, ub)); c[3] = ta_exp2(fmaf(c[3], sb, ub));
                pf[2 * e] = half_pair(c[0], c[1]);
                pf[2 * e + 1] = half_pair(c[2], c[3]);
                la = Half<__half>::add(la, pf[2 * e]); lb = Half<__half>::add(lb, pf[2 * e + 1]);
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t x[4];
                ta_ldsm4_t(at(vs, n * 16 + (lane & 15), d * 2 + (lane >> 4)), x);
                Half<__half>::mma(o[2 * d], pf, x[0], x[1]);
                Half<__half>::mma(o[2 * d + 1], pf, x[2], x[3]);
            }
        }
    }
};

template <typename T, int NS, int PER_SM>
__global__ void __launch_bounds__(160, PER_SM) k_fp4_tile(Fp4Attn a) {
    using Stage = Fp4Stage<64>;
    constexpr int ROWS = 64, KT = TA_BLOCK, STAGE = Stage::BYTES, SIDE = KT * 128;
    extern __shared__ __align__(128) char fp4_smem[];
    __shared__ __align__(8) uint64_t bars[2 * NS];
    __shared__ int abort_flag;
    char* tiles = fp4_smem;                               // [2][keys, values][64][128]
    char* ring = tiles + 4 * SIDE;
    int4* seqs = (int4*)(ring + NS * STAGE);              // [B] where sequences are cut
    uint32_t* any = (uint32_t*)(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t full = smem_u32(bars), empty = full + NS * 8;
    if (warp == 4 && lane == 0) {
        for (int i = 0; i < NS; ++i) { mbar_init(full + i * 8, 1); mbar_init(empty + i * 8, 4); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    op_begin();
    TaWork work;
    work.begin(a, seqs);
    __syncthreads();
    if (warp == 4) { fp4_load<64, 1, NS>(a, work, seqs, ring, full, empty, &abort_flag); return; }

    const int all_rows = a.T * a.group;
    auto together = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    int count = 0;                                        // blocks so far
    Part it;
    while (work.next(a, seqs, it, tid == 0)) {
        const SeqKeys& s = it.s;
        const int r0 = it.tile * ROWS, t0 = ta_node(a, r0), ra = warp * 16 + (lane >> 2), ga = r0 + ra, gb = ga + 8, ta = ta_node(a, ga), tb = ta_node(a, gb);
        const bool live_a = ga < all_rows && ta < s.nodes, live_b = gb < all_rows && tb < s.nodes;
        const bool own = a.words <= 2;                    // as in k_fp4_mma
        const uint32_t* words = a.mask + it.b * a.mask_sb;
        uint32_t seen[2] = {0, 0}, see[2][2] = {{0, 0}, {0, 0}};
        if (own) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (w < a.words && lane < s.nodes) seen[w] = words[lane * a.words + w];
                if (w < a.words && lane + 32 < s.nodes) seen[w] |= words[(lane + 32) * a.words + w];
                if (w < a.words && live_a) see[0][w] = words[ta * a.words + w];
                if (w < a.words && live_b) see[1][w] = words[tb * a.words + w];
            }
        }
        // the queries as fragments: fp16, rows scaled by powers of two
        uint32_t qf[4][4];
        float sa = a.unit_k ? a.scale * a.unit_k[it.h] : a.scale, sb = sa;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bool live = e ? live_b : live_a;
            const int gr = e ? gb : ga, node = e ? tb : ta;
            const char* p = a.q + it.b * a.q_sb + node * a.q_st + (it.h * a.group + gr - node * a.group) * a.q_sh + (lane & 3) * 4;
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = 0;
                if (live) w[i] = a.q_vec ? *reinterpret_cast<const uint32_t*>(p + i * 16) : reinterpret_cast<const unsigned short*>(p + i * 16)[0] | (uint32_t)reinterpret_cast<const unsigned short*>(p + i * 16)[1] << 16;
            }
            if constexpr (!std::is_same<T, __half>::value) {
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1)); top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int shift = row_shift(top);
                const float f = power2(shift);
                (e ? sb : sa) *= power2(-shift);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = half_pair(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) qf[i >> 1][e + 2 * (i & 1)] = w[i];
        }
        if (own) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int left = s.nodes - w * 32;
                seen[w] = __reduce_or_sync(0xffffffffu, seen[w]) & (left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u);
            }
        } else {
            ta_load_masks<128, 1>(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
        }
        auto window = [&](int e, int base) {
            if (!(e ? live_b : live_a)) return 0u;
            return own ? ta_window2(see[e][0] & seen[0], see[e][1] & seen[1], base) : ta_window(mask + ((e ? tb : ta) - t0) * a.words, a.words, base);
        };
        Fp4Tile<T> rows;
        rows.clear();
        for (int j = 0; j < it.blocks; ++j, ++count) {
            const int st = count % NS, k0 = it.k_begin + j * KT;
            const bool tail = k0 + KT > s.len, ok = mbar_wait_warp<true>(full + st * 8, (count / NS) & 1, &abort_flag, a.status, SPECDEC_CACHE_TIMEOUT);
            const char* at = ring + st * STAGE;
            char* to = tiles + (count & 1) * 2 * SIDE;
            // keys of this warp: sixteen, a lane half a key's codes: four pieces of eight channels.  Values that no query sees: zeros, whatever is there is multiplied by 0
            const int r = warp * 16 + (lane >> 1), half = lane & 1;
            bool there = true;
            if (tail) {
                const int base = k0 + (r & ~31) - s.len;
                there = (own ? ta_window2(seen[0], seen[1], base) : ta_window(any, a.words, base)) >> (r & 31) & 1;
            }
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const uint4 c = *reinterpret_cast<const uint4*>(at + side * Stage::HALF + r * 32 + half * 16);
                uint32_t z = fp4_scales2(*reinterpret_cast<const unsigned short*>(at + side * Stage::HALF + Stage::CODES + r * 4 + half * 2));
                if (side && !there) z = 0;
                const uint32_t z2[2] = {__byte_perm(z, z, 0x1010), __byte_perm(z, z, 0x3232)}, w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t x[4];
                    fp4_unpack8(w[q], x);
                    *reinterpret_cast<uint4*>(to + side * SIDE + r * 128 + (((half * 4 + q) ^ (r & 7)) << 4)) =
                        make_uint4(h2_mul(x[0], z2[q >> 1]), h2_mul(x[1], z2[q >> 1]), h2_mul(x[2], z2[q >> 1]), h2_mul(x[3], z2[q >> 1]));
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + st * 8);
            together();
            if (!ok) continue;                            // (the others wait at the barrier)
            rows.tile(qf, smem_u32(to), smem_u32(to) + SIDE, tail, k0 - s.len, sa, sb, window);
        }
        rows.finish(live_a, live_b);
        const float unit = a.unit_v ? a.unit_v[it.h] : 1.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) rows.o[i][e] *= unit;
        rows.store(a, it, r0, ra, ROWS);
        together();                                       // masks, and the tile of the next block but one, may be overwritten
    }
}

// ------------------------------------------------------------------ host
struct Plan { int rows, tiles, per_sm, direct, ctas, unit, min_blocks; long long grid, slots; };       // see TreeAttn; slots of partial results
// CTAs that an SM holds, as pick has them.
constexpr int per_sm_of(int dtype, int dim, int rows) {
    if (rows >= 128) return 1;
    if (dtype == SPECDEC_DTYPE_F32) return dim > 64 ? (rows == 64 ? 1 : 2) : rows <= 16 ? 3 : 2;
    return rows == 8 && dim == 64 ? 4 : 3;
}
Plan plan(int B, int T, int n_q_heads, int n_kv_heads, int dtype, int head_dim, long long max_keys) {
    const int all = T * (n_q_heads / n_kv_heads);
    Plan p;
    // 33 to 64 rows of 128-wide heads by eight warps of eight rows, each unpacking all of a block: 16 x 51 queries over 300 to 1000 keys 39 us, by tcgen05 28; of 64-wide heads by tcgen05
    // 128 x 51 queries 64 us, by k_fp4_tile 30.  256 rows that share what is unpacked against twice 128: 8 x 64 queries, 32/8 heads, 152 and 224 us; 100 x 256 over 10 to 60 keys 117 and 145.
    const int most_mma = head_dim > 64 ? 32 : 64;
    p.rows = all <= 8 ? 8 : all <= 16 ? 16 : all <= 32 ? 32 : all <= most_mma || dtype == SPECDEC_DTYPE_F32 ? 64 : all <= 128 || !fp4_tc_fits(head_dim, 256, T, n_q_heads / n_kv_heads) ? 128 : 256;
    p.tiles = (all + p.rows - 1) / p.rows;
    p.unit = p.rows >= 128 ? 128 : TA_BLOCK;
    p.min_blocks = 4;
    const long long columns = (long long)n_kv_heads * p.tiles, whole = B * columns, blocks = (max_keys + p.unit - 1) / p.unit;
    p.per_sm = per_sm_of(dtype, head_dim, p.rows);
    const int at_once = TA_SMS * p.per_sm;
    // Whole sequences take their rounds of CTAs times the longest's blocks, stretches an equal share of all blocks and the merge.  (64 x 51 queries over 0 to 256 keys whole 18 us, cut 29;
    // 16 x 51 over 300 to 1000 28 and 38; 32 x 16 over 1000 to 2000 37 and 30.)  Dealt by length, where they are more than CTAs: 64 x 10 over 0 to 512 keys 20 -> 15, 128 x 26 39 -> 32, 128 x 51 33 -> 30.
    p.direct = (whole + at_once - 1) / at_once * blocks <= whole * blocks / at_once + 8 || B > TA_MAX_B;
    if (p.direct && whole > at_once && 2 * columns <= at_once && B <= TA_MAX_B && blocks >= 4) p.direct = 2;
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

template <typename T, int D, int NT, int WM, int WK, int NS, int PER_SM>
cudaError_t run(const Fp4Attn& a, int grid, cudaStream_t st) {
    constexpr int ROWS = 8 * NT * WM, WORDS = ROWS < 64 ? 1 : 32;                      // words of a mask at most (smaller tiles are chosen where one holds the tree)
    auto bytes = [](int words, int B) { return NS * Fp4Stage<D>::BYTES + (ROWS + 1) * words * 4 + B * 16; };
    static_assert(NS * Fp4Stage<D>::BYTES + (ROWS + 1) * WORDS * 4 + TA_MAX_B * 16 + 1024 + 512 <= 233472 / PER_SM, "shared memory of an SM");
    if (const cudaError_t e = op_allow<k_fp4_mma<T, D, NT, WM, WK, NS, PER_SM>>(bytes(WORDS, TA_MAX_B))) return e;
    return op_launch(k_fp4_mma<T, D, NT, WM, WK, NS, PER_SM>, dim3(ta_grid(a, grid, PER_SM * TA_SMS)), 32 * (WM * WK + 1), bytes(a.words, a.direct == 1 ? 0 : a.B), st, 1, a);
}
template <typename T, int NS, int PER_SM>
cudaError_t run_tile(const Fp4Attn& a, int grid, cudaStream_t st) {
    auto bytes = [](int words, int B) { return 4 * TA_BLOCK * 128 + NS * Fp4Stage<64>::BYTES + 65 * words * 4 + B * 16; };
    static_assert(4 * TA_BLOCK * 128 + NS * Fp4Stage<64>::BYTES + 65 * 128 + TA_MAX_B * 16 + 1024 + 512 <= 233472 / PER_SM, "shared memory of an SM");
    if (const cudaError_t e = op_allow<k_fp4_tile<T, NS, PER_SM>>(bytes(32, TA_MAX_B))) return e;
    return op_launch(k_fp4_tile<T, NS, PER_SM>, dim3(ta_grid(a, grid, PER_SM * TA_SMS)), 160, bytes(a.words, a.direct == 1 ? 0 : a.B), st, 1, a);
}
template <typename T>
cudaError_t pick(const Fp4Attn& a, int rows, int grid, cudaStream_t st) {
    if constexpr (sizeof(T) == 4) {
        if (a.dim > 64) return rows == 8 ? run<T, 128, 1, 1, 3, 9, 2>(a, grid, st) : rows == 16 ? run<T, 128, 1, 2, 2, 8, 2>(a, grid, st) : rows == 32 ? run<T, 128, 1, 4, 1, 6, 2>(a, grid, st) : run<T, 128, 1, 8, 1, 8, 1>(a, grid, st);
        return rows == 8 ? run<T, 64, 1, 1, 3, 9, 3>(a, grid, st) : rows == 16 ? run<T, 64, 1, 2, 2, 8, 3>(a, grid, st) : rows == 32 ? run<T, 64, 1, 4, 1, 8, 2>(a, grid, st) : run<T, 64, 2, 4, 1, 8, 2>(a, grid, st);
    } else {
        if (a.dim > 64) return rows == 8 ? run<T, 128, 1, 1, 4, 8, 3>(a, grid, st) : rows == 16 ? run<T, 128, 1, 2, 2, 6, 3>(a, grid, st) : run<T, 128, 1, 4, 1, 6, 3>(a, grid, st);
        return rows == 8 ? run<T, 64, 1, 1, 3, 9, 4>(a, grid, st) : rows == 16 ? run<T, 64, 1, 2, 2, 8, 3>(a, grid, st) : rows == 32 ? run<T, 64, 1, 4, 1, 8, 3>(a, grid, st) : run_tile<T, 5, 3>(a, grid, st);
    }
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
