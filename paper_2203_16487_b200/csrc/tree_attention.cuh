// Attention of drafted trees over the caller's paged cache: what its kernels share (contract: specdec.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "barriers.cuh"
#include "op_error.cuh"
#include "tensor_core.cuh"

namespace sd {

// Rows of one K/V head: query row r = t * group + (head within the group), cut into tiles of a kernel's rows; (K/V head, tile) is a column of work.  The keys of a
// sequence are its length committed tokens and n nodes behind them, in blocks of `unit` keys (64, or 128).
//
// direct: sequences are never cut; CTAs that stay take every gridDim.x-th (sequence, column).  direct = 2 (more items than CTAs): each column's sequences are dealt out by
// falling length, to its CTAs there and back, so that long and short ones meet.
// Otherwise a column's blocks of all sequences form one line, of which each of its `ctas` CTAs takes an equal stretch (TaWork), so that all CTAs run equally long
// whatever the lengths are.  A stretch begins and ends inside sequences: a part that is a whole sequence writes the output, other parts write partial results
// into slots that k_ta_merge joins.  The part of sequence b in the column's CTA c has slot (c + b) * columns + column: along the line either c or b grows.
constexpr int TA_SMS = 148, TA_BLOCK = 64, TA_MAX_B = 128;            // sequences at most where they are cut
constexpr int TA_WIDE_T = 960;                            // nodes at most whose masks fit beside a 256-row tile of 128-wide heads
struct TreeAttn {
    const char* q; char* out; const char* k; const char* v;
    long long q_sb, q_st, q_sh, o_sb, o_st, o_sh, s_page, s_token, s_head;             // bytes
    const int* table; const int* length; const int* seqs; const int* n_nodes; int* status;
    const uint32_t* mask; long long mask_sb;                                           // words
    int n_pages, n_seqs, max_pages, page_shift, max_length;
    int T, words, group, kv_heads, dim, B;
    uint32_t group_mul;                                                                // see ta_node
    int tiles, direct, ctas, unit, min_blocks;                                              // row tiles; CTAs of a column; keys of a block; blocks of a stretch at least
    float scale;                                                                       // times log2(e)
    float* part; float2* part_ml;                                                      // [slot, row of the tile]: output [dim] and (maximum, sum)
    int2* where;                                                                       // [b, column]: first slot, parts
    int q_vec, out_vec;                                                                // whether q / out allow 16-byte accesses
};

// Node of query row gr: gr / group as a product (gr < 2^20, group * gr < 2^32), 0 for a group of one.
__device__ __forceinline__ int ta_node(const TreeAttn& a, int gr) { return a.group_mul ? (int)__umulhi((uint32_t)gr, a.group_mul) : gr; }

struct SeqKeys { int seq, len, nodes, keys; };
__device__ __forceinline__ SeqKeys ta_keys(const TreeAttn& a, int b) {
    SeqKeys s;
    s.seq = a.seqs[b];
    s.nodes = max(0, min(a.n_nodes ? a.n_nodes[b] : a.T, a.T));
    if ((unsigned)s.seq >= (unsigned)a.n_seqs) { s.seq = 0; s.len = 0; s.nodes = 0; }  // no such sequence: nothing to see
    else s.len = max(0, min(a.length[s.seq], a.max_length));
    s.keys = s.nodes ? s.len + s.nodes : 0;
    return s;
}

struct Part { int b, h, tile, k_begin, k_end, blocks, whole; long long slot; SeqKeys s; };     // keys [k_begin, k_end) in `blocks` blocks
struct TaWork {
    // direct: at = number of the next (sequence, column).  Else: the CTA, and what is next on the line: sequence, blocks of it to skip; blocks left, blocks of a stretch
    int column, at, b, skip, left, stretch;
    // For the whole CTA; seqs: B entries (sequence, length, nodes, blocks) of shared memory that stay (not direct).
    __device__ __forceinline__ void begin(const TreeAttn& a, int4* seqs) {
        const int columns = a.kv_heads * a.tiles;
        at = blockIdx.x;
        if (a.direct == 1) return;
        __shared__ int found[4];
        column = blockIdx.x % columns; at = blockIdx.x / columns;
        if (a.direct == 2) {
            __shared__ int length_of[TA_MAX_B];
            SeqKeys s;
            for (int i = threadIdx.x; i < a.B; i += blockDim.x) { s = ta_keys(a, i); length_of[i] = s.keys; }
            __syncthreads();
            for (int i = threadIdx.x; i < a.B; i += blockDim.x) {
                if (a.B > blockDim.x) s = ta_keys(a, i);
                int rank = 0;
                for (int j = 0; j < a.B; ++j) rank += length_of[j] > s.keys || (length_of[j] == s.keys && j < i);
                seqs[rank] = make_int4(s.seq, s.len, s.nodes, i);
            }
            skip = 0;                                     // rounds so far
            __syncthreads();
            return;
        }
        for (int i = threadIdx.x; i < a.B; i += blockDim.x) {
            const SeqKeys s = ta_keys(a, i);
            seqs[i] = make_int4(s.seq, s.len, s.nodes, max(1, (s.keys + a.unit - 1) / a.unit));        // (at least 1: rows that see nothing are written too)
        }
        __syncthreads();
        if (threadIdx.x < 32) {
            const int lane = threadIdx.x;
            unsigned long long total = 0;
            for (int i = lane; i < a.B; i += 32) total += seqs[i].w;
#pragma unroll
            for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
            const unsigned long long per = max(total < 0x40000000ull ? ((uint32_t)total + a.ctas - 1) / (uint32_t)a.ctas : (total + a.ctas - 1) / a.ctas, (unsigned long long)a.min_blocks);
            const unsigned long long start = at * per;
            unsigned long long run = 0;
            int fb = 0, fskip = 0;
            for (int i0 = 0; i0 < a.B; i0 += 32) {        // the sequence in which the stretch begins
                const int n = i0 + lane < a.B ? seqs[i0 + lane].w : 0;
                unsigned long long upto = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const unsigned long long x = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += x; }
                const unsigned m = __ballot_sync(0xffffffffu, run + upto > start);
                if (m) {
                    const int f = __ffs(m) - 1;
                    fb = i0 + f;
                    fskip = (int)(start - (run + __shfl_sync(0xffffffffu, upto - n, f)));
                    break;
                }
                run += __shfl_sync(0xffffffffu, upto, 31);
            }
            if (lane == 0) {
                found[0] = fb; found[1] = fskip;
                found[2] = start < total ? (int)min(per, total - start) : 0;
                found[3] = (int)min(per, 0x3fffffffull);
            }
        }
        __syncthreads();
        b = found[0]; skip = found[1]; left = found[2]; stretch = found[3];
    }
    // The next part.  notes: whether this thread tells the merge where a sequence's parts are.
    __device__ __forceinline__ bool next(const TreeAttn& a, const int4* seqs, Part& p, bool notes = false) {
        const int columns = a.kv_heads * a.tiles;
        if (a.direct == 1) {
            if (at >= a.B * columns) return false;
            p.b = at / columns; column = at - p.b * columns;
            at += gridDim.x;
            p.s = ta_keys(a, p.b);
            p.k_begin = 0; p.k_end = p.s.keys; p.whole = 1; p.slot = 0;
            p.blocks = (p.s.keys + a.unit - 1) / a.unit;
        } else if (a.direct == 2) {
            const int ctas = gridDim.x / columns, i = skip * ctas + (skip & 1 ? ctas - 1 - at : at);
            ++skip;
            if (i >= a.B) return false;                   // (a later round lies behind as well)
            const int4 q = seqs[i];
            p.b = q.w;
            p.s.seq = q.x; p.s.len = q.y; p.s.nodes = q.z; p.s.keys = q.z ? q.y + q.z : 0;
            p.k_begin = 0; p.k_end = p.s.keys; p.whole = 1; p.slot = 0;
            p.blocks = (p.s.keys + a.unit - 1) / a.unit;
        } else {
            if (left <= 0) return false;
            const int4 q = seqs[b];
            const int n = q.w, take = min(n - skip, left);
            p.b = b;
            p.s.seq = q.x; p.s.len = q.y; p.s.nodes = q.z; p.s.keys = q.z ? q.y + q.z : 0;
            p.k_begin = skip * a.unit; p.k_end = min(p.s.keys, (skip + take) * a.unit);
            p.blocks = max(0, (p.k_end - p.k_begin + a.unit - 1) / a.unit);
            p.whole = take == n;
            p.slot = (long long)(at + b) * columns + column;
            if (notes && skip == 0) {                     // the rest, if any, lies in the CTAs that follow
                const int rest = n - take, parts = 1 + (rest + stretch - 1) / stretch;
                a.where[b * columns + column] = make_int2((int)p.slot, parts);
            }
            left -= take;
            ++b; skip = 0;
        }
        p.h = column / a.tiles; p.tile = column - p.h * a.tiles;
        return true;
    }
};

// What a query sees of 32 keys from key k0 on, as bits: committed ones all, nodes by its row of words; base = k0 - length.
__device__ __forceinline__ uint32_t ta_window(const uint32_t* row, int words, int base) {
    if (base <= -32) return 0xffffffffu;
    if (base < 0) return ((1u << -base) - 1u) | (words ? row[0] << -base : 0u);
    const int w = base >> 5, s = base & 31;
    const uint32_t a = w < words ? row[w] : 0u, b = w + 1 < words ? row[w + 1] : 0u;
    return __funnelshift_r(a, b, s);
}
// The same from one or two words.
__device__ __forceinline__ uint32_t ta_window2(uint32_t m0, uint32_t m1, int base) {
    if (base <= -32) return 0xffffffffu;
    if (base < 0) return ((1u << -base) - 1u) | m0 << -base;
    return base < 32 ? __funnelshift_r(m0, m1, base) : base < 64 ? m1 >> (base - 32) : 0u;
}
// The mask rows of a tile's queries (cut at the nodes), and any[w]: the nodes that one of them sees.  Query rows r0 .. r0 + rows - 1.
// By the first NT threads of the CTA, which meet at barrier BAR.
template <int NT, int BAR>
__device__ __forceinline__ void ta_load_masks(const TreeAttn& a, int b, int r0, int rows, int nodes, uint32_t* mask, uint32_t* any) {
    auto sync = [] { asm volatile("bar.sync %0, %1;" ::"n"(BAR), "n"(NT) : "memory"); };
    for (int w = threadIdx.x; w < a.words; w += NT) any[w] = 0;
    sync();
    const int t0 = ta_node(a, r0), t1 = min(ta_node(a, r0 + rows - 1), a.T - 1);
    for (int i = threadIdx.x; i < (t1 - t0 + 1) * a.words; i += NT) {
        const int t = t0 + i / a.words, w = i % a.words;
        uint32_t m = t < nodes ? a.mask[b * a.mask_sb + (long long)t * a.words + w] : 0u;
        const int left = nodes - w * 32;
        if (left < 32) m &= left <= 0 ? 0u : (1u << left) - 1u;
        mask[i] = m;
        if (m) atomicOr(any + w, m);
    }
    sync();
}
// Whether one of the tile's queries may see key `key` < keys.
__device__ __forceinline__ bool ta_seen(const uint32_t* any, const SeqKeys& s, int key) {
    return key < s.len || (key < s.keys && (any[(key - s.len) >> 5] >> ((key - s.len) & 31) & 1));
}

// Zeros for the values, in a block of 64 rows of HALVES x 128 bytes, that none of the tile's queries sees: whatever is in them is multiplied by 0.  Rows
// [row0, row0 + ROWS) by one warp; seen(row): 32 rows from there on as bits.
template <int ROWS, int HALVES, typename F>
__device__ __forceinline__ void ta_zero_unseen(char* values, int row0, F seen_from) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r0 = 0; r0 < ROWS; r0 += 32) {
        constexpr int N = ROWS < 32 ? ROWS : 32;
        const uint32_t seen = seen_from(row0 + r0);
#pragma unroll
        for (int r = 0; r < N; r += 4) {
            const int mine = r + (lane >> 3);
            if (!(seen >> mine & 1))
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
                    *reinterpret_cast<uint4*>(values + hf * TA_BLOCK * 128 + (row0 + r0 + mine) * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
        }
    }
}

// 16-byte pieces of shared memory from global memory, or zeros.
__device__ __forceinline__ void ta_copy16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ float ta_exp2(float x) {       // results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void ta_ldsm4(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ta_ldsm4_t(uint32_t addr, uint32_t* r) {
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
    static __device__ __forceinline__ float add(float s, uint32_t x) {          // s + both of x
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tadd.f32.bf16 %0, l, %0;\n\tadd.f32.bf16 %0, h, %0;\n\t}" : "+f"(s) : "r"(x));
        return s;
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
    static __device__ __forceinline__ float add(float s, uint32_t x) {
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tadd.f32.f16 %0, l, %0;\n\tadd.f32.f16 %0, h, %0;\n\t}" : "+f"(s) : "r"(x));
        return s;
    }
};


// Sixteen query rows of a warp over blocks of 64 keys: lane l holds rows l / 4 and l / 4 + 8.  Running maximum m and sum l of 2^(s - m), output o; scores
// in units of log2.  The second product takes the probabilities as 16-bit numbers, and the sum adds up those: the weights add up to 1, so that their rounding moves
// the output by its share of the values' spread, not of their size, and a dominating key's cancels (sums of the unrounded ones take as long, within 1 %).  kf(row, piece) / vf(row, piece): shared-memory address of 16-byte piece `piece` of a key's row.
template <typename T, int DP>
struct TaRows {
    static constexpr int NK = TA_BLOCK / 8, ND = DP / 8;
    float o[ND][4], ma, mb, la, lb;
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        ma = mb = -INFINITY; la = lb = 0.f;
    }
    // window_a, window_b(base): what the rows see of 32 keys, asked where the block holds nodes or ends behind the last key
    template <typename WA, typename WB, typename KF, typename VF>
    __device__ __forceinline__ void block(const uint32_t (*qf)[4], int k0, int len, float scale, WA window_a, WB window_b, KF kf, VF vf) {
        const int lane = threadIdx.x & 31;
        float sc[NK][4];
#pragma unroll
        for (int i = 0; i < NK; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
#pragma unroll
            for (int n = 0; n < TA_BLOCK / 16; ++n) {
                uint32_t x[4];
                ta_ldsm4(kf(n * 16 + (lane & 7) + ((lane >> 4) << 3), kk * 2 + ((lane >> 3) & 1)), x);
                Half<T>::mma(sc[2 * n], qf[kk], x[0], x[1]);
                Half<T>::mma(sc[2 * n + 1], qf[kk], x[2], x[3]);
            }
        if (k0 + TA_BLOCK > len) {
#pragma unroll
            for (int n = 0; n < TA_BLOCK / 32; ++n) {
                const int base = k0 + n * 32 - len;
                const uint32_t wa = window_a(base), wb = window_b(base);
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
        na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 1)); na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, 2));
        nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 1)); nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, 2));
        na = fmaxf(ma, na * scale); nb = fmaxf(mb, nb * scale);
        const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
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
                c[0] = ta_exp2(fmaf(c[0], scale, -za)); c[1] = ta_exp2(fmaf(c[1], scale, -za));
                c[2] = ta_exp2(fmaf(c[2], scale, -zb)); c[3] = ta_exp2(fmaf(c[3], scale, -zb));
                pf[2 * e] = Half<T>::pack(c[0], c[1]);
                pf[2 * e + 1] = Half<T>::pack(c[2], c[3]);
                la = Half<T>::add(la, pf[2 * e]); lb = Half<T>::add(lb, pf[2 * e + 1]);
            }
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                uint32_t x[4];
                ta_ldsm4_t(vf(n * 16 + (lane & 15), d * 2 + (lane >> 4)), x);
                Half<T>::mma(o[2 * d], pf, x[0], x[1]);
                Half<T>::mma(o[2 * d + 1], pf, x[2], x[3]);
            }
        }
    }
    // The lanes' sums together.  A query behind the nodes has taken the committed keys of blocks without a mask; one that sees nothing has multiplied values by 0.
    __device__ __forceinline__ void finish(bool live_a, bool live_b) {
        la += __shfl_xor_sync(0xffffffffu, la, 1); la += __shfl_xor_sync(0xffffffffu, la, 2);
        lb += __shfl_xor_sync(0xffffffffu, lb, 1); lb += __shfl_xor_sync(0xffffffffu, lb, 2);
        if (!live_a || la == 0.f) {
            ma = -INFINITY; la = 0.f;
#pragma unroll
            for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = 0.f;
        }
        if (!live_b || lb == 0.f) {
            mb = -INFINITY; lb = 0.f;
#pragma unroll
            for (int i = 0; i < ND; ++i) o[i][2] = o[i][3] = 0.f;
        }
    }
    // Partial results in shared memory: rows of RP floats, and (maximum, sum) of each.
    static constexpr int RP = DP + 8;
    __device__ __forceinline__ void leave(float* red, float2* red_ml, int ra) const {
        const int lane = threadIdx.x & 31;
        float* pa = red + ra * RP + (lane & 3) * 2;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            *reinterpret_cast<float2*>(pa + i * 8) = make_float2(o[i][0], o[i][1]);
            *reinterpret_cast<float2*>(pa + 8 * RP + i * 8) = make_float2(o[i][2], o[i][3]);
        }
        if ((lane & 3) == 0) { red_ml[ra] = make_float2(ma, la); red_ml[ra + 8] = make_float2(mb, lb); }
    }
    __device__ __forceinline__ void join(const float* red, const float2* red_ml, int ra) {
        const float2 xa = red_ml[ra], xb = red_ml[ra + 8];
        const float na = fmaxf(ma, xa.x), nb = fmaxf(mb, xb.x);
        const float za = na == -INFINITY ? 0.f : na, zb = nb == -INFINITY ? 0.f : nb;
        const float fa = ta_exp2(ma - za), fb = ta_exp2(mb - zb), ea = ta_exp2(xa.x - za), eb = ta_exp2(xb.x - zb);
        ma = na; mb = nb;
        la = la * fa + xa.y * ea; lb = lb * fb + xb.y * eb;
        const float* pa = red + ra * RP + (threadIdx.x & 3) * 2;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const float2 u = *reinterpret_cast<const float2*>(pa + i * 8), w = *reinterpret_cast<const float2*>(pa + 8 * RP + i * 8);
            o[i][0] = o[i][0] * fa + u.x * ea; o[i][1] = o[i][1] * fa + u.y * ea;
            o[i][2] = o[i][2] * fb + w.x * eb; o[i][3] = o[i][3] * fb + w.y * eb;
        }
    }
    // Rows ra and ra + 8 of a tile of `rows` that begins at query row r0: the output, or the part's partial results.
    __device__ __forceinline__ void store(const TreeAttn& a, const Part& it, int r0, int ra, int rows) const {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = ra + 8 * e, gr = r0 + r;
            const float l = e ? lb : la, inv = l > 0.f || l != l ? 1.f / l : 0.f;
            if (gr >= a.T * a.group) continue;
            if (it.whole) {
                const int t = ta_node(a, gr);
                char* p = a.out + it.b * a.o_sb + t * a.o_st + (it.h * a.group + gr - t * a.group) * a.o_sh + (lane & 3) * 4;
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    if (i * 8 >= a.dim) break;
                    const uint32_t x = Half<T>::pack(o[i][2 * e] * inv, o[i][2 * e + 1] * inv);
                    if (a.out_vec) *reinterpret_cast<uint32_t*>(p + i * 16) = x;
                    else { reinterpret_cast<unsigned short*>(p + i * 16)[0] = (unsigned short)x; reinterpret_cast<unsigned short*>(p + i * 16)[1] = (unsigned short)(x >> 16); }
                }
            } else {
                const long long slot = it.slot * rows + r;
                float* p = a.part + slot * a.dim + (lane & 3) * 2;
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    if (i * 8 >= a.dim) break;
                    *reinterpret_cast<float2*>(p + i * 8) = make_float2(o[i][2 * e], o[i][2 * e + 1]);
                }
                if ((lane & 3) == 0) a.part_ml[slot] = make_float2(e ? mb : ma, l);
            }
        }
    }
};

// CTAs of a launch of `grid` items or stretches, where `most` run at once.
inline int ta_grid(const TreeAttn& a, int grid, int most) {
    if (!a.direct || grid <= most) return grid;
    const int columns = a.kv_heads * a.tiles;
    return a.direct == 2 ? most / columns * columns : most;
}

// A tensor map of one layer's keys and values: {head_dim, heads, tokens of a page, pages, 2 sides}; a box is 64 elements (128 bytes, swizzled) of min(page, TA_BLOCK)
// tokens of one head.  What lies beyond head_dim or the pages arrives as zeros.
__device__ __forceinline__ void ta_box(uint32_t dst, const CUtensorMap* tm, int d, int head, int token, int page, int side, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(dst), "l"(tm), "r"(bar), "r"(d), "r"(head), "r"(token), "r"(page), "r"(side) : "memory");
}
constexpr int TA_MIN_PAGE = 8;                            // tokens: a box fills whole swizzle groups of 8 rows

cudaError_t ta_tma_mma(const CUtensorMap& tm, const TreeAttn& a, int dtype, int rows, int grid, cudaStream_t st);         // tiles of 16, 32, 64 rows
cudaError_t ta_tc(const CUtensorMap& tm, const TreeAttn& a, int dtype, int rows, int grid, cudaStream_t st);              // of 128, 256

}  // namespace sd
