// Attention of drafted trees over the caller's paged cache (contract: specdec.h): entry point, warp-level kernels, merge of split keys.
//
// out = sum_j p_j v_j over the keys a query sees, p = softmax(scale q . k).  One pass over the keys with the running maximum m and sum l of
// 2^(s - m): s in units of log2, sums and outputs in fp32, rescaled where m grows.  All query heads of a K/V head share its keys, so a row tile
// mixes nodes and heads; few rows: the keys of a sequence are split over CTAs, whose partial outputs k_ta_merge joins.
#include "tree_attention.cuh"

namespace sd {
namespace {

// ------------------------------------------------------------------ 16-bit types, pages of fewer than TA_MIN_PAGE tokens
// Such pages are no TMA boxes: every thread fetches 16-byte pieces (cp.async).  4 warps of 16 rows, a ring of NS blocks of 64 keys, rows of
// DP elements whose 16-byte pieces are XORed with the row's low three bits.  Every piece is an instruction, a wait and an address of its own, which is what bounds it:
// 128 x 51 queries over 51 to 307 keys in pages of 4 tokens 42 us (by boxes, pages of 16: 28), 8 x 1 query over 8000 keys 63 (34; a tile is 64 rows here however few are real).
template <typename T, int DP, int NS>
__global__ void __launch_bounds__(128) k_ta_small_pages(TreeAttn a) {
    constexpr int ROWS = 64, KT = TA_BLOCK, PITCH = DP * 2, PIECES = DP / 8, STAGE = 2 * KT * PITCH;
    extern __shared__ __align__(128) char sm[];
    char* ring = sm;                                      // [NS][K, V][KT][PITCH]; at first the queries
    int4* seqs = (int4*)(sm + NS * STAGE);
    uint32_t* any = (uint32_t*)(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, wm = tid >> 5;
    op_begin();
    TaWork work;
    work.begin(a, seqs);
    Part it;
    while (work.next(a, seqs, it, tid == 0)) {
    __syncthreads();
    const int h = it.h, r0 = it.tile * ROWS, all_rows = a.T * a.group, t0 = r0 / a.group;
    const SeqKeys& s = it.s;
    ta_load_masks<128, 0>(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
    for (int i = tid; i < ROWS * PIECES; i += 128) {      // queries: rows through shared memory into fragments
        const int r = i / PIECES, c = i % PIECES, gr = r0 + r;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (gr < all_rows && c * 8 < a.dim) {
            const char* p = a.q + it.b * a.q_sb + (gr / a.group) * a.q_st + (h * a.group + gr % a.group) * a.q_sh + c * 16;
            if (a.q_vec) x = *reinterpret_cast<const uint4*>(p);
            else {
                const unsigned short* e = reinterpret_cast<const unsigned short*>(p);
                x = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
            }
        }
        *reinterpret_cast<uint4*>(ring + r * PITCH + ((c ^ (r & 7)) << 4)) = x;
    }
    __syncthreads();
    uint32_t qf[DP / 16][4];
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) {
        const int r = wm * 16 + (lane & 15), c = kk * 2 + (lane >> 4);
        ta_ldsm4(smem_u32(ring + r * PITCH + ((c ^ (r & 7)) << 4)), qf[kk]);
    }
    __syncthreads();

    const char* kbase = a.k + h * a.s_head;
    const char* vbase = a.v + h * a.s_head;
    if (a.dim < DP)                                       // pieces beyond the head: zero once, never written again
        for (int i = tid; i < NS * 2 * KT * PIECES; i += 128) {
            const int r = (i / PIECES) % KT, c = i % PIECES;
            if (c * 8 >= a.dim) *reinterpret_cast<uint4*>(ring + (i / PIECES) * PITCH + ((c ^ (r & 7)) << 4)) = make_uint4(0, 0, 0, 0);
        }
    const int k_begin = it.k_begin, k_end = it.k_end, blocks = it.blocks, real_pieces = a.dim / 8;
    auto load = [&](int j) {
        if (j < blocks) {
            char* st = ring + (j % NS) * STAGE;
            for (int i = tid; i < KT * PIECES; i += 128) {
                const int r = i / PIECES, c = i % PIECES, key = k_begin + j * KT + r, pi = key >> a.page_shift;
                if (c >= real_pieces) continue;
                int page = -1;
                if (key < k_end && ta_seen(any, s, key) && pi < a.max_pages) page = a.table[(long long)s.seq * a.max_pages + pi];
                const bool real = (unsigned)page < (unsigned)a.n_pages;
                const long long off = real ? page * a.s_page + (key & ((1 << a.page_shift) - 1)) * a.s_token + c * 16 : 0;
                const uint32_t d = smem_u32(st + r * PITCH + ((c ^ (r & 7)) << 4));
                ta_copy16(d, kbase + off, real);
                ta_copy16(d + KT * PITCH, vbase + off, real);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const int ra = wm * 16 + (lane >> 2), rb = ra + 8;
    const int ta = (r0 + ra) / a.group, tb = (r0 + rb) / a.group;
    const bool live_a = r0 + ra < all_rows && ta < s.nodes, live_b = r0 + rb < all_rows && tb < s.nodes;
    const uint32_t* mask_a = mask + (live_a ? ta - t0 : 0) * a.words;
    const uint32_t* mask_b = mask + (live_b ? tb - t0 : 0) * a.words;
    TaRows<T, DP> rows;
    rows.clear();
    __syncthreads();
    for (int j = 0; j < NS - 1; ++j) load(j);
    for (int j = 0; j < blocks; ++j) {
        asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
        __syncthreads();
        load(j + NS - 1);
        const uint32_t ks = smem_u32(ring + (j % NS) * STAGE), vs = ks + KT * PITCH;
        rows.block(qf, k_begin + j * KT, s.len, a.scale, [&](int base) { return live_a ? ta_window(mask_a, a.words, base) : 0u; }, [&](int base) { return live_b ? ta_window(mask_b, a.words, base) : 0u; },
                   [&](int r, int c) { return ks + r * PITCH + ((c ^ (r & 7)) << 4); }, [&](int r, int c) { return vs + r * PITCH + ((c ^ (r & 7)) << 4); });
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    rows.finish(live_a, live_b);
    rows.store(a, it, r0, ra, ROWS);
    }
}

// ------------------------------------------------------------------ fp32: FFMA
// CTA = WK warps over the same 4 RI rows, each with every WK-th block of 16 keys to itself (rings, scores and running sums are a warp's own, so nothing waits for
// another warp until the results meet).  Lane (rg, x): RI rows, for the scores the keys x and x + 8, for the output the columns 4 x + 32 c.  The next block's keys are
// fetched under this block's second product, its values under the next scores.  One row is bounded by HBM (2 x 1 query, 32/8 heads of 128, over 30000 keys 5.3 TB/s), a call of
// few CTAs by the chain of one warp, one of many rows by the shared memory's reads, 24 wavefronts for 32 fused multiply-adds (8 x 26 queries over 2000 keys 49 us, 16.7 TFLOP/s;
// two columns an instruction, with every probability twice in shared memory, 46.5, but 2 to 5 % slower where there are fewer rows).  (8 warps with blocks of 32 keys, two to a
// scheduler: no faster for 8 x 9 queries over 300 to 512 keys.)
constexpr int TF_KT = 16;
template <int DP, int RI, int PER_SM> struct TfCfg {
    static constexpr int ROWS = 4 * RI;
    static constexpr int WK = (DP > 64 ? 8 : 16) / PER_SM, KP = DP + 4, PP = TF_KT + 4;            // pitches in floats
    static constexpr int WARP = 2 * TF_KT * KP + ROWS * PP;                         // a warp's keys, values and probabilities
    static constexpr int FLOATS = ROWS * KP + WK * WARP;
};
template <int DP, int RI, int PER_SM>
__global__ void __launch_bounds__(32 * TfCfg<DP, RI, PER_SM>::WK, PER_SM) k_ta_f32(TreeAttn a) {
    using Cfg = TfCfg<DP, RI, PER_SM>;
    constexpr int ROWS = Cfg::ROWS, WK = Cfg::WK, KP = Cfg::KP, PP = Cfg::PP, NT = 32 * WK, DC = DP / 32, KE = TF_KT / 8;
    extern __shared__ __align__(128) char sm[];
    float* q = reinterpret_cast<float*>(sm);              // [ROWS][KP]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rg = lane >> 3, x = lane & 7;
    float* kt = q + ROWS * KP + warp * Cfg::WARP;      // [16][KP]
    float* vt = kt + TF_KT * KP;
    float* pt = vt + TF_KT * KP;                          // [ROWS][PP]
    int4* seqs = reinterpret_cast<int4*>(q + Cfg::FLOATS);
    uint32_t* any = reinterpret_cast<uint32_t*>(seqs + (a.direct == 1 ? 0 : a.B));
    uint32_t* mask = any + a.words;
    op_begin();
    TaWork work;
    work.begin(a, seqs);
    const int chunks = a.dim / 4;
    Part it;
    while (work.next(a, seqs, it, tid == 0)) {
        __syncthreads();
        const int r0 = it.tile * ROWS, all_rows = a.T * a.group, t0 = ta_node(a, r0);
        const SeqKeys& s = it.s;
        const int blocks = (it.k_end - it.k_begin + TF_KT - 1) / TF_KT;
        auto page_of = [&](int j) -> int {                // of this lane's key in block j
            const int key = it.k_begin + j * TF_KT + lane % TF_KT, pi = key >> a.page_shift;
            return j < blocks && key < it.k_end && pi < a.max_pages ? a.table[(long long)s.seq * a.max_pages + pi] : -1;
        };
        auto offset = [&](int j, int page) -> long long { // of the key itself; -1: zeros instead
            const int key = it.k_begin + j * TF_KT + lane % TF_KT;
            return (unsigned)page < (unsigned)a.n_pages && ta_seen(any, s, key) ? page * a.s_page + (key & ((1 << a.page_shift) - 1)) * a.s_token + it.h * a.s_head : -1;
        };
        int page = page_of(warp);
#pragma unroll
        for (int i0 = 0; i0 < ROWS * (DP / 4); i0 += NT) {
            if (ROWS * (DP / 4) % NT && i0 + tid >= ROWS * (DP / 4)) break;
            const int i = i0 + tid, r = i / (DP / 4), d = i % (DP / 4) * 4, gr = r0 + r, node = ta_node(a, gr);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (gr < all_rows && node < s.nodes && d < a.dim) {
                const float* p = reinterpret_cast<const float*>(a.q + it.b * a.q_sb + node * a.q_st + (it.h * a.group + gr - node * a.group) * a.q_sh) + d;
                v = a.q_vec ? *reinterpret_cast<const float4*>(p) : make_float4(p[0], p[1], p[2], p[3]);
            }
            *reinterpret_cast<float4*>(q + r * KP + d) = v;
        }
        if (a.dim < DP)                                   // columns beyond the head
            for (int i = lane; i < 2 * TF_KT * (DP - a.dim); i += 32) kt[i / (DP - a.dim) * KP + a.dim + i % (DP - a.dim)] = 0.f;
        ta_load_masks<NT, 0>(a, it.b, r0, min(ROWS, all_rows - r0), s.nodes, mask, any);
        auto fetch = [&](float* to, const char* base, long long off) {
#pragma unroll
            for (int r0 = 0; r0 < TF_KT; r0 += 4) {       // four keys at a time, eight lanes each
                const int r = r0 + rg;
                const long long o = __shfl_sync(0xffffffffu, off, r);
#pragma unroll
                for (int c = x; c < DP / 4; c += 8)
                    if (c < chunks) ta_copy16(smem_u32(to + r * KP + c * 4), base + (o < 0 ? 0 : o + c * 16), o >= 0);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        bool live[RI];
        const uint32_t* row[RI];
        float m[RI], l[RI];
        float4 o[RI][DC];
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            const int gr = r0 + rg * RI + i, node = ta_node(a, gr);
            live[i] = gr < all_rows && node < s.nodes;
            row[i] = mask + (live[i] ? (node - t0) * a.words : 0);
            m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
            for (int c = 0; c < DC; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        long long off = offset(warp, page);
        fetch(kt, a.k, off);
        for (int j = warp; j < blocks; j += WK) {
            fetch(vt, a.v, off);
            page = page_of(j + WK);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
            float sc[RI][KE];                              // [row][key x + 8 e]
#pragma unroll
            for (int i = 0; i < RI; ++i)
#pragma unroll
                for (int e = 0; e < KE; ++e) sc[i][e] = 0.f;
#pragma unroll 4
            for (int d = 0; d < DP; d += 4) {
                float4 qv[RI], kv[KE];
#pragma unroll
                for (int i = 0; i < RI; ++i) qv[i] = *reinterpret_cast<const float4*>(q + (rg * RI + i) * KP + d);
#pragma unroll
                for (int e = 0; e < KE; ++e) kv[e] = *reinterpret_cast<const float4*>(kt + (x + 8 * e) * KP + d);
#pragma unroll
                for (int i = 0; i < RI; ++i)
#pragma unroll
                    for (int e = 0; e < KE; ++e)
                        sc[i][e] = fmaf(qv[i].x, kv[e].x, fmaf(qv[i].y, kv[e].y, fmaf(qv[i].z, kv[e].z, fmaf(qv[i].w, kv[e].w, sc[i][e]))));
            }
            __syncwarp();
            off = offset(j + WK, page);
            fetch(kt, a.k, off);
            const int base = it.k_begin + j * TF_KT - s.len;
#pragma unroll
            for (int i = 0; i < RI; ++i) {
                const uint32_t w = live[i] ? ta_window(row[i], a.words, base) : 0u;
                float top = -INFINITY;
#pragma unroll
                for (int e = 0; e < KE; ++e) {
                    sc[i][e] = w >> (x + 8 * e) & 1 ? sc[i][e] * a.scale : -INFINITY;
                    top = fmaxf(top, sc[i][e]);
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1)); top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)); top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                top = fmaxf(top, m[i]);
                const float z = top == -INFINITY ? 0.f : top, f = ta_exp2(m[i] - z);
                m[i] = top;
                l[i] *= f;
#pragma unroll
                for (int e = 0; e < KE; ++e) {
                    const float p = ta_exp2(sc[i][e] - z);
                    l[i] += p;
                    pt[(rg * RI + i) * PP + x + 8 * e] = p;
                }
#pragma unroll
                for (int c = 0; c < DC; ++c) { o[i][c].x *= f; o[i][c].y *= f; o[i][c].z *= f; o[i][c].w *= f; }
            }
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
#pragma unroll 2
            for (int key = 0; key < TF_KT; key += 4) {
                float4 p[RI];
#pragma unroll
                for (int i = 0; i < RI; ++i) p[i] = *reinterpret_cast<const float4*>(pt + (rg * RI + i) * PP + key);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < DC; ++c) {
                        const float4 v = *reinterpret_cast<const float4*>(vt + (key + e) * KP + x * 4 + 32 * c);
#pragma unroll
                        for (int i = 0; i < RI; ++i) {
                            const float w = e == 0 ? p[i].x : e == 1 ? p[i].y : e == 2 ? p[i].z : p[i].w;
                            o[i][c].x = fmaf(w, v.x, o[i][c].x); o[i][c].y = fmaf(w, v.y, o[i][c].y); o[i][c].z = fmaf(w, v.z, o[i][c].z); o[i][c].w = fmaf(w, v.w, o[i][c].w);
                        }
                    }
            }
            __syncwarp();
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        // the warps' results meet: output in the keys' place, (maximum, sum) in the probabilities'
        __syncwarp();
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1); l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2); l[i] += __shfl_xor_sync(0xffffffffu, l[i], 4);
            const bool none = l[i] == 0.f;                // sees nothing here: values times 0
#pragma unroll
            for (int c = 0; c < DC; ++c) *reinterpret_cast<float4*>(kt + (rg * RI + i) * KP + x * 4 + 32 * c) = none ? make_float4(0.f, 0.f, 0.f, 0.f) : o[i][c];
            if (x == 0) { pt[rg * RI + i] = none ? -INFINITY : m[i]; pt[ROWS + rg * RI + i] = l[i]; }
        }
        __syncthreads();
        const float* w0 = q + ROWS * KP;               // warp w's keys: + w * WARP; its probabilities: + 2 * TF_KT * KP
        for (int i = tid; i < ROWS * (DP / 4); i += NT) {
            const int r = i / (DP / 4), c = i % (DP / 4), gr = r0 + r;
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) top = fmaxf(top, w0[w * Cfg::WARP + 2 * TF_KT * KP + r]);
            const float z = top == -INFINITY ? 0.f : top;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float* p = w0 + w * Cfg::WARP;
                const float f = exp2f(p[2 * TF_KT * KP + r] - z);
                const float4 v = *reinterpret_cast<const float4*>(p + r * KP + c * 4);
                sum += p[2 * TF_KT * KP + ROWS + r] * f;
                y.x = fmaf(v.x, f, y.x); y.y = fmaf(v.y, f, y.y); y.z = fmaf(v.z, f, y.z); y.w = fmaf(v.w, f, y.w);
            }
            if (gr >= all_rows || c * 4 >= a.dim) continue;
            if (it.whole) {
                const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                const int node = ta_node(a, gr);
                float* p = reinterpret_cast<float*>(a.out + it.b * a.o_sb + node * a.o_st + (it.h * a.group + gr - node * a.group) * a.o_sh) + c * 4;
                if (a.out_vec) *reinterpret_cast<float4*>(p) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
                else { p[0] = y.x * inv; p[1] = y.y * inv; p[2] = y.z * inv; p[3] = y.w * inv; }
            } else {
                const long long slot = it.slot * ROWS + r;
                *reinterpret_cast<float4*>(a.part + slot * a.dim + c * 4) = y;
                if (c == 0) a.part_ml[slot] = make_float2(top, sum);
            }
        }
    }
}

// ------------------------------------------------------------------ merge
// Four columns; `whole`: as one store.
template <typename T> __device__ __forceinline__ void put4(char* p, float4 x, int whole) {
    if constexpr (sizeof(T) == 4) {
        if (whole) { *reinterpret_cast<float4*>(p) = x; return; }
        float* f = reinterpret_cast<float*>(p);
        f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
    } else {
        const uint32_t u = Half<T>::pack(x.x, x.y), v = Half<T>::pack(x.z, x.w);
        if (whole) { *reinterpret_cast<uint2*>(p) = make_uint2(u, v); return; }
        unsigned short* f = reinterpret_cast<unsigned short*>(p);
        f[0] = (unsigned short)u; f[1] = (unsigned short)(u >> 16); f[2] = (unsigned short)v; f[3] = (unsigned short)(v >> 16);
    }
}

// The parts' outputs, each rescaled to the largest maximum: one warp R query rows of a tile, CTAs that stay.  Three reads that wait for one another: a tile's
// parts; their maxima and sums (32 / R lanes a row, one a part); their outputs (lane: four columns), U parts on their way at a time.  R = 4 where there are rows enough for
// all warps of the GPU that way (16384 rows of 2 or 3 parts: 16.5 us with R = 1), else 1.  Those 16384 rows of 128: 27 MB from L2 and memory, 11 us cold; two rows of 50
// parts, 9 us, the three reads' latency.
template <typename T, int R, int U>
__global__ void __launch_bounds__(128, 8) k_ta_merge(TreeAttn a, int rows) {
    constexpr int L = 32 / R;
    const int lane = threadIdx.x & 31, columns = a.kv_heads * a.tiles, all = a.T * a.group, sets = (all + R - 1) / R, x = lane / L, e = lane % L;
    op_begin();
    for (int w = blockIdx.x * 4 + (threadIdx.x >> 5); w < a.B * a.kv_heads * sets; w += gridDim.x * 4) {
        const int bh = w / sets, gr0 = (w - bh * sets) * R, b = bh / a.kv_heads, h = bh - b * a.kv_heads, tile = gr0 / rows, r0 = gr0 - tile * rows;
        const int2 at = a.where[bh * a.tiles + tile];     // first slot, parts
        if (at.y <= 1) continue;
        const long long slot0 = (long long)at.x * rows + r0, step = (long long)columns * rows;
        float m = -INFINITY;                              // of row x
        for (int s = e; s < at.y; s += L) m = fmaxf(m, a.part_ml[slot0 + x + s * step].x);
#pragma unroll
        for (int of = L / 2; of; of >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, of));
        const float z = m == -INFINITY ? 0.f : m;
        float4 o[R];
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < at.y; s0 += L) {
            float f = 0.f;                                // of row x, part s0 + e
            if (s0 + e < at.y) {
                const float2 ml = a.part_ml[slot0 + x + (s0 + e) * step];
                f = exp2f(ml.x - z);
                l += ml.y * f;
            }
            for (int s = s0; s < min(s0 + L, at.y); s += U) {
                float4 v[U][R];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        v[u][i] = lane * 4 < a.dim && s + u < at.y ? *reinterpret_cast<const float4*>(a.part + (slot0 + (s + u) * step + i) * a.dim + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < R; ++i) {
                        const float g = __shfl_sync(0xffffffffu, f, i * L + (s + u - s0) % L);
                        o[i].x = fmaf(v[u][i].x, g, o[i].x); o[i].y = fmaf(v[u][i].y, g, o[i].y); o[i].z = fmaf(v[u][i].z, g, o[i].z); o[i].w = fmaf(v[u][i].w, g, o[i].w);
                    }
            }
        }
#pragma unroll
        for (int of = L / 2; of; of >>= 1) l += __shfl_xor_sync(0xffffffffu, l, of);
        const float inv_x = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float inv = __shfl_sync(0xffffffffu, inv_x, i * L);
            const int gr = gr0 + i;
            if (gr >= all || lane * 4 >= a.dim) continue;
            const int t = ta_node(a, gr);
            put4<T>(a.out + b * a.o_sb + t * a.o_st + (h * a.group + gr - t * a.group) * a.o_sh + lane * 4 * sizeof(T), make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), a.out_vec);
        }
    }
}

// ------------------------------------------------------------------ host
struct Plan { int rows, tiles, per_sm, direct, ctas, unit, min_blocks; long long grid, slots; };       // see TreeAttn; slots of partial results
// Rows of a tile.  16-bit types: 16, 32 or 64 with mma.sync by the rows there are (64 share a block's keys among four warps; fewer rows give the warps keys of their own
// instead), 128 or 256 with tcgen05 beyond 64 rows, of heads wider than 64 beyond 32.  (64 rows, 2 x 8 heads of 128 over 8000 keys: 31 us with tcgen05, 33 without; over 2000 keys of 64
// sequences 43 and 48; heads of 64: 24.5 and 23, 32 and 27.  128 rows: 69 and 120, 136 and 243; heads of 64 50 and 67, 93 and 138.)
// fp32: as few tiles of up to 16 as there must be, of equal size in fours (8 x 1 query over 8000 keys: 57 us with 4 rows, 90 with 16; 8 x 9 over 300 to 512: 15.9 with 12, 18.3).
// CTAs that an SM holds (at least): of fp32 the more, each of fewer warps, the more work there is that they take in turn: 4 or 2 of 4 rows (64 x 1 over 0 to 512 keys 22 and 25 us, 8 x
// 1 over 8000 52 and 54, 1 x 1 over 64 5.0 and 4.4), 2 or 1 of 12 and 16 (32 x 17 over 0 to 512 keys 40 and 49; 8 x 9 over 300 to 512 16.8 and 15.9).
Plan plan(int B, int T, int n_q_heads, int n_kv_heads, int dtype, int head_dim, int page_tokens, long long max_keys) {
    const int all = T * (n_q_heads / n_kv_heads);
    Plan p;
    const int most_mma = head_dim > 64 ? 32 : 64;
    p.rows = dtype == SPECDEC_DTYPE_F32 ? ((all + (all + 15) / 16 - 1) / ((all + 15) / 16) + 3) / 4 * 4 : page_tokens < TA_MIN_PAGE ? 64 : all <= 16 ? 16 : all <= 32 ? 32 : all <= most_mma ? 64 : all <= 128 || (head_dim > 64 && T > TA_WIDE_T) ? 128 : 256;
    p.tiles = (all + p.rows - 1) / p.rows;
    p.unit = p.rows >= 128 ? 128 : TA_BLOCK;
    p.min_blocks = 4;
    const long long columns = (long long)n_kv_heads * p.tiles, whole = B * columns, blocks = (max_keys + p.unit - 1) / p.unit;
    p.per_sm = dtype != SPECDEC_DTYPE_F32 ? (p.rows >= 128 ? 1 : head_dim > 64 ? 2 : 3)
               : p.rows == 4 ? (whole * blocks >= 4 * TA_SMS ? 4 : 2) : p.rows == 8 || whole > TA_SMS ? 2 : 1;
    const int at_once = TA_SMS * p.per_sm;
    // Whole sequences take their rounds of CTAs times the longest's blocks, stretches an equal share of all blocks and the merge, which costs about as much as eight
    // blocks of 64 keys (of 128 with tcgen05 some four: there fewer sequences are cut than might be).  The longest is what max_length says: 128 x 51 queries over 51 to 307
    // keys take 27 us with it, 41 where it is unknown and the table twice as wide.
    p.direct = (whole + at_once - 1) / at_once * blocks <= whole * blocks / at_once + 8 || B > TA_MAX_B;
    if (p.direct && whole > at_once && 2 * columns <= at_once && B <= TA_MAX_B && p.rows >= 64 && blocks >= 4) p.direct = 2;    // (128 x 51 queries over 51 to 307 keys 29.5 -> 27.9 us; few rows or keys lose 2)
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

template <typename T, int DP>
cudaError_t run_small_pages(const TreeAttn& a, int grid, cudaStream_t st) {
    constexpr int NS = 3, RING = NS * 2 * TA_BLOCK * DP * 2;
    if (const cudaError_t e = op_allow<k_ta_small_pages<T, DP, NS>>(RING + 65 * 32 * 4 + TA_MAX_B * 16)) return e;
    return op_launch(k_ta_small_pages<T, DP, NS>, dim3(ta_grid(a, grid, 2 * TA_SMS)), 128, RING + 65 * a.words * 4 + (a.direct == 1 ? 0 : a.B) * 16, st, 1, a);
}
template <int DP, int RI, int PER_SM>
cudaError_t run_f32(const TreeAttn& a, int grid, cudaStream_t st) {
    using Cfg = TfCfg<DP, RI, PER_SM>;
    constexpr int BYTES = Cfg::FLOATS * 4;
    if (const cudaError_t e = op_allow<k_ta_f32<DP, RI, PER_SM>>(BYTES + (Cfg::ROWS + 1) * 32 * 4 + TA_MAX_B * 16)) return e;
    return op_launch(k_ta_f32<DP, RI, PER_SM>, dim3(ta_grid(a, grid, PER_SM * TA_SMS)), 32 * Cfg::WK, BYTES + (Cfg::ROWS + 1) * a.words * 4 + (a.direct == 1 ? 0 : a.B) * 16, st, 1, a);
}
template <int DP>
cudaError_t pick_f32(const TreeAttn& a, const Plan& p, cudaStream_t st) {
    const int grid = (int)p.grid;
    if (p.rows == 4) return p.per_sm == 4 ? run_f32<DP, 1, 4>(a, grid, st) : run_f32<DP, 1, 2>(a, grid, st);
    if (p.rows == 8) return run_f32<DP, 2, 2>(a, grid, st);
    if (p.rows == 12) return p.per_sm == 2 ? run_f32<DP, 3, 2>(a, grid, st) : run_f32<DP, 3, 1>(a, grid, st);
    return p.per_sm == 2 ? run_f32<DP, 4, 2>(a, grid, st) : run_f32<DP, 4, 1>(a, grid, st);
}
template <typename T>
cudaError_t run_merge(const TreeAttn& a, int rows, cudaStream_t st) {
    const long long every = (long long)a.B * a.kv_heads * a.T * a.group, most = 8 * TA_SMS;
    const bool four = every >= 4 * most;
    const long long ctas = (four ? every / 4 : every) / 4 + 1;
    return op_launch(four ? k_ta_merge<T, 4, 1> : k_ta_merge<T, 1, 8>, dim3((unsigned)(ctas < most ? ctas : most)), 128, 0, st, 1, a, rows);
}
PFN_encodeTiled encoder() {
    static const PFN_encodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess ? (PFN_encodeTiled)p : nullptr;
    }();
    return fn;
}
bool tensor_map(CUtensorMap& tm, const specdec_cache* c, const void* keys) {
    const cuuint64_t e = 2;
    cuuint64_t dims[5] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->n_heads, (cuuint64_t)c->page_tokens, (cuuint64_t)c->n_pages, 2};
    auto of = [&](long long stride, int extent) -> cuuint64_t { return (extent > 1 ? stride : c->head_dim) * e; };
    cuuint64_t strides[4] = {of(c->stride_head, c->n_heads), of(c->stride_token, c->page_tokens), of(c->stride_page, c->n_pages), c->stride_side * e};
    cuuint32_t box[5] = {64, 1, (cuuint32_t)(c->page_tokens < TA_BLOCK ? c->page_tokens : TA_BLOCK), 1, 1}, one[5] = {1, 1, 1, 1, 1};
    return encoder() && encoder()(&tm, c->dtype == SPECDEC_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5, const_cast<void*>(keys), dims, strides,
                                  box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_tree_attention_workspace(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int dtype, int page_tokens, int max_length) {
    if (B < 0 || T < 1 || T > 1024 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || head_dim < 8 || head_dim > 128 || head_dim % 8 ||
        !op_elem_bytes(dtype) || page_tokens < 1 || max_length < 0)
        return op_bad("tree_attention_workspace", "sizes that tree_attention does not take");
    if (B == 0) return 0;
    // Unknown lengths: the longest.  Sequences are cut into the more parts the longer they are, and never where they need not be cut however long they are.
    return workspace(plan(B, T, n_q_heads, n_kv_heads, dtype, head_dim, page_tokens, (max_length ? max_length : 0x7fffffffLL) + T), B, n_kv_heads, head_dim);
}

int specdec_tree_attention(const specdec_cache* c, const specdec_tree_attention_args* g, void* stream) {
    const char* who = "tree_attention";
    if (!c || !g || !c->d_kv || !c->d_table || !c->d_length || !c->d_status || (g->B && (!g->d_q || !g->d_out || !g->d_seqs || !g->d_mask))) return op_bad(who, "a pointer is NULL");
    const int e = op_elem_bytes(c->dtype);
    if (!e) return op_bad(who, "unknown dtype");
    if (g->B < 0 || g->B > 65535 || g->T < 1 || c->n_layers < 1 || g->layer < 0 || g->layer >= c->n_layers || c->n_heads < 1 || c->n_heads > 65535 ||
        g->n_q_heads < 1 || g->n_q_heads % c->n_heads || c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1 || g->max_length < 0)
        return op_bad(who, "a size is out of range, or the query heads are no multiple of the K/V heads");
    if (c->page_tokens < 1 || (c->page_tokens & (c->page_tokens - 1))) return op_bad(who, "page_tokens is not a power of two");
    if ((long long)c->max_pages * c->page_tokens > 0x7fffffffLL - 65536) return op_bad(who, "a sequence could pass 2^31 tokens");
    if (g->T > 1024) return op_fail(SPECDEC_ERR_CAPACITY, who, "trees have at most 1024 nodes");
    if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return op_fail(SPECDEC_ERR_UNSUPPORTED, who, "head_dim is no multiple of 8 up to 128");
    const long long st[5] = {op_stride(c->stride_layer, c->n_layers), c->stride_side, op_stride(c->stride_page, c->n_pages), op_stride(c->stride_token, c->page_tokens),
                             op_stride(c->stride_head, c->n_heads)};
    for (long long s : st) if (s < 0 || s * e % 16) return op_bad(who, "a stride of the cache is negative or not a multiple of 16 bytes");
    if ((uintptr_t)c->d_kv % 16 || (uintptr_t)g->d_q % e || (uintptr_t)g->d_out % e) return op_bad(who, "d_kv is not 16-byte aligned, or q or out not to its type");
    if (!(g->scale > 0.f) || g->scale > 3e38f) return op_bad(who, "scale is not a positive number");
    if (g->B == 0) return SPECDEC_OK;
    TreeAttn a;
    a.q = (const char*)g->d_q; a.out = (char*)g->d_out;
    a.k = (const char*)c->d_kv + g->layer * st[0] * e; a.v = a.k + st[1] * e;
    a.q_sb = op_stride(g->q_stride_b, g->B) * e; a.q_st = op_stride(g->q_stride_t, g->T) * e; a.q_sh = op_stride(g->q_stride_h, g->n_q_heads) * e;
    a.o_sb = op_stride(g->out_stride_b, g->B) * e; a.o_st = op_stride(g->out_stride_t, g->T) * e; a.o_sh = op_stride(g->out_stride_h, g->n_q_heads) * e;
    a.s_page = st[2] * e; a.s_token = st[3] * e; a.s_head = st[4] * e;
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
    const Plan p = plan(a.B, a.T, g->n_q_heads, c->n_heads, c->dtype, a.dim, c->page_tokens, (long long)a.max_length + a.T);
    if (p.grid > 0x7fffffff || p.slots > 0x7fffffff || (long long)a.B * a.kv_heads * a.T * a.group > 0x7fffffff - 65536) return op_fail(SPECDEC_ERR_CAPACITY, who, "too many sequences, heads and nodes for one launch");
    a.tiles = p.tiles; a.direct = p.direct; a.ctas = p.ctas; a.unit = p.unit; a.min_blocks = p.min_blocks;
    const long long need = workspace(p, a.B, c->n_heads, c->head_dim);
    if (need && (!g->d_workspace || (uintptr_t)g->d_workspace % 16 || g->workspace_bytes < need))
        return op_fail(SPECDEC_ERR_CAPACITY, who, "the workspace is smaller than specdec_tree_attention_workspace says, or not 16-byte aligned");
    a.part = (float*)g->d_workspace;
    a.part_ml = (float2*)(a.part + part_floats(p, a.dim));
    a.where = (int2*)(a.part_ml + p.slots * p.rows);
    const cudaStream_t s = (cudaStream_t)stream;
    const bool wide = a.dim > 64, bf = c->dtype == SPECDEC_DTYPE_BF16;
    cudaError_t rc;
    CUtensorMap tm;
    if (c->dtype == SPECDEC_DTYPE_F32) rc = wide ? pick_f32<128>(a, p, s) : pick_f32<64>(a, p, s);
    else if (c->page_tokens < TA_MIN_PAGE) {
        if (bf) rc = wide ? run_small_pages<__nv_bfloat16, 128>(a, (int)p.grid, s) : run_small_pages<__nv_bfloat16, 64>(a, (int)p.grid, s);
        else rc = wide ? run_small_pages<__half, 128>(a, (int)p.grid, s) : run_small_pages<__half, 64>(a, (int)p.grid, s);
    } else {
        if (!tensor_map(tm, c, a.k)) return op_fail(SPECDEC_ERR_CUDA, who, "the driver makes no tensor map of this cache");
        rc = p.rows >= 128 ? ta_tc(tm, a, c->dtype, p.rows, (int)p.grid, s) : ta_tma_mma(tm, a, c->dtype, p.rows, (int)p.grid, s);
    }
    if (rc == cudaSuccess && need) rc = c->dtype == SPECDEC_DTYPE_F32 ? run_merge<float>(a, p.rows, s) : bf ? run_merge<__nv_bfloat16>(a, p.rows, s) : run_merge<__half>(a, p.rows, s);
    return op_done(who, rc);
}

}  // extern "C"
