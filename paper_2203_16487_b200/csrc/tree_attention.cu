// Attention of drafted trees over the caller's paged cache (contract: specdec.h): entry point, warp-level kernels, merge of split keys.
//
// out = sum_j p_j v_j over the keys a query sees, p = softmax(scale q . k).  One pass over the keys with the running maximum m and sum l of
// 2^(s - m): s in units of log2, sums and outputs in fp32, rescaled where m grows.  All query heads of a K/V head share its keys, so a row tile
// mixes nodes and heads; few rows: the keys of a sequence are split over CTAs, whose partial outputs k_ta_merge joins.
#include <cstdlib>
#include "tree_attention.cuh"

namespace sd {
namespace {

// ------------------------------------------------------------------ 16-bit types, pages of fewer than TA_MIN_PAGE tokens
// Such pages are no TMA boxes: every thread fetches 16-byte pieces (cp.async).  4 warps of 16 rows, a ring of NS blocks of 64 keys, rows of
// DP elements whose 16-byte pieces are XORed with the row's low three bits.
template <typename T, int DP, int NS>
__global__ void __launch_bounds__(128) k_ta_small_pages(TreeAttn a) {
    constexpr int ROWS = 64, KT = TA_BLOCK, PITCH = DP * 2, PIECES = DP / 8, STAGE = 2 * KT * PITCH;
    extern __shared__ __align__(128) char sm[];
    char* ring = sm;                                      // [NS][K, V][KT][PITCH]; at first the queries
    int* units = (int*)(sm + NS * STAGE);
    uint32_t* any = (uint32_t*)(units + (a.direct ? 0 : a.B));
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, wm = tid >> 5;
    TaWork work;
    work.begin(a, units);
    Part it;
    while (work.next(a, units, it, tid == 0)) {
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
        rows.block(qf, k_begin + j * KT, s.len, a.scale, a.words, live_a ? mask_a : nullptr, live_b ? mask_b : nullptr,
                   [&](int r, int c) { return ks + r * PITCH + ((c ^ (r & 7)) << 4); }, [&](int r, int c) { return vs + r * PITCH + ((c ^ (r & 7)) << 4); });
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    rows.finish(live_a, live_b);
    rows.store(a, it, r0, ra, ROWS);
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
    int* units = reinterpret_cast<int*>(row_f + 48);
    uint32_t* any = reinterpret_cast<uint32_t*>(units + (a.direct ? 0 : a.B));
    uint32_t* mask = any + a.words;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    TaWork work;
    work.begin(a, units);
    Part it;
    while (work.next(a, units, it, tid == 0)) {
    __syncthreads();
    const int b = it.b, h = it.h, r0 = it.tile * TF_ROWS, all_rows = a.T * a.group;
    const SeqKeys& s = it.s;
    ta_load_masks<128, 0>(a, b, r0, min(TF_ROWS, all_rows - r0), s.nodes, mask, any);
    for (int i = tid; i < TF_ROWS * DP; i += 128) {
        const int r = i / DP, d = i % DP, gr = r0 + r;
        float x = 0.f;
        if (gr < all_rows && d < a.dim) x = *reinterpret_cast<const float*>(a.q + b * a.q_sb + (gr / a.group) * a.q_st + (h * a.group + gr % a.group) * a.q_sh + d * 4);
        q[r * KP + d] = x;
    }
    if (tid < 16) { row_f[16 + tid] = -INFINITY; row_f[32 + tid] = 0.f; }
    const int t0 = r0 / a.group;
    const int k_begin = it.k_begin, k_end = it.k_end;
    constexpr int DC = DP / 4, RG = 128 / DC, RR = TF_ROWS / RG;           // output: DC column groups of 4, RG row groups of RR rows
    const int oc = tid % DC, og = tid / DC;
    float4 o[RR];
#pragma unroll
    for (int i = 0; i < RR; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = k_begin; k0 < k_end; k0 += TF_KT) {
        __syncthreads();
        for (int i = tid; i < TF_KT * (DP / 4); i += 128) {
            const int r = i / (DP / 4), c = i % (DP / 4), key = k0 + r;
            bool real = key < k_end && c * 4 < a.dim && ta_seen(any, s, key);
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
    const long long slot = it.slot * TF_ROWS;
#pragma unroll
    for (int i = 0; i < RR; ++i) {
        const int r = og * RR + i, gr = r0 + r;
        if (gr >= all_rows || oc * 4 >= a.dim) continue;
        const float l = row_f[32 + r];
        if (l == 0.f) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);               // sees nothing: values times 0
        if (it.whole) {
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
}

// ------------------------------------------------------------------ merge
template <typename T> __device__ __forceinline__ void put(char* p, float x);
template <> __device__ __forceinline__ void put<float>(char* p, float x) { *reinterpret_cast<float*>(p) = x; }
template <> __device__ __forceinline__ void put<__nv_bfloat16>(char* p, float x) { *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ void put<__half>(char* p, float x) { *reinterpret_cast<__half*>(p) = __float2half_rn(x); }

// The parts' outputs, each rescaled to the largest maximum: one warp a query row, CTAs that stay.
template <typename T>
__global__ void __launch_bounds__(128) k_ta_merge(TreeAttn a, int rows) {
    const int lane = threadIdx.x & 31, ht = a.kv_heads * a.tiles, all = a.T * a.group;
    cudaGridDependencySynchronize();
    for (int w = blockIdx.x * 4 + (threadIdx.x >> 5); w < a.B * a.kv_heads * all; w += gridDim.x * 4) {
        const int bh = w / all, gr = w - bh * all, b = bh / a.kv_heads, h = bh - b * a.kv_heads, tile = gr / rows, r = gr - tile * rows;
        const int2 at = a.where[bh * a.tiles + tile];     // first slot, parts
        if (at.y <= 1) continue;
        const long long slot0 = (long long)at.x * rows + r, step = (long long)ht * rows;
        float m = -INFINITY;
        for (int s = lane; s < at.y; s += 32) m = fmaxf(m, a.part_ml[slot0 + s * step].x);
#pragma unroll
        for (int of = 16; of; of >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, of));
        const float z = m == -INFINITY ? 0.f : m;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);       // lane: four columns
        float l = 0.f;
#pragma unroll 4
        for (int s = 0; s < at.y; ++s) {
            const long long slot = slot0 + s * step;
            const float2 ml = a.part_ml[slot];
            const float f = exp2f(ml.x - z);
            l += ml.y * f;
            if (lane * 4 < a.dim) {
                const float4 x = *reinterpret_cast<const float4*>(a.part + slot * a.dim + lane * 4);
                o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
            }
        }
        if (lane * 4 >= a.dim) continue;
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
        const int t = ta_node(a, gr);
        char* p = a.out + b * a.o_sb + t * a.o_st + (h * a.group + gr - t * a.group) * a.o_sh + lane * 4 * sizeof(T);
        put<T>(p, o.x * inv); put<T>(p + sizeof(T), o.y * inv); put<T>(p + 2 * sizeof(T), o.z * inv); put<T>(p + 3 * sizeof(T), o.w * inv);
    }
}

// ------------------------------------------------------------------ host
struct Plan { int rows, tiles, direct, ctas, unit, min_units; long long grid, slots; };       // see TreeAttn; slots of partial results
// Rows of a tile: 16, 32 or 64 by the rows there are (64 share a block's keys among four warps; fewer rows give the warps keys of their own instead).
Plan plan(int B, int T, int n_q_heads, int n_kv_heads, int dtype, int head_dim, int page_tokens, long long max_keys) {
    const int all = T * (n_q_heads / n_kv_heads);
    Plan p;
    static const int thr = getenv("TA_THR") ? atoi(getenv("TA_THR")) : 64;
    p.rows = dtype == SPECDEC_DTYPE_F32 ? TF_ROWS : page_tokens < TA_MIN_PAGE ? 64 : all <= 16 && thr >= 16 ? 16 : all <= 32 && thr>=32 ? 32 : all <= thr ? 64 : all <= 128 ? 128 : 256;
    p.tiles = (all + p.rows - 1) / p.rows;
    p.unit = p.rows >= 128 ? 128 : TA_BLOCK;
    p.min_units = p.rows >= 128 ? 4 : 4;
    const int at_once = TA_SMS * (p.rows >= 128 ? 1 : head_dim > 64 ? 2 : 3);          // CTAs that an SM holds at least
    const long long columns = (long long)n_kv_heads * p.tiles, whole = B * columns, units = (max_keys + p.unit - 1) / p.unit;
    // With work for every CTA twice over, only long sequences are worth cutting, and the merge that follows.
    p.direct = units <= (whole >= 2 * at_once ? 4 * p.min_units : p.min_units) || B > TA_MAX_B;
    p.ctas = (int)(at_once / columns < 1 ? 1 : at_once / columns);
    const long long most = (B * units + p.min_units - 1) / p.min_units;                // stretches at most
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
    static const cudaError_t attr = cudaFuncSetAttribute(k_ta_small_pages<T, DP, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize, RING + 65 * 32 * 4 + TA_MAX_B * 4);
    if (attr != cudaSuccess) return attr;
    k_ta_small_pages<T, DP, NS><<<grid, 128, RING + 65 * a.words * 4 + (a.direct ? 0 : a.B) * 4, st>>>(a);
    return cudaGetLastError();
}
template <int DP>
cudaError_t run_f32(const TreeAttn& a, int grid, cudaStream_t st) {
    constexpr size_t FLOATS = (TF_ROWS + 2 * TF_KT) * (DP + 4) + TF_ROWS * (TF_KT + 4) + 48;
    static const cudaError_t attr = cudaFuncSetAttribute(k_ta_f32<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, FLOATS * 4 + (TF_ROWS + 1) * 32 * 4 + TA_MAX_B * 4);
    if (attr != cudaSuccess) return attr;
    k_ta_f32<DP><<<grid, 128, FLOATS * 4 + (TF_ROWS + 1) * a.words * 4 + (a.direct ? 0 : a.B) * 4, st>>>(a);
    return cudaGetLastError();
}
// The merge is launched while the items run, and waits for them.
template <typename T>
cudaError_t run_merge(const TreeAttn& a, int rows, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    const long long ctas = ((long long)a.B * a.kv_heads * a.T * a.group + 3) / 4;
    cfg.gridDim = dim3((unsigned)(ctas < 8 * TA_SMS ? ctas : 8 * TA_SMS)); cfg.blockDim = dim3(128); cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization; at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_ta_merge<T>, a, rows);
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
    cuuint64_t strides[4] = {c->stride_head * e, c->stride_token * e, c->stride_page * e, c->stride_side * e};
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
    return workspace(plan(B, T, n_q_heads, n_kv_heads, dtype, head_dim, page_tokens, (long long)max_length + T), B, n_kv_heads, head_dim);
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
    a.tiles = p.tiles; a.direct = p.direct; a.ctas = p.ctas; a.unit = p.unit; a.min_units = p.min_units;
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
    if (c->dtype == SPECDEC_DTYPE_F32) rc = wide ? run_f32<128>(a, (int)p.grid, s) : run_f32<64>(a, (int)p.grid, s);
    else if (c->page_tokens < TA_MIN_PAGE) {
        if (bf) rc = wide ? run_small_pages<__nv_bfloat16, 128>(a, (int)p.grid, s) : run_small_pages<__nv_bfloat16, 64>(a, (int)p.grid, s);
        else rc = wide ? run_small_pages<__half, 128>(a, (int)p.grid, s) : run_small_pages<__half, 64>(a, (int)p.grid, s);
    } else {
        if (!tensor_map(tm, c, a.k)) return op_fail(SPECDEC_ERR_CUDA, who, "the driver makes no tensor map of this cache");
        rc = p.rows >= 128 ? ta_tc(tm, a, c->dtype, p.rows, (int)p.grid, s) : ta_tma_mma(tm, a, c->dtype, p.rows, (int)p.grid, s);
    }
    if (rc == cudaSuccess && need) rc = c->dtype == SPECDEC_DTYPE_F32 ? run_merge<float>(a, p.rows, s) : bf ? run_merge<__nv_bfloat16>(a, p.rows, s) : run_merge<__half>(a, p.rows, s);
    return rc == cudaSuccess ? SPECDEC_OK : op_fail(SPECDEC_ERR_CUDA, who, cudaGetErrorString(rc));
}

}  // extern "C"
