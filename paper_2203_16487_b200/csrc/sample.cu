// One token per row of logits from a given uniform number: temperature, top-k, top-p, min-p (contract: specdec.h).
//
// Weights are whole numbers of 2^-40 of the largest, so every sum is exact and neither the order of atomics nor the split of the work can
// change a token.  With x = (l - max) / T falling along the order of the logits, an entry's weight is 0 beyond x = -27.73.
//
// A row is read from memory once, into the shared memory of one CTA or, where rows are few or long, of a cluster of up to 8, each with an equal stretch.  What a row
// goes through depends on its parameters:
//   greedy  the first index of the maximum.
//   few     top-k of at most SA_FEW.  The k-th largest of a CTA's threads' own maxima is a bound below the k-th largest entry, and so is, in a cluster of C, the least of the
//           CTAs' (k / C)-th; only the entries above the best bound are looked at again: a list of some k to 3k, ranked by counting, cut, and walked in index order.  No
//           exponential of the others is taken.  (3328 rows of 32768 bf16: k = 128 127 us, k = 129 by the histogram 299.)
//   window  top-p alone: the numbers of entries in 3000 equal steps of x, without an exponential, give a window of a few steps that the cut must lie in; one pass over
//           all weights then has their sum, what is ahead of the window, and a list of what is in it.
//   order   larger top-k, and what a window's list does not hold: a histogram over 1024 equal steps of x gives the step in which the cut falls, and a list of that step's
//           entries, ranked by counting, the cut itself.  (More entries in a step than the list holds: that step's range of logits, as ordered integers, is split into 1024
//           again until a bin is one value; entries equal to it have equal weights, so how many of them stay is arithmetic; which, is by index.)
//   then    the kept weights by stretches of the row, one a warp, and the goal's stretch entry by entry.
//
// What bounds it is the instruction rate: per entry the exponential and its two whole parts are some 20 instructions, the histogram adds one atomic (shared memory takes
// about ten lanes a clock).  3328 rows of 32768 bf16 (218 MB, 33 us at the memory's rate), every row: greedy 46 us, top-k 40 83, no cut 128, top-p 249 (by the histogram
// over 1024 steps, which takes every exponential twice, 287).  64 rows of 131072 with top-p: 34 us, by the histogram 45.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "barriers.cuh"
#include "op_error.cuh"

namespace sd {
namespace {

typedef unsigned long long u64;
constexpr int SA_BINS = 1024, SA_FINE = 3000, SA_FEW = 128, SA_LIST = 512, SA_WIDE = 1024;
constexpr float SA_RANGE = 27.75f;                        // e^-27.73 = 2^-40

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T lowest();                              // -inf
template <> __device__ __forceinline__ float lowest<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __nv_bfloat16 lowest<__nv_bfloat16>() { return __float2bfloat16_rn(-INFINITY); }
template <> __device__ __forceinline__ __half lowest<__half>() { return __float2half_rn(-INFINITY); }

template <typename T> __device__ __forceinline__ T zero();
template <> __device__ __forceinline__ float zero<float>() { return 0.f; }
template <> __device__ __forceinline__ __nv_bfloat16 zero<__nv_bfloat16>() { return __float2bfloat16_rn(0.f); }
template <> __device__ __forceinline__ __half zero<__half>() { return __float2half_rn(0.f); }

// Order-preserving integer of a logit; NaN lowest, the two zeros equal.
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);
    return l != l ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
constexpr uint32_t KEY_NEG_INF = 0x007fffffu;

struct SampleArgs {
    const void* logits; long long stride; int V;
    const float* uniform; const float* temperature; const int* top_k; const float* top_p; const float* min_p; int per_param;
    int* token; float* logprob;
};

// floor(w 2^40) as 2^20 hi + lo for w in [0, 1]: additions that round down leave the whole parts in the low bits of a float (no conversions).
constexpr uint32_t MAGIC = 0x4b000000u;                   // 2^23
__device__ __forceinline__ void split_units(float w, uint32_t& hi, uint32_t& lo) {          // both with MAGIC added
    const float t = __fmaf_rd(w, 1048576.f, 8388608.f);
    const float rest = fmaf(w, 1048576.f, 8388608.f - t);                                    // exact
    hi = __float_as_uint(t);
    lo = __float_as_uint(__fmaf_rd(rest, 1048576.f, 8388608.f));
}
// Two floats at a time (the same results as one at a time).
__device__ __forceinline__ u64 pair2(float lo, float hi) { u64 d; asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi)); return d; }
__device__ __forceinline__ float lo2(u64 d) { return __uint_as_float((uint32_t)d); }
__device__ __forceinline__ float hi2(u64 d) { return __uint_as_float((uint32_t)(d >> 32)); }
__device__ __forceinline__ u64 add2(u64 a, u64 b) { u64 d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ u64 mul2(u64 a, u64 b) { u64 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) { u64 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ u64 fma2_rd(u64 a, u64 b, u64 c) { u64 d; asm("fma.rm.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
// split_units of two weights.
__device__ __forceinline__ void split_units2(u64 w, u64& hi, u64& lo) {
    const u64 scale = pair2(1048576.f, 1048576.f), magic = pair2(8388608.f, 8388608.f);
    hi = fma2_rd(w, scale, magic);
    lo = fma2_rd(fma2(w, scale, fma2(hi, pair2(-1.f, -1.f), magic)), scale, magic);
}

// What turns a logit into a weight.  (Rows whose maximum is +inf, or whose 1 / T is, have been rewritten to 0 and -inf: nothing here is inf - inf.)
struct Row {
    float top, inv_t;
    __device__ __forceinline__ float x_of(float l) const { return __fmul_rn(l - top, inv_t); }        // (never one rounding with what follows)
    __device__ __forceinline__ u64 x_of2(u64 l) const { return mul2(add2(l, pair2(-top, -top)), pair2(inv_t, inv_t)); }
    __device__ __forceinline__ float w_of(float l) const { return fmaxf(expf(x_of(l)), 0.f); }          // NaN: 0
    __device__ __forceinline__ static u64 units(float w) {
        uint32_t hi, lo;
        split_units(w, hi, lo);
        return ((u64)(hi - MAGIC) << 20) + (lo - MAGIC);
    }
    // step of x, to the nearest: 0 for the largest; SA_BINS and more: weight 0 (NaN, -inf and all that is too small)
    static constexpr float STEPS = SA_BINS / SA_RANGE, FINE_STEPS = SA_FINE / SA_RANGE;
    __device__ __forceinline__ static uint32_t bin_of(float x) { return __float_as_uint(fmaf(x, -STEPS, 8388608.f)) - MAGIC; }
};

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ u64 warp_scan(u64 v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const u64 u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += u; }
    return v;
}

struct Hist {
    alignas(16) uint32_t cnt[SA_BINS]; uint32_t lo[SA_BINS + 32], hi[SA_BINS]; // entries; weight as two words (bins beyond the last: a lane each for what weighs nothing)
    template <int NT> __device__ __forceinline__ void clear() { for (int i = threadIdx.x; i < SA_BINS; i += NT) { cnt[i] = 0; lo[i] = 0; hi[i] = 0; } }
    __device__ __forceinline__ u64 sum(int b) const { return (u64)hi[b] << 32 | lo[b]; }
    __device__ __forceinline__ void add(int b, u64 u) {
        const uint32_t l = (uint32_t)u, old = atomicAdd(lo + b, l), h = (uint32_t)(u >> 32) + (old + l < old);
        if (h) atomicAdd(hi + b, h);
    }
};
template <int NT> struct Shared {
    union {
        Hist h;
        struct { u64 units[SA_FEW], part[8][SA_FEW]; };   // few, once the histogram of maxima has been searched
        uint32_t fine[SA_FINE + 32];                      // entries by finer steps (a lane each for what weighs nothing)
        struct { u64 wide[SA_WIDE]; uint32_t part_lo[64], part_hi[64]; };  // a longer list and the weights of parts of it, once the finer steps have been searched
    };
    u64 any[SA_LIST], sorted[SA_LIST];                    // entries as key << 32 | ~index: the order's composite
    int rank[SA_LIST];
    u64 w_sum[32], w_ahead[32];
    int w_cnt[32];
    float w_max[32];
    // what the CTAs of a cluster tell one another (each written once between two barriers)
    float x_top, x_bound, x_share, x_weight;
    int x_bin, x_end, x_window, x_n;
    u64 x_cnt, x_sum, x_cnt_before, x_sum_before, x_total;
    // answers
    int bin, bin_end, n_window, n_list, index, winner;
    u64 cnt_before, sum_before, total, cut, cut_sum;
};

// The CTAs of a row: their barrier, and the shared memory of the others.
template <int C> struct Group {
    int rank;
    __device__ __forceinline__ Group() { if (C > 1) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank)); else rank = 0; }
    __device__ __forceinline__ void sync() const { if (C > 1) tc_cluster_sync(); else __syncthreads(); }
    template <typename S> __device__ __forceinline__ S* of(S* mine, int r) const {
        if (C == 1) return mine;
        u64 p;
        asm("mapa.u64 %0, %1, %2;" : "=l"(p) : "l"((u64)mine), "r"(r));
        return (S*)p;
    }
};
// Sum over the warps ahead of this one, and over all, of what each warp's lane 0 left in v[].
template <int NT, typename V> __device__ __forceinline__ V warps_before(const V* v, V& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V x = lane < NT / 32 ? v[lane] : V(0);
    const V own = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const V y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
    all = __shfl_sync(0xffffffffu, x, 31);
    return __shfl_sync(0xffffffffu, x - own, warp);
}

// First bin, in ascending order, behind which the search ends: by entries (the bin that holds entry number `k` from 1) or by weight (the last bin of any
// weight with weight ahead < thr), over the histograms of C CTAs (1: this one's alone).  sh.cnt_before / sum_before: what is ahead of it, added to what was given.  sh.bin = -1: none
// (k beyond all).  Each CTA searches its share of the bins.
// share > 0: thr is that share of all weight, which is left in sh.total.
template <int NT, int C>
__device__ void find_bin(Shared<NT>& sh, const Group<C>& cta, bool by_weight, u64 k, double thr, u64 cnt0, u64 sum0, float share = 0.f) {
    constexpr int SHARE = SA_BINS / C, PER = SHARE >= NT ? SHARE / NT : 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b0 = cta.rank * SHARE + threadIdx.x * PER;
    const bool mine = threadIdx.x * PER < SHARE;
    uint32_t n[PER];
    u64 w[PER], c = 0, s = 0;
    cta.sync();                                           // the histograms are complete
#pragma unroll
    for (int j = 0; j < PER; ++j) { n[j] = 0; w[j] = 0; }
    if (mine)
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const Hist* h = cta.of(&sh.h, r);
#pragma unroll
            for (int j = 0; j < PER; ++j) { n[j] += h->cnt[b0 + j]; w[j] += h->sum(b0 + j); }
        }
#pragma unroll
    for (int j = 0; j < PER; ++j) { c += n[j]; s += w[j]; }
    const u64 ic = warp_scan(c), is = warp_scan(s);
    if (lane == 31) { sh.w_cnt[warp] = (int)ic; sh.w_sum[warp] = is; }
    if (threadIdx.x == 0) sh.bin = -1;
    __syncthreads();
    int cta_c;
    u64 cta_s;
    u64 bc = cnt0 + warps_before<NT>(sh.w_cnt, cta_c) + ic - c, bs = sum0 + warps_before<NT>(sh.w_sum, cta_s) + is - s, all = cta_s;
    if (C > 1) {                                          // shares ahead of this CTA's
        if (threadIdx.x == 0) { sh.x_cnt = cta_c; sh.x_sum = cta_s; }
        cta.sync();
        all = 0;
        for (int r = 0; r < C; ++r) {
            const Shared<NT>* o = cta.of(&sh, r);
            if (r < cta.rank) { bc += o->x_cnt; bs += o->x_sum; }
            all += o->x_sum;
        }
    }
    if (share > 0.f) thr = (double)share * (double)all;
    if (threadIdx.x == 0) sh.total = all;
    int found = -1;
    u64 mc = 0, ms = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (by_weight ? w[j] && (double)bs < thr : (bc < k && k <= bc + n[j])) { found = b0 + j; mc = bc; ms = bs; }
        bc += n[j]; bs += w[j];
    }
    if (found >= 0) atomicMax(&sh.bin, found);
    __syncthreads();
    if (found >= 0 && sh.bin == found) { sh.cnt_before = mc; sh.sum_before = ms; }
    __syncthreads();
    if (C > 1) {                                          // of the CTAs' answers the last
        if (threadIdx.x == 0) { sh.x_bin = sh.bin; sh.x_cnt_before = sh.cnt_before; sh.x_sum_before = sh.sum_before; }
        cta.sync();
        if (threadIdx.x == 0) {
            int best = -1;
            for (int r = 0; r < C; ++r) {
                const Shared<NT>* o = cta.of(&sh, r);
                if (o->x_bin > best) { best = o->x_bin; sh.cnt_before = o->x_cnt_before; sh.sum_before = o->x_sum_before; }
            }
            sh.bin = best;
        }
        __syncthreads();
    }
}

// The finer steps [sh.bin, sh.bin_end) in which the cut by weight must lie, and how many entries they hold (sh.n_window), from the steps' entries (all CTAs').  An entry's weight is within d = 0.6 of a step of its
// step's middle (0.5, and room for roundings), so of all weight A + B the share of the steps ahead lies between A (1 - d) / (A (1 - d) + B (1 + d)) and the same with d's sign turned: a cut at
// 0.95 is known to 0.05 % of all weight before one exponential has been taken.
// Each CTA weighs its share of the steps.  (Floats: an estimate, of which all CTAs see the same numbers; what is made of it is checked with exact sums.)
template <int NT, int C>
__device__ void find_window(Shared<NT>& sh, const Group<C>& cta, float top_p) {
    constexpr int SHARE = SA_FINE / C, PER = (SHARE + NT - 1) / NT;
    static_assert(SA_FINE % C == 0 && SHARE % PER == 0, "equal shares");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b0 = cta.rank * SHARE + threadIdx.x * PER;
    const bool mine = threadIdx.x * PER < SHARE;
    uint32_t n[PER];
    float w[PER], s = 0.f;
    cta.sync();                                           // the counts are complete
#pragma unroll
    for (int j = 0; j < PER; ++j) n[j] = 0;
    if (mine)
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const uint32_t* fine = cta.of(&sh, r)->fine + b0;
#pragma unroll
            for (int j = 0; j < PER; ++j) n[j] += fine[j];
        }
#pragma unroll
    for (int j = 0; j < PER; ++j) { w[j] = n[j] * __expf((b0 + j) * (-1.f / Row::FINE_STEPS)); s += w[j]; }
    float is = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const float y = __shfl_up_sync(0xffffffffu, is, o); if (lane >= o) is += y; }
    if (lane == 31) sh.w_max[warp] = is;
    if (threadIdx.x == 0) { sh.bin = 0; sh.bin_end = SA_FINE; sh.n_window = 0; }
    __syncthreads();
    float all, before = warps_before<NT>(sh.w_max, all) + (is - s);
    if (C > 1) {
        if (threadIdx.x == 0) sh.x_weight = all;
        cta.sync();
        all = 0.f;
        for (int r = 0; r < C; ++r) {
            if (r == cta.rank) before += all;
            all += cta.of(&sh, r)->x_weight;
        }
    }
    constexpr float d = 0.6f / Row::FINE_STEPS;
    const float p = fminf(top_p, 1.f), up = p * (1 + d), down = p * (1 - d), q = 1 - p;
    const float least = down / (down + q * (1 + d)) * all, most = up / (up + q * (1 - d)) * all;
    unsigned first = 0, end = SA_FINE, in = 0;
    if (mine)
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (before <= least) first = b0 + j;
            if (before >= most) end = min(end, (unsigned)(b0 + j));
            else if (before + w[j] > least) in += n[j];
            before += w[j];
        }
    first = __reduce_max_sync(0xffffffffu, first);
    end = __reduce_min_sync(0xffffffffu, end);
    in = __reduce_add_sync(0xffffffffu, in);
    if (lane == 0) {
        if (in) atomicAdd(&sh.n_window, (int)in);
        if (first) atomicMax(&sh.bin, (int)first);
        if (end < SA_FINE) atomicMin(&sh.bin_end, (int)end);
    }
    __syncthreads();
    if (C > 1) {
        if (threadIdx.x == 0) { sh.x_bin = sh.bin; sh.x_end = sh.bin_end; sh.x_window = sh.n_window; }
        cta.sync();
        if (threadIdx.x == 0) {
            sh.n_window = 0;
            for (int r = 0; r < C; ++r) {
                const Shared<NT>* o = cta.of(&sh, r);
                sh.bin = max(sh.bin, o->x_bin); sh.bin_end = min(sh.bin_end, o->x_end); sh.n_window += o->x_window;
            }
        }
        __syncthreads();
    }
}

// The bin, in ascending order, that holds entry number k (from 1), or -1; every warp looks for itself.
__device__ int bin_of_kth(const Hist& hist, int k) {
    static_assert(alignof(Hist) % 16 == 0 && offsetof(Hist, cnt) == 0, "counts are read four at a time");
    const uint32_t* cnt = hist.cnt;
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int i = 0; i < SA_BINS / 128; ++i) {
        const int4 c = reinterpret_cast<const int4*>(cnt)[i * 32 + lane];
        const int s = c.x + c.y + c.z + c.w, all = __reduce_add_sync(0xffffffffu, s);
        if (before + all >= k) {
            int upto = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += y; }
            int bin = -1, b = before + upto - s;
            if (b < k && k <= b + s) {
                bin = i * 128 + lane * 4;
                if ((b += c.x) < k) ++bin;
                if (b < k && (b += c.y) < k) ++bin;
                if (b < k && (b += c.z) < k) ++bin;
            }
            return __reduce_max_sync(0xffffffffu, bin);
        }
        before += all;
    }
    return -1;
}

// Keys whose step is b: [lo, hi].  The step falls as the key grows, so both ends are found by a search of 32 probes at a time.
__device__ void key_range(const Row& row, uint32_t b, uint32_t top_key, uint32_t& lo, uint32_t& hi) {
    const int lane = threadIdx.x & 31;
    auto first_with = [&](uint32_t most) {                     // smallest key in (KEY_NEG_INF, top_key] whose step is <= most
        uint32_t a = KEY_NEG_INF + 1, n = top_key - a;    // the answer is in [a, a + n]
        while (n) {
            const uint32_t step = n / 32 + 1;
            const uint64_t probe = (uint64_t)a + (uint64_t)lane * step;              // last key of which it is known to be below or at
            const bool in = probe >= (uint64_t)a + n || Row::bin_of(row.x_of(of_key((uint32_t)probe))) <= most;
            const unsigned m = __ballot_sync(0xffffffffu, in);
            if (!m) { a += 31 * step + 1; n -= 31 * step + 1; continue; }
            const int f = __ffs(m) - 1;
            if (f == 0) { n = 0; continue; }
            const uint32_t left = a + (f - 1) * step + 1, right = (uint32_t)min((uint64_t)a + (uint64_t)f * step, (uint64_t)a + n);
            a = left; n = right - left;
        }
        return a;
    };
    lo = first_with(b);
    hi = b == 0 ? top_key : first_with(b - 1) - 1;
}

// Maximum of a vector: packed for the 16-bit types.
template <typename T> struct TwoOf { typedef float type; };
template <> struct TwoOf<__nv_bfloat16> { typedef __nv_bfloat162 type; };
template <> struct TwoOf<__half> { typedef __half2 type; };
template <typename T> using Two = typename TwoOf<T>::type;
__device__ __forceinline__ float max4(const float* x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }
__device__ __forceinline__ float max4(const __nv_bfloat162* x) {
    const __nv_bfloat162 m = __hmax2(__hmax2(x[0], x[1]), __hmax2(x[2], x[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float max4(const __half2* x) {
    const __half2 m = __hmax2(__hmax2(x[0], x[1]), __hmax2(x[2], x[3]));
    return fmaxf(__low2float(m), __high2float(m));
}
// A CTA's stretch of a row as 16-byte vectors of N entries in shared memory; the row's first vector may begin ahead of the row (what is ahead and behind is -inf).
// Warp w owns a stretch of vectors; f(value, index) of one warp's share, lane by lane.
template <typename T> struct RowData {
    static constexpr int N = 16 / sizeof(T);
    const T* smem;                                        // the stretch's vector 0
    int first;                                            // index in the row of its entry 0 (the row's lead: negative)
    __device__ __forceinline__ float at(int i) const { return to_f(smem[i - first]); }
    template <typename F> __device__ __forceinline__ void vec(int v, F f) const {
        union { int4 raw; T x[N]; } u;
        u.raw = reinterpret_cast<const int4*>(smem)[v];
#pragma unroll
        for (int j = 0; j < N; ++j) f(to_f(u.x[j]), first + v * N + j);
    }
    __device__ __forceinline__ float most(int v) const {              // a vector's maximum (NaN does not count)
        union { int4 raw; T x[N]; Two<T> two[4]; } u;
        u.raw = reinterpret_cast<const int4*>(smem)[v];
        return max4(u.two);
    }
    __device__ __forceinline__ void pairs(int v, u64* l) const {      // a vector's entries, two by two
        union { int4 raw; T x[N]; } u;
        u.raw = reinterpret_cast<const int4*>(smem)[v];
#pragma unroll
        for (int j = 0; j < N / 2; ++j) l[j] = pair2(to_f(u.x[2 * j]), to_f(u.x[2 * j + 1]));
    }
    template <typename F> __device__ __forceinline__ void each(int v0, int v1, F f) const {       // vectors [v0, v1), by one warp, in few instructions
        for (int v = v0 + (threadIdx.x & 31); v < v1; v += 32)
#pragma unroll 1
            for (int i = first + v * N; i < first + v * N + N; ++i) f(at(i), i);
    }
};
__device__ __forceinline__ u64 composite(float l, int i) { return (u64)key_of(l) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float logit_of(u64 e) { return of_key((uint32_t)(e >> 32)); }

// sh.any[0 .. n) in falling order into sh.sorted (n at most SA_LIST): every entry counts those ahead of it, several threads an entry.
template <int NT>
__device__ void rank_list(Shared<NT>& sh, int n) {
    const int width = n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512, parts = NT / width;
    for (int i = threadIdx.x; i < n; i += NT) sh.rank[i] = 0;
    __syncthreads();
    const int e = threadIdx.x % width;
    if (e < n) {
        const u64 x = sh.any[e];
        int c = 0;
#pragma unroll 4
        for (int j = threadIdx.x / width; j < n; j += parts) c += sh.any[j] > x;
        if (c) atomicAdd(sh.rank + e, c);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) sh.sorted[sh.rank[i]] = sh.any[i];
    __syncthreads();
}

template <typename T, int NT, int C>
__global__ void __launch_bounds__(NT, 1024 / NT) k_sample(SampleArgs a) {
    constexpr int NW = NT / 32, N = RowData<T>::N;
    extern __shared__ __align__(16) char row_smem[];
    __shared__ Shared<NT> sh;
    op_begin();
    const Group<C> cta;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V;
    const int r = blockIdx.x / C, pr = r / a.per_param;
    const T* global = (const T*)a.logits + r * a.stride;
    const int lead = (int)((uintptr_t)global & 15) / (int)sizeof(T), nvec = (lead + V + N - 1) / N;
    const int per_cta = (nvec + C - 1) / C, c0 = min(cta.rank * per_cta, nvec), mine_vec = min(c0 + per_cta, nvec) - c0;
    const RowData<T> data{(const T*)row_smem, c0 * N - lead};
    const int per_warp = (per_cta + NW - 1) / NW, v0 = min(warp * per_warp, mine_vec), v1 = min(v0 + per_warp, mine_vec);
    {                                                     // each thread fetches the vectors that it reads first
        const int4* from = reinterpret_cast<const int4*>(global - lead) + c0;
        for (int v = v0 + lane; v < v1; v += 32) {
            const int i0 = data.first + v * N;
            if (i0 >= 0 && i0 + N <= V) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(row_smem + v * 16)), "l"(from + v) : "memory");
            } else {
                union { int4 raw; T x[N]; } u;
#pragma unroll
                for (int j = 0; j < N; ++j) u.x[j] = i0 + j >= 0 && i0 + j < V ? global[i0 + j] : lowest<T>();
                reinterpret_cast<int4*>(row_smem)[v] = u.raw;
            }
        }
    }
    const float temperature = a.temperature ? a.temperature[pr] : 1.f;
    const float p_in = a.top_p ? a.top_p[pr] : 1.f, m_in = a.min_p ? a.min_p[pr] : 0.f;
    const float top_p = p_in < 1.f ? p_in : 1.f, min_p = m_in > 0.f ? m_in : 0.f;        // (NaN: off)
    const int k_in = a.top_k ? a.top_k[pr] : 0;
    const float u = a.uniform[r];
    const int k = k_in <= 0 || k_in > V ? V : k_in;
    const bool greedy = !(temperature > 0.f) || !(top_p > 0.f) || !(min_p <= 1.f) || k == 1;        // the largest entry alone
    const bool few = k <= SA_FEW && k < V, cuts = k < V || top_p < 1.f;
    if (few) for (int i = tid; i < SA_BINS; i += NT) sh.h.cnt[i] = 0;
    else if (k < V) sh.h.template clear<NT>();
    else if (cuts) for (int i = tid; i < SA_FINE; i += NT) sh.fine[i] = 0;
    if (tid == 0) { sh.index = V; sh.n_list = 0; sh.winner = -1; }
    asm volatile("cp.async.wait_all;" ::: "memory");

    float mine = -INFINITY;                               // this thread's maximum (NaN does not count)
    for (int v = v0 + lane; v < v1; v += 32) mine = fmaxf(mine, data.most(v));
    float top = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) sh.w_max[warp] = top;
    __syncthreads();
    top = lane < NW ? sh.w_max[lane] : -INFINITY;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float cta_top = top;
    if (C > 1) {
        if (tid == 0) sh.x_top = top;
        cta.sync();
        for (int q = 0; q < C; ++q) top = fmaxf(top, cta.of(&sh, q)->x_top);
    }
    if (top == -INFINITY || greedy) {
        if (top > -INFINITY && mine == top) {
            int first = V;
            for (int v = v0 + lane; v < v1; v += 32)
                if (data.most(v) == top) data.vec(v, [&](float l, int i) { if (l == top) first = min(first, i); });
            atomicMin(&sh.index, first);
        }
        if (C > 1) {                                      // the first CTA that holds the maximum answers
            __syncthreads();
            if (tid == 0) {
                bool ahead = false;
                for (int q = 0; q < cta.rank; ++q) ahead |= cta.of(&sh, q)->x_top == top;
                if (!ahead && (cta_top == top)) { a.token[r] = top > -INFINITY ? sh.index : -1; if (a.logprob) a.logprob[r] = top > -INFINITY ? 0.f : -INFINITY; }
            }
            cta.sync();                                   // until the others have read x_top
        } else {
            __syncthreads();
            if (tid == 0) { a.token[r] = top > -INFINITY ? sh.index : -1; if (a.logprob) a.logprob[r] = top > -INFINITY ? 0.f : -INFINITY; }
        }
        return;
    }
    float inv_t = 1.f / temperature;
    if (top == INFINITY || inv_t == INFINITY) {           // only what equals the maximum weighs anything
        for (int v = v0 + lane; v < v1; v += 32) {
            union { int4 raw; T x[N]; } y;
            y.raw = reinterpret_cast<const int4*>(row_smem)[v];
#pragma unroll
            for (int j = 0; j < N; ++j) y.x[j] = to_f(y.x[j]) == top ? zero<T>() : lowest<T>();
            reinterpret_cast<int4*>(row_smem)[v] = y.raw;
        }
        mine = mine == top ? 0.f : -INFINITY;
        top = 0.f; inv_t = 1.f;
        __syncthreads();
    }
    const Row row{top + 0.f, inv_t};
    const uint32_t top_key = key_of(top);
    auto goal_of = [&](u64 total) -> u64 { return u > 0.f ? min((u64)((double)u * (double)total), total - 1) : 0; };
    auto log_of = [](u64 total) { return logf((float)total * 9.094947017729282e-13f); };             // total 2^-40

    if (few) {
        const uint32_t b = Row::bin_of(row.x_of(mine));
        if (b < SA_BINS) atomicAdd(sh.h.cnt + b, 1u);
        __syncthreads();
        // entries from a step on up: all of steps 0 .. bin (a little more does no harm)
        auto from_step = [&](int bin) {
            const float depth = (bin + 0.5f) * (SA_RANGE / SA_BINS) / inv_t;
            return bin < 0 ? -INFINITY : row.top - depth - (fabsf(row.top) + depth) * 1e-6f;
        };
        float bound = from_step(bin_of_kth(sh.h, k));
        if (C > 1) {                                      // k entries of one CTA, or k / C of each
            const float share = from_step(bin_of_kth(sh.h, (k + C - 1) / C));
            if (tid == 0) { sh.x_bound = bound; sh.x_share = share; }
            cta.sync();
            float least = INFINITY;
            for (int q = 0; q < C; ++q) { bound = fmaxf(bound, cta.of(&sh, q)->x_bound); least = fminf(least, cta.of(&sh, q)->x_share); }
            bound = fmaxf(bound, least);
        }
        Shared<NT>* lead_sh = cta.of(&sh, 0);
        // the threads that have seen one, four at a time: eight lanes take a vector each of one thread's
        const unsigned seen = __ballot_sync(0xffffffffu, bound > -INFINITY && mine >= bound);
        int nth = 0;                                      // the lane-th of them
#pragma unroll
        for (int s = 16; s; s >>= 1) if (__popc(seen & ((1u << (nth + s)) - 1)) <= lane) nth += s;
        for (int first = 0; first < __popc(seen); first += 4) {
            const int of = __shfl_sync(0xffffffffu, nth, first + (lane >> 3));
            const bool some = first + (lane >> 3) < __popc(seen);
            for (int v = v0 + of + 32 * (lane & 7), more = v1 - v0; more > 0; v += 256, more -= 256) {
                unsigned in = 0;
                if (some && v < v1) {
                    int bit = 0;
                    data.vec(v, [&](float l, int) { in |= (l >= bound ? 1u : 0u) << bit++; });
                }
                const int n = __popc(in);
                int upto = n;
#pragma unroll
                for (int s = 1; s < 32; s <<= 1) { const int y = __shfl_up_sync(0xffffffffu, upto, s); if (lane >= s) upto += y; }
                int at = 0;
                if (lane == 31 && upto) at = atomicAdd(&lead_sh->n_list, upto);
                at = __shfl_sync(0xffffffffu, at, 31) + upto - n;
                for (; in; in &= in - 1, ++at) {
                    const int i = data.first + v * N + __ffs(in) - 1;
                    if (at < SA_LIST) lead_sh->any[at] = composite(data.at(i), i);
                }
            }
        }
        cta.sync();
        const int n = lead_sh->n_list;
        cta.sync();                                       // all have read it
        if (n >= k && n <= SA_LIST) {
            if (cta.rank) return;
            rank_list<NT>(sh, n);
            if (warp == 0) {                              // the order's cut, and the smaller entries that min_p drops: at most SA_FEW, four a lane
                u64 un[SA_FEW / 32], all = 0;
                float w[SA_FEW / 32];
#pragma unroll
                for (int j = 0; j < SA_FEW / 32; ++j) {
                    const int e = lane * (SA_FEW / 32) + j;
                    w[j] = e < k ? row.w_of(logit_of(sh.sorted[e])) : 0.f;
                    un[j] = Row::units(w[j]);
                    all += un[j];
                }
                const u64 upto = warp_scan(all);
                const u64 total = __shfl_sync(0xffffffffu, upto, 31);
                const double thr = (double)top_p * (double)total;
                u64 before = upto - all, kept = 0;
#pragma unroll
                for (int j = 0; j < SA_FEW / 32; ++j) {
                    const bool keep = (top_p >= 1.f || (double)before < thr) && w[j] >= min_p;
                    before += un[j];
                    un[j] = keep ? un[j] : 0;
                    kept += un[j];
                    sh.units[lane * (SA_FEW / 32) + j] = un[j];
                }
                kept = warp_sum(kept);
                if (lane == 0) sh.total = kept;
            }
            __syncthreads();
            // weight of the kept entries with a lower index, several threads an entry
            constexpr int PARTS = NT / SA_FEW;
            const int e = tid % SA_FEW, p = tid / SA_FEW;
            if (e < k) {
                const uint32_t me = (uint32_t)sh.sorted[e];            // ~index
                u64 s = 0;
#pragma unroll 4
                for (int j = p; j < k; j += PARTS) if ((uint32_t)sh.sorted[j] > me) s += sh.units[j];
                sh.part[p][e] = s;
            }
            __syncthreads();
            if (tid < k) {
                u64 before = 0;
#pragma unroll
                for (int j = 0; j < PARTS; ++j) before += sh.part[j][tid];
                const u64 total = sh.total, goal = goal_of(total);
                if (before <= goal && goal < before + sh.units[tid]) {
                    const u64 x = sh.sorted[tid];
                    a.token[r] = (int)~(uint32_t)x;
                    if (a.logprob) a.logprob[r] = row.x_of(logit_of(x)) - log_of(total);
                }
            }
            return;
        }
        sh.h.template clear<NT>();
        if (tid == 0) sh.n_list = 0;
        __syncthreads();
    }

    u64 cut = 0;                                          // entries with a composite from here on stay
    u64 s = 0;                                            // of this warp's stretch: kept weight
    if (cuts) {
        // the histogram over steps
        auto fill = [&](bool count) {
            for (int v = v0 + lane; v < v1; v += 32) {
                u64 l[N / 2];
                uint32_t b[N], wl[N], wh[N], old[N];
                data.pairs(v, l);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) {
                    const u64 x = row.x_of2(l[j]), step = fma2(x, pair2(-Row::STEPS, -Row::STEPS), pair2(8388608.f, 8388608.f));
                    u64 hi, lo;
                    split_units2(pair2(fmaxf(expf(lo2(x)), 0.f), fmaxf(expf(hi2(x)), 0.f)), hi, lo);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t h = e ? (uint32_t)(hi >> 32) : (uint32_t)hi, w = e ? (uint32_t)(lo >> 32) : (uint32_t)lo;
                        b[2 * j + e] = min((e ? (uint32_t)(step >> 32) : (uint32_t)step) - MAGIC, (uint32_t)SA_BINS + lane);
                        wl[2 * j + e] = (h << 20) + (w - MAGIC);       // (h's offset is a multiple of 2^12)
                        wh[2 * j + e] = (h - MAGIC) >> 12;
                    }
                }
                // all atomics of a vector are on their way before the first answer is looked at
#pragma unroll
                for (int j = 0; j < N; ++j) old[j] = atomicAdd(sh.h.lo + b[j], wl[j]);
                if (count)
#pragma unroll
                    for (int j = 0; j < N; ++j) if (b[j] < SA_BINS) atomicAdd(sh.h.cnt + b[j], 1u);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const uint32_t h = wh[j] + (old[j] + wl[j] < old[j]);
                    if (h) atomicAdd(sh.h.hi + min(b[j], SA_BINS - 1u), h);
                }
            }
        };
        u64 total = 0;                                    // of the k largest, where k cuts
        // All CTAs' lists (each CTA's is list(its shared memory)), behind this one's n entries; the length of the whole.
        auto gather = [&](int n, int most, auto list) {
            __syncthreads();                              // all have read n
            if (C > 1) {
                if (tid == 0) sh.x_n = n;
                cta.sync();
                int at = n;
                for (int q = 0; q < C; ++q) if (q != cta.rank) {
                    const Shared<NT>* o = cta.of(&sh, q);
                    const int m = o->x_n;
                    if (at + m <= most) for (int i = tid; i < m; i += NT) list(&sh)[at + i] = list(o)[i];
                    at += m;
                }
                n = at;
                __syncthreads();
            }
            if (tid == 0) sh.n_list = 0;
            return n;
        };
        // The cut among the list's n entries, with c0 entries of weight s0 ahead of them.  sum: adds to s what stays of them.  Returns the list's weight.
        auto cut_in_list = [&](int n, u64 c0, u64 s0, bool by_weight, double thr, bool sum) {
            rank_list<NT>(sh, n);
            u64 w = 0;
            if (tid < n) w = Row::units(row.w_of(logit_of(sh.sorted[tid])));
            const u64 upto = warp_scan(w);
            if (lane == 31) sh.w_sum[warp] = upto;
            __syncthreads();
            u64 all;
            const u64 before = s0 + warps_before<NT>(sh.w_sum, all) + upto - w;
            // the last entry that stays: by weight the last whose weight ahead is below thr
            const bool stays = tid < n && (by_weight ? (double)before < thr : c0 + tid + 1 <= (u64)k);
            const bool next = tid + 1 < n && (by_weight ? (double)(before + w) < thr : c0 + tid + 2 <= (u64)k);
            if (stays && !next) { sh.cut = sh.sorted[tid]; sh.cut_sum = before + w; }
            __syncthreads();
            if (sum)                                      // those of this warp's stretch
                for (int e = lane; e < n; e += 32) {
                    const u64 y = sh.sorted[e];
                    const int i = (int)~(uint32_t)y;
                    if (y >= sh.cut && i >= data.first + v0 * N && i < data.first + v1 * N) {
                        const float w2 = row.w_of(logit_of(y));
                        if (w2 >= min_p) s += Row::units(w2);
                    }
                }
            return all;
        };
        // By weight alone, in two passes: entries by finer steps, without an exponential, give a window that the cut must lie in; then all weights once, with what is ahead of
        // the window, and a list of what is in it.  Whether the cut was found this way (sh.cut, s): not where the window holds more than the list does.
        auto by_window = [&]() {
            const u64 step2 = pair2(-Row::FINE_STEPS * row.inv_t, -Row::FINE_STEPS * row.inv_t), top2 = pair2(-row.top, -row.top);
            for (int v = v0 + lane; v < v1; v += 32) {
                u64 l[N / 2];
                data.pairs(v, l);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) {
                    const u64 b = fma2(add2(l[j], top2), step2, pair2(8388608.f, 8388608.f));
                    atomicAdd(sh.fine + (min((uint32_t)b, MAGIC + SA_FINE + lane) - MAGIC), 1u);
                    atomicAdd(sh.fine + (min((uint32_t)(b >> 32), MAGIC + SA_FINE + lane) - MAGIC), 1u);
                }
            }
            find_window<NT, C>(sh, cta, top_p);
            if (sh.n_window > SA_WIDE) return false;
            const float unit = SA_RANGE / SA_FINE / row.inv_t;
            const float high = sh.bin ? row.top - (sh.bin - 0.5f) * unit : INFINITY, low = row.top - (sh.bin_end - 0.5f) * unit;
            uint32_t all_hi = 0, all_lo = 0, ahead_hi = 0, ahead_lo = 0, n_ahead = 0, drop_hi = 0, drop_lo = 0, n_drop = 0, n = 0;
            auto weigh = [&](auto drops) {                // drops: whether min_p drops any
                for (int v = v0 + lane; v < v1; v += 32, n += N) {
                    u64 l[N / 2];
                    data.pairs(v, l);
                    unsigned in = 0;                          // those of the window
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) {
                        const u64 x = row.x_of2(l[j]);
                        const float w0 = fmaxf(expf(lo2(x)), 0.f), w1 = fmaxf(expf(hi2(x)), 0.f), l0 = lo2(l[j]), l1 = hi2(l[j]);
                        u64 hi, lo;
                        split_units2(pair2(w0, w1), hi, lo);
                        all_hi += (uint32_t)hi + (uint32_t)(hi >> 32); all_lo += (uint32_t)lo + (uint32_t)(lo >> 32);
                        if (l0 > high) {
                            ahead_hi += (uint32_t)hi; ahead_lo += (uint32_t)lo; ++n_ahead;
                            if (drops.value && !(w0 >= min_p)) { drop_hi += (uint32_t)hi; drop_lo += (uint32_t)lo; ++n_drop; }
                        }
                        if (l1 > high) {
                            ahead_hi += (uint32_t)(hi >> 32); ahead_lo += (uint32_t)(lo >> 32); ++n_ahead;
                            if (drops.value && !(w1 >= min_p)) { drop_hi += (uint32_t)(hi >> 32); drop_lo += (uint32_t)(lo >> 32); ++n_drop; }
                        }
                        if (l0 >= low && !(l0 > high)) in |= 1u << 2 * j;
                        if (l1 >= low && !(l1 > high)) in |= 2u << 2 * j;
                    }
                    for (; in; in &= in - 1) {
                        const int i = data.first + v * N + __ffs(in) - 1, at = atomicAdd(&sh.n_list, 1);
                        if (at < SA_WIDE) sh.wide[at] = composite(data.at(i), i);
                    }
                }
            };
            if (min_p > 0.f) weigh(std::true_type());
            else weigh(std::false_type());
            auto units = [](uint32_t hi, uint32_t lo, uint32_t m) { return ((u64)(hi - m * MAGIC) << 20) + (lo - m * MAGIC); };
            const u64 mine_ahead = units(ahead_hi, ahead_lo, n_ahead);
            const u64 wa = warp_sum(units(all_hi, all_lo, n)), wh = warp_sum(mine_ahead);
            s = mine_ahead - units(drop_hi, drop_lo, n_drop);
            if (lane == 0) { sh.w_sum[warp] = wa; sh.w_ahead[warp] = wh; }
            __syncthreads();
            u64 all, ahead;
            warps_before<NT>(sh.w_sum, all);
            warps_before<NT>(sh.w_ahead, ahead);
            if (C > 1 && tid == 0) { sh.x_sum = all; sh.x_cnt = ahead; }
            const int m = gather(sh.n_list, SA_WIDE, [](auto* o) { return o->wide; });
            if (C > 1) {
                all = ahead = 0;
                for (int q = 0; q < C; ++q) { all += cta.of(&sh, q)->x_sum; ahead += cta.of(&sh, q)->x_cnt; }
            }
            const double thr = (double)top_p * (double)all;
            if (m > SA_WIDE || !((double)ahead < thr)) return false;
            if (m <= SA_LIST / 2) {                       // few enough to be ranked as they are (some 150 entries: 1 us less than in parts; 700: 64 rows of 131072 50 us, in parts 37)
                for (int e = tid; e < m; e += NT) sh.any[e] = sh.wide[e];
                __syncthreads();
                return (double)(ahead + cut_in_list(m, 0, ahead, true, thr, true)) >= thr;
            }
            // the part of the window that holds the cut: of 64 equal ones the last of any weight with weight ahead below thr
            const float from = fminf(high, row.top), scale = 64.f / (from - low);
            auto part_of = [&](u64 e) { return max(0, min((int)((from - logit_of(e)) * scale), 63)); };
            if (tid < 64) sh.part_lo[tid] = sh.part_hi[tid] = 0;
            __syncthreads();
            for (int e = tid; e < m; e += NT) {
                const u64 y = sh.wide[e];
                const u64 w = Row::units(row.w_of(logit_of(y)));
                const int b = part_of(y);
                const uint32_t old = atomicAdd(sh.part_lo + b, (uint32_t)w), h = (uint32_t)(w >> 32) + (old + (uint32_t)w < old);
                if (h) atomicAdd(sh.part_hi + b, h);
            }
            __syncthreads();
            const u64 p0 = (u64)sh.part_hi[2 * lane] << 32 | sh.part_lo[2 * lane], p1 = (u64)sh.part_hi[2 * lane + 1] << 32 | sh.part_lo[2 * lane + 1];
            const u64 upto = warp_scan(p0 + p1), before = ahead + upto - p0 - p1;
            if (!((double)(ahead + __shfl_sync(0xffffffffu, upto, 31)) >= thr)) return false;
            const bool in0 = p0 && (double)before < thr, in1 = p1 && (double)(before + p0) < thr;
            const int part = __reduce_max_sync(0xffffffffu, in1 ? 2 * lane + 1 : in0 ? 2 * lane : 0);
            const u64 s0 = __shfl_sync(0xffffffffu, part & 1 ? before + p0 : before, part >> 1);
            for (int e = tid; e < m; e += NT) {
                const u64 y = sh.wide[e];
                if (part_of(y) == part) {
                    const int at = atomicAdd(&sh.n_list, 1);
                    if (at < SA_LIST) sh.any[at] = y;
                }
            }
            __syncthreads();
            const int of_part = sh.n_list;
            __syncthreads();                              // all have read it
            if (tid == 0) sh.n_list = 0;
            if (of_part > SA_LIST) return false;
            cut_in_list(of_part, 0, s0, true, thr, false);
            for (int e = lane; e < m; e += 32) {          // what stays of the window, that of this warp's stretch
                const u64 y = sh.wide[e];
                const int i = (int)~(uint32_t)y;
                if (y >= sh.cut && i >= data.first + v0 * N && i < data.first + v1 * N) {
                    const float w = row.w_of(logit_of(y));
                    if (w >= min_p) s += Row::units(w);
                }
            }
            return true;
        };
        // The cut in sh.bin: sh.cut = composite of the last entry that stays, sh.cut_sum = weight of all that stay.  sum: whether to add up the kept weights ahead of the step.
        bool filled = true;                               // whether sh.h is the histogram over steps
        auto locate = [&](bool by_weight, double thr, bool sum) {
            const int bin = sh.bin;
            const u64 c0 = sh.cnt_before, s0 = sh.sum_before;
            // logits of step bin, and a little more on either side
            const float unit = SA_RANGE / SA_BINS / row.inv_t, slack = (fabsf(row.top) + (bin + 1) * unit) * 1e-6f;
            const float high = row.top - (bin - 0.5f) * unit + slack, low = row.top - (bin + 0.5f) * unit - slack;
            const bool usable = low > -INFINITY && high < INFINITY;                     // (not for a temperature near the type's ends)
            uint32_t sum_hi = 0, sum_lo = 0, added = 0;
            if (usable)
                for (int v = v0 + lane; v < v1; v += 32) {
                    if (!(data.most(v) >= low)) continue;
                    u64 l[N / 2];
                    data.pairs(v, l);
                    added += N;
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) {
                        const u64 x = row.x_of2(l[j]);
                        float w[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float le = e ? hi2(l[j]) : lo2(l[j]), xe = e ? hi2(x) : lo2(x);
                            bool ahead = le > high;
                            if (le >= low && !ahead) {    // in the step, or next to it
                                const uint32_t b = Row::bin_of(xe);
                                if (b == (uint32_t)bin) {
                                    const int at = atomicAdd(&sh.n_list, 1);
                                    if (at < SA_LIST) sh.any[at] = composite(le, data.first + v * N + 2 * j + e);
                                }
                                ahead = b < (uint32_t)bin;
                            }
                            w[e] = sum && ahead ? expf(xe) : 0.f;
                            w[e] = w[e] >= min_p ? w[e] : 0.f;
                        }
                        u64 hi, lo;
                        split_units2(pair2(w[0], w[1]), hi, lo);
                        sum_hi += (uint32_t)hi + (uint32_t)(hi >> 32); sum_lo += (uint32_t)lo + (uint32_t)(lo >> 32);
                    }
                }
            s = ((u64)(sum_hi - added * MAGIC) << 20) + (sum_lo - added * MAGIC);
            __syncthreads();
            const int n = gather(usable ? sh.n_list : SA_LIST + 1, SA_LIST, [](auto* o) { return o->any; });
            if (n <= SA_LIST) {
                cut_in_list(n, c0, s0, by_weight, thr, sum);
                return sum;
            }
            // more than the list holds
            filled = false;
            uint32_t lo, hi;
            key_range(row, bin, top_key, lo, hi);
            u64 cb = c0, sb = s0;
            while (true) {
                const int width = 32 - __clz(hi - lo), shift = max(0, width - 10);                    // 2^10 bins
                cta.sync();
                sh.h.template clear<NT>();
                __syncthreads();
                data.each(v0, v1, [&](float l, int) {
                    const uint32_t key = key_of(l);
                    if (key >= lo && key <= hi) {
                        const int b = (int)((hi - key) >> shift);
                        sh.h.add(b, Row::units(row.w_of(l)));
                        atomicAdd(sh.h.cnt + b, 1u);
                    }
                });
                find_bin<NT, C>(sh, cta, by_weight, k, thr, cb, sb);
                const uint32_t h2 = hi - ((uint32_t)sh.bin << shift);
                lo = shift ? max(lo, h2 - ((1u << shift) - 1)) : h2;
                hi = h2;
                cb = sh.cnt_before; sb = sh.sum_before;
                if (shift == 0) break;
            }
            // entries equal to one key, of weight w each: how many stay
            u64 n_eq = 0;
            for (int q = 0; q < C; ++q) n_eq += cta.of(&sh, q)->h.cnt[sh.bin];
            const u64 w = Row::units(row.w_of(of_key(lo)));
            u64 m = n_eq;
            if (!by_weight) m = k - cb;
            else if (w) {                                 // entries j with sb + j w < thr
                const double gap = thr - (double)sb;
                m = gap > 0 ? min((u64)(gap / (double)w) + 2, n_eq) : 0;
                while (m > 0 && !((double)(sb + (m - 1) * w) < thr)) --m;
            }
            // the index of the m-th: counts by CTA, by warp, then 32 entries at a time
            int ne = 0;
            data.each(v0, v1, [&](float l, int) { ne += key_of(l) == lo; });
#pragma unroll
            for (int o = 16; o; o >>= 1) ne += __shfl_xor_sync(0xffffffffu, ne, o);
            __syncthreads();
            if (lane == 0) sh.w_cnt[warp] = ne;
            __syncthreads();
            int cta_n;
            u64 ahead = warps_before<NT>(sh.w_cnt, cta_n);
            if (C > 1) {
                if (tid == 0) { sh.x_n = cta_n; sh.winner = -1; }
                cta.sync();
                for (int q = 0; q < cta.rank; ++q) ahead += cta.of(&sh, q)->x_n;
            }
            if (ahead < m && m <= ahead + ne)
                for (int v = v0 * N; v < v1 * N; v += 32) {
                    const int i = data.first + v + lane;
                    const bool is = v + lane < v1 * N && key_of(data.at(i)) == lo;
                    const unsigned ms = __ballot_sync(0xffffffffu, is);
                    if (m <= ahead + __popc(ms)) {
                        if (is && ahead + __popc(ms & ((2u << lane) - 1)) == m) {
                            for (int q = 0; q < C; ++q) cta.of(&sh, q)->cut = (u64)lo << 32 | (uint32_t)~i;
                        }
                        break;
                    }
                    ahead += __popc(ms);
                }
            if (tid == 0) sh.cut_sum = sb + m * w;
            cta.sync();
            return false;
        };
        bool summed = k == V && by_window();
        if (summed) {
            cut = sh.cut;
        } else {
            if (k == V) {
                cta.sync();
                sh.h.template clear<NT>();
                __syncthreads();
            }
            fill(k < V);
            if (k < V) {
                find_bin<NT, C>(sh, cta, false, k, 0., 0, 0);
                if (sh.bin >= 0) {
                    summed = locate(false, 0., !(top_p < 1.f));
                    cut = sh.cut; total = sh.cut_sum;
                }
            }
            if (top_p < 1.f) {
                if (!filled) {                            // the search for the k-th entry took the histogram
                    cta.sync();
                    sh.h.template clear<NT>();
                    __syncthreads();
                    fill(false);
                }
                double thr = (double)top_p * (double)total;
                find_bin<NT, C>(sh, cta, true, 0, thr, 0, 0, total ? 0.f : top_p);
                if (!total) thr = (double)top_p * (double)sh.total;
                summed = locate(true, thr, true);
                cut = sh.cut;
            }
        }
        if (!summed) {
            s = 0;
            data.each(v0, v1, [&](float l, int i) {
                if (composite(l, i) >= cut) { const float w = row.w_of(l); if (w >= min_p) s += Row::units(w); }
            });
        }
    } else {                                              // all entries, or all that min_p leaves
        uint32_t sum_hi = 0, sum_lo = 0, n = 0;           // with MAGIC in each: at most 2^18 / NT entries of up to 2^20
        for (int v = v0 + lane; v < v1; v += 32, n += N) {
            u64 l[N / 2];
            data.pairs(v, l);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const u64 x = row.x_of2(l[j]);
                const float w0 = expf(lo2(x)), w1 = expf(hi2(x));
                u64 hi, lo;
                split_units2(pair2(w0 >= min_p ? w0 : 0.f, w1 >= min_p ? w1 : 0.f), hi, lo);
                sum_hi += (uint32_t)hi + (uint32_t)(hi >> 32); sum_lo += (uint32_t)lo + (uint32_t)(lo >> 32);
            }
        }
        s = ((u64)(sum_hi - n * MAGIC) << 20) + (sum_lo - n * MAGIC);
    }

    // the warp whose stretch holds the goal
    s = warp_sum(s);
    __syncthreads();
    if (lane == 0) sh.w_sum[warp] = s;
    __syncthreads();
    u64 total;
    u64 before = warps_before<NT>(sh.w_sum, total);
    if (C > 1) {
        if (tid == 0) sh.x_total = total;
        cta.sync();
        u64 all = 0;
        for (int q = 0; q < C; ++q) {
            const u64 t = cta.of(&sh, q)->x_total;
            if (q < cta.rank) before += t;
            all += t;
        }
        total = all;
        cluster_arrive();                                 // (a CTA stays until the others have read its total)
    }
    const u64 goal = goal_of(total);
    if (lane == 0 && before <= goal && goal < before + s) { sh.winner = warp; sh.sum_before = before; }
    __syncthreads();
    if (sh.winner < 0) {                                  // in another CTA
        if (C > 1) cluster_wait();
        return;
    }
    // its stretch again, consecutive entries to a thread (loops as they stand: unrolled, the code of a row's rarer parts pushes the rest out of the instruction cache)
    const int w0 = data.first + min(sh.winner * per_warp, mine_vec) * N, w1 = data.first + min((sh.winner + 1) * per_warp, mine_vec) * N, each = (w1 - w0 + NT - 1) / NT;
    const int t0 = min(w0 + tid * each, w1), t1 = min(t0 + each, w1);
    auto kept = [&](float l, int i) -> u64 {
        if (composite(l, i) < cut) return 0;
        const float w = row.w_of(l);
        return w >= min_p ? Row::units(w) : 0;
    };
    u64 t = 0;
#pragma unroll 1
    for (int i = t0; i < t1; ++i) t += kept(data.at(i), i);
    const u64 start = sh.sum_before, upto = warp_scan(t);
    if (lane == 31) sh.w_sum[warp] = upto;
    __syncthreads();
    u64 unused;
    u64 at = start + warps_before<NT>(sh.w_sum, unused) + upto - t;
    if (at <= goal && goal < at + t)
#pragma unroll 1
        for (int i = t0; i < t1; ++i) {
            const u64 w = kept(data.at(i), i);
            if (at <= goal && goal < at + w) {
                a.token[r] = i;
                if (a.logprob) a.logprob[r] = row.x_of(data.at(i)) - log_of(total);
            }
            at += w;
        }
    if (C > 1) { __syncwarp(); cluster_wait(); }
}

constexpr size_t SA_STATIC = 25 * 1024, SA_SMEM = 232448; // shared memory beside the row, and of an SM at most
template <typename T, int NT, int C>
cudaError_t run(const SampleArgs& a, int rows, size_t smem, cudaStream_t st) {
    static_assert(sizeof(Shared<NT>) <= SA_STATIC, "what is beside the row");
    if (const cudaError_t e = op_allow<k_sample<T, NT, C>>((int)(SA_SMEM - SA_STATIC))) return e;
    return op_launch(k_sample<T, NT, C>, dim3(rows * C), NT, smem, st, C, a);
}
// CTAs of a row: as few as hold it, and more while every CTA has an SM to itself and 8192 entries (26 rows of 32768 fp32, top-p: 1, 2, 4, 8 CTAs 17.8, 16.3, 15.1, 20.3 us).  An SM to
// itself have 74 clusters of 2 CTAs, 33 of 4 and 15 of 8 (SMs come in groups of up to 18 that a cluster does not leave): 33 and 34 rows of 32768 on 4 CTAs 15.4 and 17.9 us, on 2 16.2 and
// 16.3; 15 and 16 rows of 131072 on 8 CTAs 23.0 and 28.6, on 4 25.6 and 25.6; 74 rows of 50265 on 1 and 2 25.6 and 21.8, 96 rows 25.6 and 37.9.  1024 threads where a whole row has an SM to
// itself (74 rows of 50265 25.6, with 512 26.4); else 512, two CTAs to an SM (160 rows of 32768 bf16: 25.0 us, with 1024 31.1; 26 rows on 4 CTAs each 15.1 and 17.3).
template <typename T>
cudaError_t launch(const SampleArgs& a, int rows, cudaStream_t st) {
    auto bytes = [&](int c) { return ((size_t)a.V * sizeof(T) / 16 + 2 + c) / c * 16 + 16; };
    int c = 1;
    while (bytes(c) > SA_SMEM - SA_STATIC) c *= 2;
    while (c < 8 && rows <= (c == 1 ? 74 : c == 2 ? 33 : 15) && a.V >= 2 * c * 8192) c *= 2;
    const size_t smem = bytes(c);
    if ((c > 1 || rows > 148) && 2 * (smem + SA_STATIC + 1024) <= SA_SMEM)
        return c == 1 ? run<T, 512, 1>(a, rows, smem, st) : c == 2 ? run<T, 512, 2>(a, rows, smem, st) : c == 4 ? run<T, 512, 4>(a, rows, smem, st) : run<T, 512, 8>(a, rows, smem, st);
    if constexpr (sizeof(T) == 4)                         // (an eighth of the longest 16-bit row leaves room for two CTAs)
        if (c == 8) return run<T, 1024, 8>(a, rows, smem, st);
    return c == 1 ? run<T, 1024, 1>(a, rows, smem, st) : c == 2 ? run<T, 1024, 2>(a, rows, smem, st) : run<T, 1024, 4>(a, rows, smem, st);
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" int specdec_sample(const void* d_logits, int dtype, long long stride, int rows, int V, const float* d_uniform,
                              const float* d_temperature, const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, int rows_per_param,
                              int32_t* d_token, float* d_logprob, void* stream) {
    if (rows < 0 || V < 1 || rows_per_param < 1) return op_bad("sample", "rows is negative, or V or rows_per_param below 1");
    if (!op_elem_bytes(dtype)) return op_bad("sample", "unknown dtype");
    if (V > 1 << 18) return op_fail(SPECDEC_ERR_CAPACITY, "sample", "at most 262144 entries a row");       // 2^18 weights of up to 2^40 units stay far below 2^64
    if (rows == 0) return SPECDEC_OK;
    if (!d_logits || !d_uniform || !d_token || (uintptr_t)d_logits % op_elem_bytes(dtype)) return op_bad("sample", "a pointer is NULL, or d_logits not aligned to its type");
    if (rows > 1 << 27) return op_fail(SPECDEC_ERR_CAPACITY, "sample", "at most 2^27 rows");
    const SampleArgs a{d_logits, stride, V, d_uniform, d_temperature, d_top_k, d_top_p, d_min_p, rows_per_param, d_token, d_logprob};
    const cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == SPECDEC_DTYPE_F32 ? launch<float>(a, rows, st) : dtype == SPECDEC_DTYPE_BF16 ? launch<__nv_bfloat16>(a, rows, st) : launch<__half>(a, rows, st);
    return op_done("sample", e);
}
