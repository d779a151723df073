// One token per row of logits from a given uniform number: temperature, top-k, top-p, min-p (contract: specdec.h).
//
// Weights are whole numbers of 2^-40 of the largest, so every sum is exact and neither the order of atomics nor the split of the work can
// change a token.  With x = (l - max) / T falling along the order of the logits, an entry's weight is 0 beyond x = -27.73.
//
// One CTA a row, which it reads from memory once: the row stays in shared memory, rows beyond that are read again (from L2).  What a row goes through depends on
// its parameters:
//   greedy  the first index of the maximum.
//   few     top-k of at most SA_FEW.  The k-th largest of the threads' own maxima is a bound below the k-th largest entry, so only the entries above it are
//           looked at again: a list of some k to 3k, ranked by counting, cut, and walked in index order.  No exponential of the others is taken.
//   order   other cuts: a histogram over 2048 equal steps of x gives the step in which the cut falls; that step's range of logits (as ordered integers) is split
//           into 2048 again until a bin is one value: entries equal to it have equal weights, so how many of them stay is arithmetic; which, is by index.
//   then    the kept weights by stretches of the row, one a warp, then of the stretch that holds the goal, then entry by entry.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "barriers.cuh"
#include "op_error.cuh"

namespace sd {
namespace {

typedef unsigned long long u64;
constexpr int SA_BINS = 2048, SA_FEW = 128, SA_LIST = 1024;
constexpr float SA_RANGE = 27.75f;                        // e^-27.73 = 2^-40

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T lowest();                              // -inf
template <> __device__ __forceinline__ float lowest<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __nv_bfloat16 lowest<__nv_bfloat16>() { return __float2bfloat16_rn(-INFINITY); }
template <> __device__ __forceinline__ __half lowest<__half>() { return __float2half_rn(-INFINITY); }

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
struct Row {                                              // what turns a logit into a weight
    float top, inv_t;
    __device__ __forceinline__ float x_of(float l) const { return l == top ? 0.f : (l - top) * inv_t; }
    __device__ __forceinline__ float w_of(float l) const { return fmaxf(expf(x_of(l)), 0.f); }          // NaN: 0
    __device__ __forceinline__ static u64 units(float w) {
        uint32_t hi, lo;
        split_units(w, hi, lo);
        return ((u64)(hi - MAGIC) << 20) + (lo - MAGIC);
    }
    // step of x: 0 for the largest; SA_BINS: weight 0 (NaN, -inf and all that is too small)
    __device__ __forceinline__ static int bin_of(float x) {
        return x > -SA_RANGE ? min((int)(-x * (SA_BINS / SA_RANGE)), SA_BINS - 1) : SA_BINS;
    }
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
    uint32_t cnt[SA_BINS], lo[SA_BINS], hi[SA_BINS];      // entries; weight as two words
    template <int NT> __device__ __forceinline__ void clear() { for (int i = threadIdx.x; i < SA_BINS; i += NT) { cnt[i] = 0; lo[i] = 0; hi[i] = 0; } }
    __device__ __forceinline__ void add(int b, u64 u) {   // (most weights are below 2^32 units: one addition)
        const uint32_t l = (uint32_t)u, old = atomicAdd(lo + b, l);
        const uint32_t h = (uint32_t)(u >> 32) + (old + l < old);
        if (h) atomicAdd(hi + b, h);
    }
    __device__ __forceinline__ u64 sum(int b) const { return (u64)hi[b] << 32 | lo[b]; }
};
struct List {                                             // the entries that may be among the k largest
    u64 any[SA_LIST], sorted[SA_FEW], units[SA_FEW], part[8][SA_FEW];
    int rank[SA_LIST];
};

template <int NT> struct Shared {
    union { Hist h; List list; };
    u64 w_sum[NT / 32];
    int w_cnt[NT / 32];
    float w_max[NT / 32];
    // a search's answer
    int bin; u64 cnt_before, sum_before;
    int index, n_list, n_kept;
    u64 total;
};

// First bin, in ascending order, behind which the search ends: by entries (the bin that holds entry number `k` from 1) or by weight (the last bin of any
// weight with sum_before + weight ahead < thr).  Entries and weight ahead of it in sh.*_before, added to what was given.  sh.bin = -1: none (k beyond all).
template <int NT>
__device__ void find_bin(Shared<NT>& sh, bool by_weight, u64 k, double thr, u64 cnt0, u64 sum0) {
    constexpr int PER = SA_BINS / NT;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 c = 0, s = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) { c += sh.h.cnt[threadIdx.x * PER + j]; s += sh.h.sum(threadIdx.x * PER + j); }
    u64 ic = warp_scan(c), is = warp_scan(s);
    if (lane == 31) { sh.w_cnt[warp] = (int)ic; sh.w_sum[warp] = is; }
    if (threadIdx.x == 0) sh.bin = -1;
    __syncthreads();
    u64 bc = cnt0 + ic - c, bs = sum0 + is - s;
    for (int w = 0; w < warp; ++w) { bc += sh.w_cnt[w]; bs += sh.w_sum[w]; }
    int mine = -1;
    u64 mc = 0, ms = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int b = threadIdx.x * PER + j;
        const u64 n = sh.h.cnt[b], w = sh.h.sum(b);
        if (by_weight ? w && (double)bs < thr : (bc < k && k <= bc + n)) { mine = b; mc = bc; ms = bs; }
        bc += n; bs += w;
    }
    if (mine >= 0) atomicMax(&sh.bin, mine);
    __syncthreads();
    if (mine >= 0 && sh.bin == mine) { sh.cnt_before = mc; sh.sum_before = ms; }
    __syncthreads();
}

// Keys whose step is b: [lo, hi].  The step falls as the key grows, so both ends are found by a search of 32 probes at a time.
__device__ void key_range(const Row& row, int b, uint32_t top_key, uint32_t& lo, uint32_t& hi) {
    const int lane = threadIdx.x & 31;
    auto first_with = [&](int most) {                     // smallest key in (KEY_NEG_INF, top_key] whose step is <= most
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

// A row as 16-byte vectors of N entries, the first of which may begin ahead of the row: in shared memory (what is ahead and behind is -inf) or, if it does not fit,
// in global memory.  Warp w owns a stretch of vectors; f(value, index) of one warp's share, lane by lane.
template <typename T> struct RowData {
    static constexpr int N = 16 / sizeof(T);
    const T* smem;                                        // vector 0, or null
    const T* global;                                      // entry 0
    int lead, V, nvec;                                    // entries of vector 0 that lie ahead of the row
    __device__ __forceinline__ float at(int i) const { return to_f(smem ? smem[lead + i] : global[i]); }
    template <typename F> __device__ __forceinline__ void each(int v0, int v1, F f) const {       // vectors [v0, v1), by one warp
        for (int v = v0 + (threadIdx.x & 31); v < v1; v += 32) {
            const int i0 = v * N - lead;
            if (smem) {
                union { int4 raw; T x[N]; } u;
                u.raw = reinterpret_cast<const int4*>(smem)[v];
#pragma unroll
                for (int j = 0; j < N; ++j) f(to_f(u.x[j]), i0 + j);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) if (i0 + j >= 0 && i0 + j < V) f(to_f(global[i0 + j]), i0 + j);
            }
        }
    }
};

template <typename T, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_sample(SampleArgs a, int resident) {
    constexpr int NW = NT / 32, N = RowData<T>::N;
    extern __shared__ __align__(16) char row_smem[];
    __shared__ Shared<NT> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V;
    const int r = blockIdx.x, pr = r / a.per_param;
    RowData<T> data;
    data.global = (const T*)a.logits + r * a.stride;
    data.lead = (int)((uintptr_t)data.global & 15) / (int)sizeof(T);
    data.V = V; data.nvec = (data.lead + V + N - 1) / N;
    data.smem = resident ? (const T*)row_smem : nullptr;
    const int per_warp = (data.nvec + NW - 1) / NW, v0 = min(warp * per_warp, data.nvec), v1 = min(v0 + per_warp, data.nvec);
    if (resident) {                                       // each thread fetches the vectors that it reads first
        const int4* from = reinterpret_cast<const int4*>(data.global - data.lead);
        for (int v = v0 + lane; v < v1; v += 32) {
            const int i0 = v * N - data.lead;
            if (i0 >= 0 && i0 + N <= V) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(row_smem + v * 16)), "l"(from + v) : "memory");
            } else {
                union { int4 raw; T x[N]; } u;
#pragma unroll
                for (int j = 0; j < N; ++j) u.x[j] = i0 + j >= 0 && i0 + j < V ? data.global[i0 + j] : lowest<T>();
                reinterpret_cast<int4*>(row_smem)[v] = u.raw;
            }
        }
    }
    const float temperature = a.temperature ? a.temperature[pr] : 1.f;
    const float top_p = a.top_p ? a.top_p[pr] : 1.f, min_p = a.min_p ? a.min_p[pr] : 0.f;
    const int k_in = a.top_k ? a.top_k[pr] : 0;
    const int k = k_in <= 0 || k_in > V ? V : k_in;
    const bool greedy = !(temperature > 0.f) || !(top_p > 0.f) || !(min_p <= 1.f) || k == 1;        // the largest entry alone
    const bool few = k <= SA_FEW && k < V;
    sh.h.template clear<NT>();
    if (tid == 0) { sh.index = V; sh.n_list = 0; }
    asm volatile("cp.async.wait_all;" ::: "memory");

    float mine = -INFINITY;                               // this thread's maximum (NaN does not count)
    data.each(v0, v1, [&](float l, int) { mine = fmaxf(mine, l); });
    float top = mine;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) sh.w_max[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sh.w_max[w]);
    if (top == -INFINITY) {
        if (tid == 0) { a.token[r] = -1; if (a.logprob) a.logprob[r] = -INFINITY; }
        return;
    }
    if (greedy) {
        if (mine == top) {
            int first = V;
            data.each(v0, v1, [&](float l, int i) { if (l == top) first = min(first, i); });
            atomicMin(&sh.index, first);
        }
        __syncthreads();
        if (tid == 0) { a.token[r] = sh.index; if (a.logprob) a.logprob[r] = 0.f; }
        return;
    }
    const Row row{top + 0.f, 1.f / temperature};
    const uint32_t top_key = key_of(top);
    const float u = a.uniform[r];
    auto goal_of = [&](u64 total) -> u64 { return u > 0.f ? min((u64)((double)u * (double)total), total - 1) : 0; };
    auto log_of = [](u64 total) { return logf((float)total * 9.094947017729282e-13f); };             // total 2^-40

    if (few) {
        const int b = Row::bin_of(row.x_of(mine));
        if (b < SA_BINS) atomicAdd(sh.h.cnt + b, 1u);
        __syncthreads();
        find_bin<NT>(sh, false, k, 0., 0, 0);
        const int bin = sh.bin;
        // entries from here on up: all of steps 0 .. bin (a little more does no harm)
        const float depth = (bin + 1) * (SA_RANGE / SA_BINS) * temperature;
        const float bound = bin < 0 ? -INFINITY : row.top - depth - (fabsf(row.top) + depth) * 1e-6f;
        if (bin >= 0 && bound > -INFINITY) {
            __syncthreads();                              // the list takes the histogram's place
            if (mine >= bound)
                data.each(v0, v1, [&](float l, int i) {
                    if (l >= bound) {
                        const int at = atomicAdd(&sh.n_list, 1);
                        if (at < SA_LIST) sh.list.any[at] = (u64)key_of(l) << 32 | (uint32_t)~i;
                    }
                });
            __syncthreads();
        }
        const int n = sh.n_list;
        if (n >= k && n <= SA_LIST) {
            const int width = n <= 128 ? 128 : n <= 256 ? 256 : n <= 512 ? 512 : 1024, parts = max(NT / width, 1);   // entry, share of the others
            for (int i = tid; i < n; i += NT) sh.list.rank[i] = 0;
            __syncthreads();
            for (int e = tid % width; e < n; e += NT) {
                const u64 x = sh.list.any[e];
                int c = 0;
                for (int j = tid / width; j < n; j += parts) c += sh.list.any[j] > x;
                if (c) atomicAdd(sh.list.rank + e, c);
            }
            __syncthreads();
            for (int e = tid; e < n; e += NT) { const int at = sh.list.rank[e]; if (at < k) sh.list.sorted[at] = sh.list.any[e]; }
            __syncthreads();
            if (warp == 0) {                              // the order's cut, and the smaller entries that min_p drops: at most SA_FEW, four a lane
                u64 un[SA_FEW / 32], all = 0;
                float w[SA_FEW / 32];
#pragma unroll
                for (int j = 0; j < SA_FEW / 32; ++j) {
                    const int e = lane * (SA_FEW / 32) + j;
                    w[j] = e < k ? row.w_of(of_key((uint32_t)(sh.list.sorted[e] >> 32))) : 0.f;
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
                    sh.list.units[lane * (SA_FEW / 32) + j] = un[j];
                }
                kept = warp_sum(kept);
                if (lane == 0) sh.total = kept;
            }
            __syncthreads();
            {   // weight of the kept entries with a lower index, eight or four threads an entry
                constexpr int PARTS = NT / SA_FEW;
                const int e = tid % SA_FEW, p = tid / SA_FEW;
                if (e < k) {
                    const uint32_t me = (uint32_t)sh.list.sorted[e];                   // ~index
                    u64 s = 0;
                    for (int j = p; j < k; j += PARTS) if ((uint32_t)sh.list.sorted[j] > me) s += sh.list.units[j];
                    sh.list.part[p][e] = s;
                }
                __syncthreads();
                if (tid < k) {
                    u64 before = 0;
#pragma unroll
                    for (int j = 0; j < PARTS; ++j) before += sh.list.part[j][tid];
                    const u64 total = sh.total, goal = goal_of(total);
                    if (before <= goal && goal < before + sh.list.units[tid]) {
                        const u64 x = sh.list.sorted[tid];
                        a.token[r] = (int)~(uint32_t)x;
                        if (a.logprob) a.logprob[r] = row.x_of(of_key((uint32_t)(x >> 32))) - log_of(total);
                    }
                }
            }
            return;
        }
        __syncthreads();
        sh.h.template clear<NT>();
    }

    // the key and the number of its entries at which the order is cut
    uint32_t cut_key = KEY_NEG_INF + 1;                   // entries above stay; of those equal to it the first cut_n
    u64 cut_n = ~0ull;
    if (k < V || top_p < 1.f) {
        const bool count = k < V;
        u64 all = 0;
        __syncthreads();
        auto fill = [&](bool count) {
            data.each(v0, v1, [&](float l, int) {
                const float x = row.x_of(l);
                const int b = Row::bin_of(x);
                if (b < SA_BINS) {
                    const u64 u = Row::units(expf(x));
                    sh.h.add(b, u);
                    if (count) atomicAdd(sh.h.cnt + b, 1u);
                    all += u;
                }
            });
            __syncthreads();
        };
        fill(count);
        all = warp_sum(all);
        if (lane == 0) sh.w_sum[warp] = all;
        __syncthreads();
        u64 total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) total += sh.w_sum[w];
        __syncthreads();
        bool first_level = true;                          // whether sh.h is the histogram of x
        auto refine = [&](bool by_weight, double thr) {
            // sh.bin, sh.*_before: the step.  Afterwards cut_key, cut_n, and sh.sum_before = the weight ahead of the key's first entry
            uint32_t lo, hi;
            key_range(row, sh.bin, top_key, lo, hi);
            while (true) {
                const u64 c0 = sh.cnt_before, s0 = sh.sum_before;
                const int width = 32 - __clz(hi - lo), shift = max(0, width - 11);
                __syncthreads();
                sh.h.template clear<NT>();
                __syncthreads();
                first_level = false;
                data.each(v0, v1, [&](float l, int) {
                    const uint32_t key = key_of(l);
                    if (key >= lo && key <= hi) {
                        const int b = (int)((hi - key) >> shift);
                        sh.h.add(b, Row::units(row.w_of(l)));
                        atomicAdd(sh.h.cnt + b, 1u);
                    }
                });
                __syncthreads();
                find_bin<NT>(sh, by_weight, k, thr, c0, s0);
                const uint32_t h2 = hi - ((uint32_t)sh.bin << shift);
                lo = shift ? max(lo, h2 - ((1u << shift) - 1)) : h2;
                hi = h2;
                if (shift == 0) break;
            }
            cut_key = lo;
            const u64 n = sh.h.cnt[sh.bin], w = sh.h.sum(sh.bin) / n;      // n entries of weight w each
            if (!by_weight) { cut_n = k - sh.cnt_before; if (cut_n == n && !(top_p < 1.f)) cut_n = ~0ull; return; }
            u64 m = n;                                    // entries j < n with sum_before + j w < thr
            if (w) {
                const double gap = thr - (double)sh.sum_before;
                m = gap > 0 ? min((u64)(gap / (double)w) + 2, n) : 0;
                while (m > 0 && !((double)(sh.sum_before + (m - 1) * w) < thr)) --m;
            }
            cut_n = m == n ? ~0ull : m;
        };
        if (count) {
            find_bin<NT>(sh, false, k, 0., 0, 0);
            if (sh.bin >= 0) {
                refine(false, 0.);
                const u64 w = sh.h.sum(sh.bin) / sh.h.cnt[sh.bin];
                total = sh.sum_before + (k - sh.cnt_before) * w;
            }
        }
        if (top_p < 1.f) {
            const double thr = (double)top_p * (double)total;
            if (!first_level) {                           // the search for the k-th entry took the histogram
                __syncthreads();
                sh.h.template clear<NT>();
                __syncthreads();
                fill(false);
            }
            find_bin<NT>(sh, true, 0, thr, 0, 0);
            refine(true, thr);
        }
    }
    // of the entries equal to cut_key, the index of the last that stays
    int cut_index = V;
    if (cut_n != ~0ull) {
        int n = 0;
        data.each(v0, v1, [&](float l, int) { n += key_of(l) == cut_key; });
#pragma unroll
        for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        __syncthreads();
        if (lane == 0) sh.w_cnt[warp] = n;
        __syncthreads();
        u64 ahead = 0;
        for (int w = 0; w < warp; ++w) ahead += sh.w_cnt[w];
        if (ahead < cut_n && cut_n <= ahead + n)
            for (int i0 = max(v0 * N - data.lead, 0); i0 < V; i0 += 32) {
                const unsigned m = __ballot_sync(0xffffffffu, i0 + lane < V && key_of(data.at(min(i0 + lane, V - 1))) == cut_key);
                if (cut_n <= ahead + __popc(m)) {
                    if ((m >> lane & 1) && ahead + __popc(m & ((2u << lane) - 1)) == cut_n) sh.index = i0 + lane;
                    break;
                }
                ahead += __popc(m);
            }
        __syncthreads();
        cut_index = sh.index;
    }
    // the goal's entry
    auto kept = [&](float l, int i) -> float {            // weight, or 0
        const uint32_t key = key_of(l);
        if (key < cut_key || (key == cut_key && i > cut_index)) return 0.f;
        const float w = row.w_of(l);
        return w >= min_p ? w : 0.f;
    };
    int lo = 0, hi = data.nvec;                           // vectors
    u64 goal = 0, ahead = 0, total = 0;
    for (int len = per_warp, first = 1; ; len = (hi - lo + NW - 1) / NW, first = 0) {
        uint32_t sum_hi = 0, sum_lo = 0, n = 0;           // as split_units gives them: at most 2^18 / NT entries of up to 2^20 each a thread
        const int a0 = min(lo + warp * len, hi), a1 = min(a0 + len, hi);
        data.each(a0, a1, [&](float l, int i) {
            uint32_t x, y;
            split_units(kept(l, i), x, y);
            sum_hi += x; sum_lo += y; ++n;
        });
        const u64 s = warp_sum(((u64)(sum_hi - n * MAGIC) << 20) + (sum_lo - n * MAGIC));
        __syncthreads();
        if (lane == 0) sh.w_sum[warp] = s;
        __syncthreads();
        if (first) {
#pragma unroll
            for (int w = 0; w < NW; ++w) total += sh.w_sum[w];
            goal = goal_of(total);
        }
        int w = 0;
        for (; w < NW - 1 && ahead + sh.w_sum[w] <= goal; ++w) ahead += sh.w_sum[w];
        lo = min(lo + w * len, hi); hi = min(lo + len, hi);
        if (len <= 32 / N) break;
    }
    if (warp == 0) {                                      // at most 32 entries are left
        const int i = lo * N - data.lead + lane;
        const bool in = i >= 0 && i < V && i < hi * N - data.lead;
        const float l = in ? data.at(i) : 0.f;
        const u64 s = ahead + warp_scan(in ? Row::units(kept(l, i)) : 0);
        const unsigned m = __ballot_sync(0xffffffffu, s > goal);
        if (lane == __ffs(m) - 1) {
            a.token[r] = i;
            if (a.logprob) a.logprob[r] = row.x_of(l) - log_of(total);
        }
    }
}

template <typename T, int NT>
cudaError_t run(const SampleArgs& a, int rows, int resident, size_t smem, cudaStream_t st) {
    static const cudaError_t attr = cudaFuncSetAttribute(k_sample<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448 - 28 * 1024);
    if (attr != cudaSuccess) return attr;
    k_sample<T, NT><<<rows, NT, smem, st>>>(a, resident);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch(const SampleArgs& a, int rows, cudaStream_t st) {
    size_t smem = ((size_t)a.V * sizeof(T) + 47) / 16 * 16;
    const int resident = smem <= 232448 - 28 * 1024;
    if (!resident) smem = 0;
    // two CTAs of 512 threads share an SM while two rows fit its shared memory; beyond, one CTA has the SM to itself
    return smem <= 84 * 1024 ? run<T, 512>(a, rows, resident, smem, st) : run<T, 1024>(a, rows, resident, smem, st);
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
    const SampleArgs a{d_logits, stride, V, d_uniform, d_temperature, d_top_k, d_top_p, d_min_p, rows_per_param, d_token, d_logprob};
    const cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == SPECDEC_DTYPE_F32 ? launch<float>(a, rows, st) : dtype == SPECDEC_DTYPE_BF16 ? launch<__nv_bfloat16>(a, rows, st) : launch<__half>(a, rows, st);
    return e == cudaSuccess ? SPECDEC_OK : op_fail(SPECDEC_ERR_CUDA, "sample", cudaGetErrorString(e));
}
