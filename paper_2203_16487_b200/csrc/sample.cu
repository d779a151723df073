// One token per row of logits from a given uniform number: temperature, top-k, top-p, min-p (contract: specdec.h).
//
// Weights are whole numbers of 2^-40 of the largest, so every sum is exact and neither the order of atomics nor the split of the work can
// change a token.  With x = (l - max) / T falling along the order of the logits, an entry's weight is 0 beyond x = -27.73.
//
//   1. maximum of the row and its first index.
//   2. histogram over 2048 equal steps of x: entries and weight in each.  A scan finds the step in which the k-th entry, then the step in which
//      top_p of the weight falls; entries in other steps need no closer look.
//   3. that step's range of logits (as ordered integers) is split into 2048 again until a bin is one value: entries equal to it have equal weights, so
//      how many of them stay is arithmetic; which, is by index.
//   4. the kept weights by 16 stretches of the row, then of the stretch that holds the goal, then entry by entry.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "op_error.cuh"

namespace sd {
namespace {

typedef unsigned long long u64;
constexpr int SA_THREADS = 512, SA_WARPS = SA_THREADS / 32, SA_BINS = 2048;
constexpr float SA_RANGE = 27.75f;                        // e^-27.73 = 2^-40

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

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

struct Row {                                              // what turns a logit into a weight
    float top, inv_t;
    __device__ __forceinline__ float x_of(float l) const { return l == top ? 0.f : (l - top) * inv_t; }
    __device__ __forceinline__ static u64 units(float w) { return (u64)(w * 1099511627776.f); }
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
    __device__ __forceinline__ void clear() { for (int i = threadIdx.x; i < SA_BINS; i += SA_THREADS) { cnt[i] = 0; lo[i] = 0; hi[i] = 0; } }
    __device__ __forceinline__ void add(int b, u64 u) {
        atomicAdd(cnt + b, 1u);
        const uint32_t l = (uint32_t)u, old = atomicAdd(lo + b, l);
        const uint32_t h = (uint32_t)(u >> 32) + (old + l < old);
        if (h) atomicAdd(hi + b, h);
    }
    __device__ __forceinline__ u64 sum(int b) const { return (u64)hi[b] << 32 | lo[b]; }
};

struct Shared {
    Hist h;
    u64 w_sum[SA_WARPS], w_best[SA_WARPS];
    int w_cnt[SA_WARPS];
    // a search's answer
    int bin; u64 cnt_before, sum_before;
    int index;
};

// First bin, in ascending order, behind which the search ends: by entries (the bin that holds entry number `k` from 1) or by weight (the last
// non-empty bin with sum_before + weight ahead < thr).  Entries and weight ahead of it in sh.*_before, added to what was given.  sh.bin = -1: none (k beyond all).
__device__ void find_bin(Shared& sh, bool by_weight, u64 k, double thr, u64 cnt0, u64 sum0) {
    constexpr int PER = SA_BINS / SA_THREADS;
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
        if (n && (by_weight ? (double)bs < thr : (bc < k && k <= bc + n))) { mine = b; mc = bc; ms = bs; }
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

template <typename T>
__global__ void __launch_bounds__(SA_THREADS) k_sample(SampleArgs a) {
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V;
    const int r = blockIdx.x, pr = r / a.per_param;
    const T* logits = (const T*)a.logits + r * a.stride;
    const float temperature = a.temperature ? a.temperature[pr] : 1.f;
    const float top_p = a.top_p ? a.top_p[pr] : 1.f, min_p = a.min_p ? a.min_p[pr] : 0.f;
    const int k_in = a.top_k ? a.top_k[pr] : 0;
    const u64 k = k_in <= 0 || k_in > V ? (u64)V : (u64)k_in;
    const bool greedy = !(temperature > 0.f);

    // 1. maximum and its first index
    u64 best = 0;
    for (int i = tid; i < V; i += SA_THREADS) best = max(best, (u64)key_of(to_f(logits[i])) << 32 | (uint32_t)~i);
#pragma unroll
    for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) sh.w_best[warp] = best;
    sh.h.clear();
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SA_WARPS; ++w) best = max(best, sh.w_best[w]);
    const uint32_t top_key = (uint32_t)(best >> 32);
    const int top_index = (int)~(uint32_t)best;
    if (top_key <= KEY_NEG_INF || greedy) {
        if (tid == 0) {
            const bool any = top_key > KEY_NEG_INF;
            a.token[r] = any ? top_index : -1;
            if (a.logprob) a.logprob[r] = any ? 0.f : -INFINITY;
        }
        return;
    }
    const Row row{of_key(top_key), 1.f / temperature};

    // 2., 3. the key and the number of its entries at which the order is cut
    uint32_t cut_key = KEY_NEG_INF + 1;                   // entries above stay; of those equal to it the first cut_n
    u64 cut_n = ~0ull;
    if (k < (u64)V || top_p < 1.f) {
        u64 all = 0;
        for (int i = tid; i < V; i += SA_THREADS) {
            const float x = row.x_of(to_f(logits[i]));
            const int b = Row::bin_of(x);
            if (b < SA_BINS) { const u64 u = Row::units(expf(x)); sh.h.add(b, u); all += u; }
        }
        all = warp_sum(all);
        if (lane == 0) sh.w_best[warp] = all;
        __syncthreads();
        u64 total = 0;
#pragma unroll
        for (int w = 0; w < SA_WARPS; ++w) total += sh.w_best[w];
        bool first_level = true;                          // whether sh.h is the histogram of x
        auto refine = [&](bool by_weight, double thr) {
            // sh.bin, sh.*_before: the step.  Afterwards cut_key, cut_n, and sh.sum_before = the weight ahead of the key's first entry
            uint32_t lo, hi;
            key_range(row, sh.bin, top_key, lo, hi);
            while (true) {
                const u64 c0 = sh.cnt_before, s0 = sh.sum_before;
                const int width = 32 - __clz(hi - lo), shift = max(0, width - 11);
                __syncthreads();
                sh.h.clear();
                __syncthreads();
                first_level = false;
                for (int i = tid; i < V; i += SA_THREADS) {
                    const float l = to_f(logits[i]);
                    const uint32_t key = key_of(l);
                    if (key >= lo && key <= hi) sh.h.add((int)((hi - key) >> shift), Row::units(expf(row.x_of(l))));
                }
                __syncthreads();
                find_bin(sh, by_weight, k, thr, c0, s0);
                const uint32_t h2 = hi - ((uint32_t)sh.bin << shift);
                lo = shift ? max(lo, h2 - ((1u << shift) - 1)) : h2;
                hi = h2;
                if (shift == 0) break;
            }
            cut_key = lo;
            const u64 n = sh.h.cnt[sh.bin], u = sh.h.sum(sh.bin) / n;      // n entries of weight u each
            if (!by_weight) { cut_n = k - sh.cnt_before; return; }
            u64 m = n;                                    // entries j < n with sum_before + j u < thr
            if (u) {
                const double gap = thr - (double)sh.sum_before;
                m = gap > 0 ? min((u64)(gap / (double)u) + 2, n) : 0;
                while (m > 0 && !((double)(sh.sum_before + (m - 1) * u) < thr)) --m;
            }
            cut_n = m;
        };
        if (k < (u64)V) {
            find_bin(sh, false, k, 0., 0, 0);
            if (sh.bin >= 0) {
                refine(false, 0.);
                const u64 u = sh.h.sum(sh.bin) / sh.h.cnt[sh.bin];
                total = sh.sum_before + cut_n * u;
            }
        }
        if (top_p < 1.f) {
            const double thr = (double)top_p * (double)total;
            if (!first_level) {                           // the search for the k-th entry took the histogram
                __syncthreads();
                sh.h.clear();
                __syncthreads();
                for (int i = tid; i < V; i += SA_THREADS) {
                    const float x = row.x_of(to_f(logits[i]));
                    const int b = Row::bin_of(x);
                    if (b < SA_BINS) sh.h.add(b, Row::units(expf(x)));
                }
                __syncthreads();
            }
            find_bin(sh, true, 0, thr, 0, 0);
            if (sh.bin >= 0) refine(true, thr);
            else { cut_key = top_key; cut_n = 1; }        // top_p <= 0 or NaN: the largest entry alone
        }
        if (cut_n == 0) { cut_key = top_key; cut_n = 1; }
    }
    // of the entries equal to cut_key, the index of the last that stays
    int cut_index = V;
    const int seg = ((V + SA_WARPS - 1) / SA_WARPS + 31) / 32 * 32;
    if (cut_n != ~0ull) {
        int n = 0;
        for (int i = warp * seg + lane; i < min((warp + 1) * seg, V); i += 32) n += key_of(to_f(logits[i])) == cut_key;
#pragma unroll
        for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        __syncthreads();
        if (lane == 0) sh.w_cnt[warp] = n;
        if (tid == 0) sh.index = V;
        __syncthreads();
        u64 ahead = 0;
        for (int w = 0; w < warp; ++w) ahead += sh.w_cnt[w];
        if (ahead < cut_n && cut_n <= ahead + n)
            for (int i0 = warp * seg; i0 < min((warp + 1) * seg, V); i0 += 32) {
                const unsigned m = __ballot_sync(0xffffffffu, i0 + lane < V && key_of(to_f(logits[min(i0 + lane, V - 1)])) == cut_key);
                if (cut_n <= ahead + __popc(m)) {
                    if ((m >> lane & 1) && ahead + __popc(m & ((2u << lane) - 1)) == cut_n) sh.index = i0 + lane;
                    break;
                }
                ahead += __popc(m);
            }
        __syncthreads();
        cut_index = sh.index;
    }
    // 4. the goal's entry
    auto kept = [&](int i) -> u64 {
        const float l = to_f(logits[i]);
        const uint32_t key = key_of(l);
        if (key < cut_key || (key == cut_key && i > cut_index)) return 0;
        const float w = expf(row.x_of(l));
        return w >= min_p || i == top_index ? Row::units(w) : 0;
    };
    int lo = 0, hi = V;
    u64 goal = 0, ahead = 0, total = 0;
    float log_total = 0.f;
    for (int len = seg; ; len = ((hi - lo + SA_WARPS - 1) / SA_WARPS + 31) / 32 * 32) {
        u64 s = 0;
        const int a0 = lo + warp * len, a1 = min(a0 + len, hi);
        for (int i = a0 + lane; i < a1; i += 32) s += kept(i);
        s = warp_sum(s);
        __syncthreads();
        if (lane == 0) sh.w_sum[warp] = s;
        __syncthreads();
        if (len == seg && lo == 0 && hi == V) {
#pragma unroll
            for (int w = 0; w < SA_WARPS; ++w) total += sh.w_sum[w];
            const float u = a.uniform[r];
            goal = u > 0.f ? min((u64)((double)u * (double)total), total - 1) : 0;
            log_total = logf((float)total * 9.094947017729282e-13f);       // 2^-40
        }
        int w = 0;
        for (; w < SA_WARPS - 1 && ahead + sh.w_sum[w] <= goal; ++w) ahead += sh.w_sum[w];
        lo += w * len; hi = min(lo + len, hi);
        if (len == 32) break;
    }
    if (warp == 0) {                                      // 32 entries are left
        const int i = lo + lane;
        const u64 s = ahead + warp_scan(i < hi ? kept(i) : 0);
        const unsigned m = __ballot_sync(0xffffffffu, s > goal);
        const int token = lo + __ffs(m) - 1;
        if (lane == 0) {
            a.token[r] = token;
            if (a.logprob) a.logprob[r] = row.x_of(to_f(logits[token])) - log_total;
        }
    }
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
    if (!d_logits || !d_uniform || !d_token) return op_bad("sample", "a pointer is NULL");
    const SampleArgs a{d_logits, stride, V, d_uniform, d_temperature, d_top_k, d_top_p, d_min_p, rows_per_param, d_token, d_logprob};
    const cudaStream_t st = (cudaStream_t)stream;
    if (dtype == SPECDEC_DTYPE_F32) k_sample<float><<<rows, SA_THREADS, 0, st>>>(a);
    else if (dtype == SPECDEC_DTYPE_BF16) k_sample<__nv_bfloat16><<<rows, SA_THREADS, 0, st>>>(a);
    else k_sample<__half><<<rows, SA_THREADS, 0, st>>>(a);
    return op_launched("sample");
}
