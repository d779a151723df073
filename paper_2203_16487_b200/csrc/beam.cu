// Beam search's selection: the n best continuations of a sentence's beams over the whole vocabulary (contract: specdec.h).
//
// k_beam_rows: a CTA takes a stretch of a row into registers, with every load under way at once, and leaves its maximum m, its sum of e^(l - m) and its n largest entries.
// k_beam_join: a CTA a sentence joins the stretches' sums, ranks the entries that are left (a few hundred) and writes the best n.  The logits are read once; no log-probability but those of the
// entries that are left is ever taken.  What bounds k_beam_rows is instructions (an exponential, a comparison and their share of loads for each logit): 128 sentences of 8 x 32768 in bf16 (67 MB)
// 19 us, issue 54 %, and 6.5 for the join.
//
// The n largest: the q-th largest of a warp's lanes' maxima, q = n / 8 rounded up, has q entries of the warp at or above it, so the least of the eight warps' is a bound below the n-th largest entry of
// the stretch.  What lies above it (some 2 n entries) is listed and ranked by counting.  Where ties make more of it than the list holds, the largest entry below the last one is looked for n times.
//
// Sums are fp32, off by some 2^-22, by less than 2^-19 in any case; scores and ranks are 64 bits from there on.  Of two entries of different beams, one of which is among the best n, either the order is certain, as
// their ranks lie more than twice that (times norm) apart, or the sums of both beams are taken again in 64 bits: the choice is that of exact sums.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "barriers.cuh"
#include "op_error.cuh"

namespace sd {
namespace {

typedef unsigned long long u64;
constexpr int BM_NT = 256, BM_MOST = 64, BM_LIST = 512;   // threads of a stretch; beams and results at most; listed entries of a stretch
constexpr int BJ_NT = 512, BJ_STAGE = 2048, BJ_LIST = 512;            // threads of a sentence; entries that it keeps in shared memory; that it ranks
constexpr int BO_CLUSTER = 8, BO_NV = 8, BO_ITEMS = 2;    // sentences in one launch: CTAs of one, vectors of a thread, stretches of a CTA at most
constexpr float LOG2E = 1.4426950408889634f;
constexpr double NEAR = 1.0 / (1 << 19);

// Order-preserving integer of a logit: NaN and -inf at most NOTHING, the two zeros equal.
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);
    return l != l ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
constexpr uint32_t NOTHING = 0x007fffffu;                 // -inf
__device__ __forceinline__ u64 entry(float l, int index) { return (u64)key_of(l) << 32 | ~(uint32_t)index; }      // larger: ahead in the order

struct BeamArgs {
    const void* logits; long long s_row; int V;           // elements between rows
    const float* scores; const unsigned char* finished; const float* norm;
    int end_token, B, K, n, stretches, span;             // vectors of a stretch
    float* out_scores; int* out_parent; int* out_token;
    float2* sums; u64* lists;                             // [row, stretch]: (maximum, sum); [row, stretch, n], best first, 0 where there are fewer
    __device__ __forceinline__ bool alive(int row) const { return scores[row] > -INFINITY && !(finished && finished[row]); }       // (NaN: dead)
};

template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    // The largest element (NaN: passed over), of 16-bit types two at a time.
    static __device__ __forceinline__ float max_of(const uint4& v) {
        if constexpr (sizeof(T) == 4) return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            auto h = [](const uint32_t& w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
            const float2 f = __bfloat1622float2(__hmax2(__hmax2(h(v.x), h(v.y)), __hmax2(h(v.z), h(v.w))));
            return fmaxf(f.x, f.y);
        } else {
            auto h = [](const uint32_t& w) { return *reinterpret_cast<const __half2*>(&w); };
            const float2 f = __half22float2(__hmax2(__hmax2(h(v.x), h(v.y)), __hmax2(h(v.z), h(v.w))));
            return fmaxf(f.x, f.y);
        }
    }
    static __device__ __forceinline__ float at(const uint4& v, int i) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else { const __half2 h = *reinterpret_cast<const __half2*>(w + i / 2); return i & 1 ? __high2float(h) : __low2float(h); }
    }
    static __device__ __forceinline__ float pick(const uint4& v, int i) {                // ... of an index that is not known before
        const int q = sizeof(T) == 4 ? i : i >> 1;
        const uint32_t w = q & 2 ? (q & 1 ? v.w : v.z) : q & 1 ? v.y : v.x;
        if constexpr (sizeof(T) == 4) return __uint_as_float(w);
        const uint32_t h = i & 1 ? w >> 16 : w & 0xffffu;
        if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(h << 16);
        else return __half2float(__ushort_as_half((unsigned short)h));
    }
};
template <typename T> __device__ __forceinline__ float as_float(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __bfloat162float(x);
    else return __half2float(x);
}
__device__ __forceinline__ float exp2_of(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ u64 pair2(float lo, float hi) { u64 d; asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi)); return d; }
__device__ __forceinline__ float lo2(u64 d) { return __uint_as_float((uint32_t)d); }
__device__ __forceinline__ float hi2(u64 d) { return __uint_as_float((uint32_t)(d >> 32)); }
__device__ __forceinline__ u64 add2(u64 a, u64 b) { u64 d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) { u64 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
// A term of a stretch's sum: e^(l - m) with c = m log2 e rounded, and what that rounding has put into every term.
__device__ __forceinline__ float term(float l, float c) { return exp2_of(fmaf(l, LOG2E, -c)); }
__device__ __forceinline__ float remainder_of(float m) { return exp2f(-fmaf(m, LOG2E, -(m * LOG2E))); }
__device__ __forceinline__ u64 warp_max(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) { const u64 u = __shfl_xor_sync(0xffffffffu, v, o); if (u > v) v = u; }
    return v;
}

// A stretch of a row by a CTA of NT threads, NV vectors each.
template <typename T, int NV, int NT>
__device__ __forceinline__ void stretch_of_row(const BeamArgs& a, int row, int stretch) {
    constexpr int VE = Vec<T>::N, BM_NT = NT, BM_WARPS = NT / 32;
    __shared__ float w_max[BM_WARPS], w_sum[BM_WARPS];
    __shared__ uint32_t w_bound[BM_WARPS];
    __shared__ u64 list[BM_LIST], w_best[BM_WARPS];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long at = (long long)row * a.stretches + stretch;
    if (!a.alive(row)) return;
    const T* p = (const T*)a.logits + row * a.s_row;
    const int lead = (int)(((uintptr_t)p & 15) / sizeof(T));          // elements of the first vector that lie ahead of the row
    const int first = stretch * a.span;
    auto place = [&](int j, int i) { return (first + j * BM_NT + tid) * VE - lead + i; };
    // Vectors of the stretch, by number from the row's first on: whole ones from whole to whole_end, ends of the row beside them.
    const T* base = p - lead;
    const int mine0 = first + tid, end = min(first + a.span, (a.V + lead + VE - 1) / VE), whole = lead > 0, whole_end = min(end, (a.V + lead) / VE);
    auto fetch = [&](int j) {                             // what lies outside: -inf
        const int g = mine0 + j * BM_NT;
        uint4 v = sizeof(T) == 4 ? make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u) : std::is_same<T, __half>::value ? make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u)
                                                                                                                                   : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
        if (g >= whole && g < whole_end) v = *reinterpret_cast<const uint4*>(base + (long long)g * VE);
        else if (g < end) {
            T e[VE];
            *reinterpret_cast<uint4*>(e) = v;
            for (int i = 0; i < VE; ++i) if (g * VE + i >= lead && g * VE + i < a.V + lead) e[i] = base[g * VE + i];
            v = *reinterpret_cast<uint4*>(e);
        }
        return v;
    };
    uint4 x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j] = fetch(j);
    if (tid == 0) count = 0;
    float vmax[NV], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        vmax[j] = fmaxf(Vec<T>::max_of(x[j]), -INFINITY);                                // (all NaN: none)
        top = fmaxf(top, vmax[j]);
    }
    {   // the warp's q largest lanes' maxima, one after another
        uint32_t mine = key_of(top), best = 0;
        for (int q = (a.n + BM_WARPS - 1) / BM_WARPS; q; --q) {
            best = __reduce_max_sync(0xffffffffu, mine);
            if (q == (a.n + BM_WARPS - 1) / BM_WARPS && lane == 0) w_max[warp] = of_key(best > NOTHING ? best : NOTHING);
            const unsigned who = __ballot_sync(0xffffffffu, mine == best);
            if (lane == __ffs(who) - 1) mine = 0;
        }
        if (lane == 0) w_bound[warp] = best;
    }
    __syncthreads();
    float m = w_max[0];
    uint32_t bound = w_bound[0];
#pragma unroll
    for (int w = 1; w < BM_WARPS; ++w) { m = fmaxf(m, w_max[w]); bound = min(bound, w_bound[w]); }
    // (the same for all threads) a warp has too few, as at a row's end: the n-th largest of all threads' maxima, each compared with all.  Rows that fill no stretch all go this way, 4 x 12 of 1000 in fp32 29 us
    // in a graph (of 32768: 10), 128 x 8 of 1000 in bf16 28 (27).
    if (bound <= NOTHING) {
        const uint32_t mine = key_of(top);
        uint32_t* maxima = reinterpret_cast<uint32_t*>(list);
        maxima[tid] = mine;
        __syncthreads();
        int more = 0, same = 0;
        for (int i = 0; i < BM_NT; ++i) { more += maxima[i] > mine; same += maxima[i] == mine; }
        if (more < a.n && more + same >= a.n) w_bound[0] = mine;      // (by all that have it)
        __syncthreads();
        bound = w_bound[0];
    }
    bound = max(bound, NOTHING + 1);
    // the sum
    float s = 0.f;
    const bool far = fabsf(m) >= 65536.f;                 // (as where a mask has put its type's lowest value) there m log2 e overflows, or its rounding is larger than the exponents that a float has
    if (m > -INFINITY && m < INFINITY) {
        const float c = m * LOG2E;
        u64 part[2] = {0, 0};                             // two sums each
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            // (hidden from the compiler once more: it would keep what it has unpacked from a vector in registers of their own)
            asm volatile("" : "+r"(x[j].x), "+r"(x[j].y), "+r"(x[j].z), "+r"(x[j].w));
#pragma unroll
            for (int i = 0; i < VE; i += 2) {
                const u64 y = fma2(pair2(Vec<T>::at(x[j], i), Vec<T>::at(x[j], i + 1)), pair2(LOG2E, LOG2E), pair2(-c, -c));
                part[i / 2 & 1] = add2(part[i / 2 & 1], pair2(exp2_of(lo2(y)), exp2_of(hi2(y))));
            }
        }
        part[0] = add2(part[0], part[1]);
        s = lo2(part[0]) + hi2(part[0]);
        if (far || s != s) {                              // NaN weigh nothing
            s = 0.f;
#pragma unroll 1
            for (int j = 0; j < NV; ++j) {
                const uint4 v = fetch(j);
                for (int i = 0; i < VE; ++i) s += fmaxf(far ? exp2_of((Vec<T>::at(v, i) - m) * LOG2E) : term(Vec<T>::at(v, i), c), 0.f);
            }
        }
    } else if (m == INFINITY) {                           // the infinite ones share the row
#pragma unroll 1
        for (int j = 0; j < NV; ++j) {
            const uint4 v = fetch(j);
            for (int i = 0; i < VE; ++i) s += Vec<T>::at(v, i) == INFINITY ? 1.f : 0.f;
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) w_sum[warp] = s;
    // what is above the bound: few threads have any, and those read the vector once more (unrolled over all vectors the code ran out of the instruction cache)
    const float least = of_key(bound);
    uint32_t have = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) have |= vmax[j] >= least ? 1u << j : 0u;
    for (uint32_t left = have; left; left &= left - 1) {
        const int j = __ffs(left) - 1;
        const uint4 v = fetch(j);
        uint32_t hits = 0;
#pragma unroll
        for (int i = 0; i < VE; ++i) hits |= Vec<T>::at(v, i) >= least ? 1u << i : 0u;
        for (; hits; hits &= hits - 1) {
            const int i = __ffs(hits) - 1, k = atomicAdd(&count, 1);
            if (k < BM_LIST) list[k] = entry(Vec<T>::pick(v, i), place(j, i));
        }
    }
    __syncthreads();
    if (tid == 0) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < BM_WARPS; ++w) sum += w_sum[w];
        if (!far) sum *= remainder_of(m);
        a.sums[at] = make_float2(m, sum);
    }
    u64* out = a.lists + at * a.n;
    const int c = count;
    if (c <= BM_LIST) {
        if (tid < a.n && tid >= c) out[tid] = 0;
        for (int k = tid / 8; k < (c + 3) / 4 * 4; k += BM_NT / 8) {                     // eight lanes an entry, whole warps
            const u64 mine = list[min(k, c - 1)];
            int rank = 0;
            for (int i = lane & 7; i < c; i += 8) rank += list[i] > mine;
#pragma unroll
            for (int o = 4; o; o >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
            if ((lane & 7) == 0 && k < c && rank < a.n) out[rank] = mine;
        }
        return;
    }
    u64 last = ~0ull;
    for (int k = 0; k < a.n; ++k) {
        u64 best = 0;
        for (uint32_t left = have; left; left &= left - 1) {
            const int j = __ffs(left) - 1;
            const uint4 v = fetch(j);
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const u64 e = entry(Vec<T>::at(v, i), place(j, i));
                if (Vec<T>::at(v, i) >= least && e < last && e > best) best = e;
            }
        }
        best = warp_max(best);
        if (lane == 0) w_best[warp] = best;
        __syncthreads();
        best = warp_max(w_best[lane % BM_WARPS]);
        __syncthreads();
        if (tid == 0) out[k] = best;
        last = best;
    }
}

// CTA = (stretch, row).
template <typename T, int NV>
__global__ void __launch_bounds__(BM_NT, NV == 8 ? 4 : 5) k_beam_rows(BeamArgs a) {
    op_begin();
    stretch_of_row<T, NV, BM_NT>(a, blockIdx.y, blockIdx.x);
}

__device__ __forceinline__ u64 ordered(double r) {        // order-preserving; NaN and -inf are not asked for
    const u64 u = (u64)__double_as_longlong(r);
    return u >> 63 ? ~u : u | 1ull << 63;
}

struct Beam { double ln_sum, score, norm; float top; int exact, done; };     // done: 1: goes on as it is, 2: dead
struct Candidate { double rank; u64 e; int beam; };
__device__ __forceinline__ bool ahead(const Candidate& x, const Candidate& y) {                   // by rank, lower beam, then the row's order
    return x.rank > y.rank || (x.rank == y.rank && (x.beam < y.beam || (x.beam == y.beam && x.e > y.e)));
}
__device__ __forceinline__ double log_probability(const Beam& b, u64 e) {
    const float l = of_key((uint32_t)(e >> 32));
    return (l == b.top ? 0.0 : (double)l - (double)b.top) - b.ln_sum;
}

// A sentence, by a CTA.  Its entries (K lists a stretch) are asked for at once, ahead of the sums.
template <typename T>
__device__ __forceinline__ void join_sentence(const BeamArgs& a, int b) {
    constexpr int BJ_WARPS = BJ_NT / 32;
    __shared__ Beam beams[BM_MOST];
    __shared__ u64 stage[BJ_STAGE];
    __shared__ Candidate list[BJ_LIST], sorted[BM_MOST], w_best[BJ_WARPS];
    __shared__ uint32_t w_bound[BJ_WARPS];
    __shared__ double w_sum[BJ_WARPS];
    __shared__ int count, again[BM_MOST];
    const int row0 = b * a.K, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = a.stretches * a.n, all = a.K * per;
    const u64* lists = a.lists + (long long)row0 * per;
    u64 mine_e[BJ_STAGE / BJ_NT];
#pragma unroll
    for (int j = 0; j < BJ_STAGE / BJ_NT; ++j) mine_e[j] = tid + j * BJ_NT < all ? lists[tid + j * BJ_NT] : 0;      // (rows that were not read leave anything: see candidate)
    for (int k = warp; k < a.K; k += BJ_WARPS) {          // the rows' sums
        const int row = row0 + k;
        const float score = a.scores[row];
        Beam x{0.0, (double)score, a.norm ? (double)a.norm[row] : 1.0, -INFINITY, 0, a.finished && a.finished[row] ? 1 : 0};
        if (!(score > -INFINITY)) x.done = 2;
        if (!x.done) {
            const float2* sums = a.sums + (long long)row * a.stretches;
            for (int i = lane; i < a.stretches; i += 32) x.top = fmaxf(x.top, sums[i].x);
#pragma unroll
            for (int o = 16; o; o >>= 1) x.top = fmaxf(x.top, __shfl_xor_sync(0xffffffffu, x.top, o));
            double s = 0.0;
            for (int i = lane; i < a.stretches; i += 32) { const float2 v = sums[i]; s += v.x == x.top ? (double)v.y : (double)v.y * exp((double)v.x - (double)x.top); }
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            x.ln_sum = log(s);
            if (x.top == -INFINITY) x.done = 2;
        }
        if (lane == 0) { beams[k] = x; again[k] = 0; }
    }
#pragma unroll
    for (int j = 0; j < BJ_STAGE / BJ_NT; ++j) stage[tid + j * BJ_NT] = mine_e[j];
    if (tid == 0) count = 0;
    __syncthreads();
    const float inv_per = 1.f / per;
    auto candidate = [&](int i, Candidate& c) {           // the i-th: beam, stretch, place in its list
        c.beam = (int)((i + 0.5f) * inv_per);             // i / per: `all` is at most 2^20, so the product is off by less than the half
        const Beam& x = beams[c.beam];
        if (x.done) {
            c.e = ~(uint32_t)a.end_token;
            c.rank = x.score * x.norm;
            if (x.done == 2 || i != c.beam * per) return false;
        } else {
            c.e = i < BJ_STAGE ? stage[i] : lists[i];
            if (!c.e) return false;
            c.rank = (x.score + log_probability(x, c.e)) * x.norm;
        }
        return c.rank > -INFINITY;
    };
    // a bound below the n-th best, as in a row, by the upper halves of the ranks as ordered integers
    // (a thread takes entries from all over: neighbours are of one sorted list, and a warp of poor ones makes a poor bound)
    uint32_t mine = 0;
    Candidate c;
    const int mixed = tid * 97 & (BJ_NT - 1);
    const bool has = mixed < all && candidate(mixed, c);  // (of most calls a thread's only one)
    if (has) mine = (uint32_t)(ordered(c.rank) >> 32);
    Candidate d;
    for (int i = mixed + BJ_NT; i < all; i += BJ_NT) if (candidate(i, d)) mine = max(mine, (uint32_t)(ordered(d.rank) >> 32));
    uint32_t bound = 0;
    for (int q = (a.n + BJ_WARPS - 1) / BJ_WARPS; q; --q) {
        bound = __reduce_max_sync(0xffffffffu, mine);
        const unsigned who = __ballot_sync(0xffffffffu, mine == bound);
        if (lane == __ffs(who) - 1) mine = 0;
    }
    double norm = 0.0;
    for (int k = 0; k < a.K; ++k) norm = fmax(norm, fabs(beams[k].norm));
    if (lane == 0) w_bound[warp] = bound;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < BJ_WARPS; ++w) bound = min(bound, w_bound[w]);
    double least = -INFINITY;
    if (bound) {
        const u64 u = (u64)bound << 32;
        least = __longlong_as_double((long long)(u >> 63 ? u & ~(1ull << 63) : ~u)) - 4 * NEAR * norm;       // (ranks may still move by a quarter of that, the n-th's too, and twice that is near)
    }
    if (has && !(c.rank < least)) {
        const int k = atomicAdd(&count, 1);
        if (k < BJ_LIST) list[k] = c;
    }
    for (int i = mixed + BJ_NT; i < all; i += BJ_NT)
        if (candidate(i, d) && !(d.rank < least)) {
            const int k = atomicAdd(&count, 1);
            if (k < BJ_LIST) list[k] = d;
        }
    __syncthreads();
    const int found = count;
    const int best_n = min(found, a.n);                   // sorted ones
    const double near = 2 * NEAR * norm;
    for (int round = 0; round <= a.K; ++round) {
        if (found <= BJ_LIST) {
            for (int i = tid / 8; i < (found + 3) / 4 * 4; i += BJ_NT / 8) {          // eight lanes an entry, whole warps
                const Candidate x = list[min(i, found - 1)];
                int rank = 0;
                for (int j = lane & 7; j < found; j += 8) rank += ahead(list[j], x);
#pragma unroll
                for (int o = 4; o; o >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
                if ((lane & 7) == 0 && i < found && rank < a.n) sorted[rank] = x;
            }
        } else {                                          // (more ties than the list holds)
            for (int k = 0; k < a.n; ++k) {
                Candidate top{-INFINITY, 0, a.K};
                for (int i = tid; i < all; i += BJ_NT)
                    if (candidate(i, c) && (k == 0 || ahead(sorted[k - 1], c)) && ahead(c, top)) top = c;
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const Candidate u{__shfl_xor_sync(0xffffffffu, top.rank, o), __shfl_xor_sync(0xffffffffu, top.e, o), __shfl_xor_sync(0xffffffffu, top.beam, o)};
                    if (ahead(u, top)) top = u;
                }
                if (lane == 0) w_best[warp] = top;
                __syncthreads();
                if (tid == 0) {
                    for (int w = 1; w < BJ_WARPS; ++w) if (ahead(w_best[w], top)) top = w_best[w];
                    sorted[k] = top;
                }
                __syncthreads();
            }
        }
        __syncthreads();
        // entries of different beams whose order the sums' errors could turn, one of them at least among the best
        bool open = false;
        auto settle = [&](const Candidate& one, const Candidate& other) {
            if (one.beam == other.beam || one.rank - other.rank > NEAR * (fabs(beams[one.beam].norm) + fabs(beams[other.beam].norm))) return;
            for (int k : {one.beam, other.beam})
                if (!beams[k].done && !beams[k].exact && beams[k].top < INFINITY) { again[k] = 1; open = true; }
        };
        if (tid < best_n)
            for (int i = tid + 1; i < best_n && sorted[tid].rank - sorted[i].rank <= near; ++i) settle(sorted[tid], sorted[i]);
        auto behind = [&](const Candidate& x) {
            for (int i = best_n - 1; i >= 0 && sorted[i].rank - x.rank <= near && ahead(sorted[i], x); --i) settle(sorted[i], x);
        };
        if (found <= BJ_LIST) { if (tid < found) behind(list[tid]); }
        else for (int i = tid; i < all; i += BJ_NT) if (candidate(i, c)) behind(c);
        if (!__syncthreads_or(open)) break;
        for (int k = 0; k < a.K; ++k) {                   // (the same for all threads)
            if (!again[k] || beams[k].exact) continue;
            const T* p = (const T*)a.logits + (long long)(row0 + k) * a.s_row;
            const double top = beams[k].top;
            double s = 0.0;
            for (int i0 = tid; i0 < a.V; i0 += 8 * BJ_NT) {
                float l[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) l[j] = i0 + j * BJ_NT < a.V ? as_float(p[i0 + j * BJ_NT]) : -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) s += l[j] > -INFINITY ? exp((double)l[j] - top) : 0.0;     // (NaN weigh nothing; eight in flight)
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0) w_sum[warp] = s;
            __syncthreads();
            if (tid == 0) {
                for (int w = 1; w < BJ_WARPS; ++w) s += w_sum[w];
                beams[k].ln_sum = log(s); beams[k].exact = 1;
            }
            __syncthreads();
        }
        if (found <= BJ_LIST)
            for (int i = tid; i < found; i += BJ_NT) {
                const Beam& x = beams[list[i].beam];
                if (!x.done) list[i].rank = (x.score + log_probability(x, list[i].e)) * x.norm;
            }
        __syncthreads();
    }
    if (tid < a.n) {
        const long long o = (long long)b * a.n + tid;
        float score = -INFINITY;
        int parent = -1, token = -1;
        if (tid < best_n) {
            const Candidate x = sorted[tid];
            const Beam& y = beams[x.beam];
            parent = x.beam;
            token = (int)~(uint32_t)x.e;
            score = (float)(y.done ? y.score : y.score + log_probability(y, x.e));
        }
        a.out_scores[o] = score; a.out_parent[o] = parent; a.out_token[o] = token;
    }
}

template <typename T>
__global__ void __launch_bounds__(BJ_NT) k_beam_join(BeamArgs a) {
    op_begin();
    join_sentence<T>(a, blockIdx.x);
}
// Both in one launch, a cluster a sentence: its CTAs take the stretches of all its rows in turn, the first joins them.
template <typename T>
__global__ void __launch_bounds__(BJ_NT, 2) k_beam_one(BeamArgs a) {
    op_begin();
    const int b = blockIdx.x / BO_CLUSTER, rank = blockIdx.x % BO_CLUSTER;
    for (int i = rank; i < a.K * a.stretches; i += BO_CLUSTER) {
        stretch_of_row<T, BO_NV, BJ_NT>(a, b * a.K + i / a.stretches, i % a.stretches);
        __syncthreads();
    }
    tc_cluster_sync();
    if (rank == 0) join_sentence<T>(a, b);
}

// Vectors of a thread: as many as leave two CTAs for every SM, so that few rows are spread over the GPU and many are read in few, large stretches.
int vectors(long long rows, int V, int e) {               // (two launches)
    for (int nv = 8; nv > 1; nv /= 2) if (rows * ((V + BM_NT * nv * (16 / e) - 1) / (BM_NT * nv * (16 / e))) >= 2 * 148) return nv;
    return 1;
}
// Stretches of a row whose first element is `lead` elements into a vector.
int stretches(int threads, int nv, int V, int e, int lead) { const int per = threads * nv * (16 / e); return (V + lead + per - 1) / per; }
// Sentences in one launch: where each CTA has an SM, and two stretches at most.  The host is what small calls wait for, and a launch is 2.7 us of it: one sentence of 4 x 32768 16.3 -> 13.7 us, though the
// GPU alone takes 9.0 instead of 7.8.  (32 of 5 x 50265, three stretches a CTA and two CTAs an SM: 20 us instead of 12.)
bool in_one(int B, int K, int V, int e) { return (long long)B * BO_CLUSTER <= 148 && K * stretches(BJ_NT, BO_NV, V, e, 16 / e - 1) <= BO_ITEMS * BO_CLUSTER; }
int most_stretches(int B, int K, int V, int e) {
    return in_one(B, K, V, e) ? stretches(BJ_NT, BO_NV, V, e, 16 / e - 1) : stretches(BM_NT, vectors((long long)B * K, V, e), V, e, 16 / e - 1);
}
const char* why_not(int B, int K, int V, int n, int dtype) {
    if (B < 0 || K < 1 || V < 1 || n < 1) return "a size is below 1";
    if (!op_elem_bytes(dtype)) return "unknown dtype";
    return nullptr;
}
bool too_large(int B, int K, int V, int n) { return K > BM_MOST || n > BM_MOST || V > 1 << 20 || (long long)B * K > 65535; }
constexpr const char* LARGE = "more than 64 beams or results, 2^20 tokens or 65535 rows";

template <typename T>
cudaError_t run(const BeamArgs& a, int nv, bool one, cudaStream_t st) {
    if (one) return op_launch(k_beam_one<T>, dim3(a.B * BO_CLUSTER), BJ_NT, 0, st, BO_CLUSTER, a);
    const dim3 grid(a.stretches, a.B * a.K);
    auto k = nv == 8 ? k_beam_rows<T, 8> : nv == 4 ? k_beam_rows<T, 4> : nv == 2 ? k_beam_rows<T, 2> : k_beam_rows<T, 1>;
    if (const cudaError_t e = op_launch(k, grid, BM_NT, 0, st, 1, a)) return e;
    return op_launch(k_beam_join<T>, dim3(a.B), BJ_NT, 0, st, 1, a);
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_beam_select_workspace(int B, int K, int V, int n, int dtype) {
    if (const char* why = why_not(B, K, V, n, dtype)) return op_bad("beam_select_workspace", why);
    if (too_large(B, K, V, n)) return op_fail(SPECDEC_ERR_CAPACITY, "beam_select_workspace", LARGE);
    const int e = op_elem_bytes(dtype);
    return (long long)B * K * most_stretches(B, K, V, e) * (8 + 8LL * n);
}

int specdec_beam_select(const specdec_beam_select_args* g, void* stream) {
    const char* who = "beam_select";
    if (!g) return op_bad(who, "a pointer is NULL");
    const int B = g->B, K = g->K, V = g->V, n = g->n, dtype = g->dtype;
    if (const char* why = why_not(B, K, V, n, dtype)) return op_bad(who, why);
    if (too_large(B, K, V, n)) return op_fail(SPECDEC_ERR_CAPACITY, who, LARGE);
    if (B == 0) return SPECDEC_OK;
    if (!g->d_logits || !g->d_scores || !g->d_out_scores || !g->d_out_parent || !g->d_out_token) return op_bad(who, "a pointer is NULL");
    const int e = op_elem_bytes(dtype);
    if ((uintptr_t)g->d_logits % e || g->stride < 0) return op_bad(who, "d_logits is not aligned to its type, or the stride is negative");
    const long long need = specdec_beam_select_workspace(B, K, V, n, dtype);
    if (!g->d_workspace || (uintptr_t)g->d_workspace % 8 || g->workspace_bytes < need)
        return op_fail(SPECDEC_ERR_CAPACITY, who, "the workspace is smaller than specdec_beam_select_workspace says, or not 8-byte aligned");
    BeamArgs a;
    const bool one = in_one(B, K, V, e);
    const int nv = one ? BO_NV : vectors((long long)B * K, V, e);
    a.logits = g->d_logits; a.s_row = op_stride(g->stride, B * K); a.V = V;
    a.scores = g->d_scores; a.finished = g->d_finished; a.norm = g->d_norm;
    a.end_token = g->end_token; a.B = B; a.K = K; a.n = n;
    const int lead = ((uintptr_t)g->d_logits | (uintptr_t)(a.s_row * e)) % 16 ? 16 / e - 1 : 0, vecs = (V + lead + 16 / e - 1) / (16 / e);
    a.stretches = stretches(one ? BJ_NT : BM_NT, nv, V, e, lead);
    a.span = (vecs + a.stretches - 1) / a.stretches;      // (equal ones)
    a.out_scores = g->d_out_scores; a.out_parent = g->d_out_parent; a.out_token = g->d_out_token;
    a.sums = (float2*)g->d_workspace; a.lists = (u64*)(a.sums + (long long)B * K * a.stretches);
    const cudaStream_t st = (cudaStream_t)stream;
    return op_done(who, dtype == SPECDEC_DTYPE_F32 ? run<float>(a, nv, one, st) : dtype == SPECDEC_DTYPE_BF16 ? run<__nv_bfloat16>(a, nv, one, st) : run<__half>(a, nv, one, st));
}

}  // extern "C"
