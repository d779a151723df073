// Beam search's selection: the n best continuations of a sentence's beams over the whole vocabulary (contract: specdec.h).
//
// Two launches.  k_beam_rows: a CTA takes a stretch of a row into registers, with every load under way at once, and leaves its maximum m, its sum of e^(l - m) and its n largest entries.
// k_beam_join: a CTA a sentence joins the stretches' sums, ranks the entries that are left (a few hundred) and writes the best n.  The logits are read once; no log-probability but those of the
// entries that are left is ever taken.
//
// The n largest: the q-th largest of a warp's lanes' maxima, q = n / 8 rounded up, has q entries of the warp at or above it, so the least of the eight warps' is a bound below the n-th largest entry of
// the stretch.  What lies above it (some 2 n entries) is listed and ranked by counting.  Where ties make more of it than the list holds, the largest entry below the last one is looked for n times.
//
// Sums are fp32, off by some 2^-22; scores and ranks are 64 bits from there on.  Where ranks of two beams lie within 2^-19 (times norm) of one another and the order of the best n would turn on it, the
// sums of those beams are taken again in 64 bits: the choice is that of exact sums.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "op_error.cuh"

namespace sd {
namespace {

typedef unsigned long long u64;
constexpr int BM_NT = 256, BM_WARPS = BM_NT / 32, BM_MOST = 64, BM_LIST = 512, BM_JOIN = 512;       // threads; beams and results at most; listed entries of a stretch, of a sentence
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
    int end_token, B, K, n, stretches;
    float* out_scores; int* out_parent; int* out_token;
    float2* sums; u64* lists;                             // [row, stretch]: (maximum, sum); [row, stretch, n], best first, 0 where there are fewer
    __device__ __forceinline__ bool alive(int row) const { return scores[row] > -INFINITY && !(finished && finished[row]); }       // (NaN: dead)
};

template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    static __device__ __forceinline__ float at(const uint4& v, int i) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else { const __half2 h = *reinterpret_cast<const __half2*>(w + i / 2); return i & 1 ? __high2float(h) : __low2float(h); }
    }
};
template <typename T> __device__ __forceinline__ float as_float(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __bfloat162float(x);
    else return __half2float(x);
}
__device__ __forceinline__ float exp2_of(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ u64 warp_max(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) { const u64 u = __shfl_xor_sync(0xffffffffu, v, o); if (u > v) v = u; }
    return v;
}

// CTA = (stretch, row) of NV vectors a thread.
template <typename T, int NV>
__global__ void __launch_bounds__(BM_NT) k_beam_rows(BeamArgs a) {
    constexpr int VE = Vec<T>::N;
    __shared__ float w_max[BM_WARPS], w_sum[BM_WARPS];
    __shared__ uint32_t w_bound[BM_WARPS];
    __shared__ u64 list[BM_LIST], w_best[BM_WARPS];
    __shared__ int count;
    op_begin();
    const int row = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long at = (long long)row * a.stretches + blockIdx.x;
    if (!a.alive(row)) return;
    const T* p = (const T*)a.logits + row * a.s_row;
    const int lead = (int)(((uintptr_t)p & 15) / sizeof(T));          // elements of the first vector that lie ahead of the row
    const int first = blockIdx.x * BM_NT * NV;
    auto place = [&](int j, int i) { return (first + j * BM_NT + tid) * VE - lead + i; };
    uint4 x[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i0 = place(j, 0);
        if (i0 >= 0 && i0 + VE <= a.V) x[j] = *reinterpret_cast<const uint4*>(p + i0);
        else {
            T e[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                if (i0 + i >= 0 && i0 + i < a.V) e[i] = p[i0 + i];
                else if constexpr (sizeof(T) == 4) e[i] = -INFINITY;
                else if constexpr (std::is_same<T, __nv_bfloat16>::value) e[i] = __float2bfloat16_rn(-INFINITY);
                else e[i] = __float2half_rn(-INFINITY);
            }
            x[j] = *reinterpret_cast<const uint4*>(e);
        }
    }
    if (tid == 0) count = 0;
    float vmax[NV], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        vmax[j] = -INFINITY;
#pragma unroll
        for (int i = 0; i < VE; ++i) vmax[j] = fmaxf(vmax[j], Vec<T>::at(x[j], i));      // (NaN: passed over)
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
    if (bound <= NOTHING) {                               // (the same for all threads) a warp has too few, as at a row's end: the n-th largest of all threads' maxima
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
    if (m > -INFINITY && m < INFINITY) {
        const float c = m * LOG2E;
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) part[i & 3] += exp2_of(fmaf(Vec<T>::at(x[j], i), LOG2E, -c));
        s = (part[0] + part[1]) + (part[2] + part[3]);
        if (s != s) {                                     // NaN weigh nothing
            s = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) s += fmaxf(exp2_of(fmaf(Vec<T>::at(x[j], i), LOG2E, -c)), 0.f);
        }
    } else if (m == INFINITY) {                           // the infinite ones share the row
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) s += Vec<T>::at(x[j], i) == INFINITY ? 1.f : 0.f;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) w_sum[warp] = s;
    // what is above the bound
    const float least = of_key(bound);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (vmax[j] >= least) {
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const float l = Vec<T>::at(x[j], i);
                if (l >= least) {
                    const int k = atomicAdd(&count, 1);
                    if (k < BM_LIST) list[k] = entry(l, place(j, i));
                }
            }
        }
    __syncthreads();
    if (tid == 0) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < BM_WARPS; ++w) sum += w_sum[w];
        if (m > -INFINITY && m < INFINITY) sum *= exp2f(-fmaf(m, LOG2E, -(m * LOG2E)));          // what the rounding of m log2 e has put into every term
        a.sums[at] = make_float2(m, sum);
    }
    u64* out = a.lists + at * a.n;
    const int c = count;
    if (c <= BM_LIST) {
        if (tid < a.n && tid >= c) out[tid] = 0;
        for (int k = tid; k < c; k += BM_NT) {
            const u64 mine = list[k];
            int rank = 0;
            for (int i = 0; i < c; ++i) rank += list[i] > mine;
            if (rank < a.n) out[rank] = mine;
        }
        return;
    }
    u64 last = ~0ull;
    for (int k = 0; k < a.n; ++k) {
        u64 best = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (vmax[j] >= least)
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float l = Vec<T>::at(x[j], i);
                    const u64 e = entry(l, place(j, i));
                    if (l >= least && e < last && e > best) best = e;
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
// The i-th candidate of a sentence: beam, stretch, place in its list.
__device__ __forceinline__ bool candidate(const BeamArgs& a, const Beam* beams, int row0, int i, Candidate& c) {
    const int per = a.stretches * a.n;
    c.beam = i / per;
    const Beam& b = beams[c.beam];
    if (b.done == 2) return false;
    if (b.done) {
        if (i - c.beam * per) return false;
        c.e = ~(uint32_t)a.end_token;
        c.rank = b.score * b.norm;
    } else {
        c.e = a.lists[(long long)row0 * per + i];
        if (!c.e) return false;
        c.rank = (b.score + log_probability(b, c.e)) * b.norm;
    }
    return c.rank > -INFINITY;
}

// CTA = sentence.
template <typename T>
__global__ void __launch_bounds__(BM_NT) k_beam_join(BeamArgs a) {
    __shared__ Beam beams[BM_MOST];
    __shared__ Candidate list[BM_JOIN], sorted[BM_MOST + 1];
    __shared__ uint32_t w_bound[BM_WARPS];
    __shared__ double w_sum[BM_WARPS];
    __shared__ Candidate w_best[BM_WARPS];
    __shared__ int count, again[BM_MOST];
    op_begin();
    const int b = blockIdx.x, row0 = b * a.K, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int k = warp; k < a.K; k += BM_WARPS) {          // the rows' sums
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
    if (tid == 0) count = 0;
    __syncthreads();
    // a bound below the n-th best, as in a row, by the upper halves of the ranks as ordered integers
    const int all = a.K * a.stretches * a.n;
    uint32_t mine = 0;
    Candidate c;
    for (int i = tid; i < all; i += BM_NT) if (candidate(a, beams, row0, i, c)) mine = max(mine, (uint32_t)(ordered(c.rank) >> 32));
    uint32_t bound = 0;
    for (int q = (a.n + 1 + BM_WARPS - 1) / BM_WARPS; q; --q) {       // (the one behind the n-th is looked at too)
        bound = __reduce_max_sync(0xffffffffu, mine);
        const unsigned who = __ballot_sync(0xffffffffu, mine == bound);
        if (lane == __ffs(who) - 1) mine = 0;
    }
    double norm = 0.0;
    for (int k = lane; k < a.K; k += 32) norm = fmax(norm, fabs(beams[k].norm));
#pragma unroll
    for (int o = 16; o; o >>= 1) norm = fmax(norm, __shfl_xor_sync(0xffffffffu, norm, o));
    if (lane == 0) w_bound[warp] = bound;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < BM_WARPS; ++w) bound = min(bound, w_bound[w]);
    double least = -INFINITY;
    if (bound) {
        const u64 u = (u64)bound << 32;
        least = __longlong_as_double((long long)(u >> 63 ? u & ~(1ull << 63) : ~u)) - 4 * NEAR * norm;       // (ranks may still move by as much)
    }
    for (int i = tid; i < all; i += BM_NT)
        if (candidate(a, beams, row0, i, c) && (!(c.rank < least))) {
            const int k = atomicAdd(&count, 1);
            if (k < BM_JOIN) list[k] = c;
        }
    __syncthreads();
    const int found = count;
    int best_n = min(found, a.n + 1);                     // sorted ones
    for (int round = 0; round <= a.K; ++round) {
        if (found <= BM_JOIN) {
            for (int i = tid; i < found; i += BM_NT) {
                const Candidate x = list[i];
                int rank = 0;
                for (int j = 0; j < found; ++j) rank += ahead(list[j], x);
                if (rank <= a.n) sorted[rank] = x;
            }
        } else {                                          // (more ties than the list holds)
            for (int k = 0; k <= a.n; ++k) {
                Candidate top{-INFINITY, 0, a.K};
                for (int i = tid; i < all; i += BM_NT)
                    if (candidate(a, beams, row0, i, c) && (k == 0 || ahead(sorted[k - 1], c)) && ahead(c, top)) top = c;
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const Candidate u{__shfl_xor_sync(0xffffffffu, top.rank, o), __shfl_xor_sync(0xffffffffu, top.e, o), __shfl_xor_sync(0xffffffffu, top.beam, o)};
                    if (ahead(u, top)) top = u;
                }
                if (lane == 0) w_best[warp] = top;
                __syncthreads();
                if (tid == 0) {
                    for (int w = 1; w < BM_WARPS; ++w) if (ahead(w_best[w], top)) top = w_best[w];
                    sorted[k] = top;
                }
                __syncthreads();
            }
        }
        __syncthreads();
        // neighbours of different beams whose order the sums' errors could turn
        bool open = false;
        if (tid + 1 < best_n) {
            const Candidate x = sorted[tid], y = sorted[tid + 1];
            if (x.beam != y.beam && x.rank - y.rank <= NEAR * (fabs(beams[x.beam].norm) + fabs(beams[y.beam].norm)))
                for (int k : {x.beam, y.beam})
                    if (!beams[k].done && !beams[k].exact && beams[k].top < INFINITY) { again[k] = 1; open = true; }
        }
        if (!__syncthreads_or(open)) break;
        for (int k = 0; k < a.K; ++k) {                   // (the same for all threads)
            if (!again[k] || beams[k].exact) continue;
            const T* p = (const T*)a.logits + (long long)(row0 + k) * a.s_row;
            const double top = beams[k].top;
            double s = 0.0;
            for (int i = tid; i < a.V; i += BM_NT) {
                const float l = as_float(p[i]);
                if (l == l) s += exp((double)l - top);
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0) w_sum[warp] = s;
            __syncthreads();
            if (tid == 0) {
                for (int w = 1; w < BM_WARPS; ++w) s += w_sum[w];
                beams[k].ln_sum = log(s); beams[k].exact = 1;
            }
            __syncthreads();
        }
        if (found <= BM_JOIN)
            for (int i = tid; i < found; i += BM_NT) {
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

// Vectors of a thread: as many as leave two CTAs for every SM, so that few rows are spread over the GPU and many are read in few, large stretches.
int vectors(long long rows, int V, int e) {
    for (int nv = 8; nv > 1; nv /= 2) if (rows * ((V + BM_NT * nv * (16 / e) - 1) / (BM_NT * nv * (16 / e))) >= 2 * 148) return nv;
    return 1;
}
int stretches(int nv, int V, int e) { const int per = BM_NT * nv * (16 / e); return (V + 16 / e - 1 + per - 1) / per; }       // (a row may begin inside a vector)
const char* why_not(int B, int K, int V, int n, int dtype) {
    if (B < 0 || K < 1 || V < 1 || n < 1) return "a size is below 1";
    if (!op_elem_bytes(dtype)) return "unknown dtype";
    return nullptr;
}
bool too_large(int B, int K, int V, int n) { return K > BM_MOST || n > BM_MOST || V > 1 << 20 || (long long)B * K > 65535; }
constexpr const char* LARGE = "more than 64 beams or results, 2^20 tokens or 65535 rows";

template <typename T>
cudaError_t run(const BeamArgs& a, int nv, cudaStream_t st) {
    const dim3 grid(a.stretches, a.B * a.K);
    auto k = nv == 8 ? k_beam_rows<T, 8> : nv == 4 ? k_beam_rows<T, 4> : nv == 2 ? k_beam_rows<T, 2> : k_beam_rows<T, 1>;
    if (const cudaError_t e = op_launch(k, grid, BM_NT, 0, st, 1, a)) return e;
    return op_launch(k_beam_join<T>, dim3(a.B), BM_NT, 0, st, 1, a);
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_beam_select_workspace(int B, int K, int V, int n, int dtype) {
    if (const char* why = why_not(B, K, V, n, dtype)) return op_bad("beam_select_workspace", why);
    if (too_large(B, K, V, n)) return op_fail(SPECDEC_ERR_CAPACITY, "beam_select_workspace", LARGE);
    const int e = op_elem_bytes(dtype);
    return (long long)B * K * stretches(vectors((long long)B * K, V, e), V, e) * (8 + 8LL * n);
}

int specdec_beam_select(const void* d_logits, int dtype, long long stride, int B, int K, int V, const float* d_scores, const unsigned char* d_finished, int end_token, const float* d_norm, int n,
                        float* d_out_scores, int32_t* d_out_parent, int32_t* d_out_token, void* d_workspace, long long workspace_bytes, void* stream) {
    const char* who = "beam_select";
    if (const char* why = why_not(B, K, V, n, dtype)) return op_bad(who, why);
    if (too_large(B, K, V, n)) return op_fail(SPECDEC_ERR_CAPACITY, who, LARGE);
    if (B == 0) return SPECDEC_OK;
    if (!d_logits || !d_scores || !d_out_scores || !d_out_parent || !d_out_token) return op_bad(who, "a pointer is NULL");
    const int e = op_elem_bytes(dtype);
    if ((uintptr_t)d_logits % e || stride < 0) return op_bad(who, "d_logits is not aligned to its type, or the stride is negative");
    const long long need = specdec_beam_select_workspace(B, K, V, n, dtype);
    if (!d_workspace || (uintptr_t)d_workspace % 8 || workspace_bytes < need) return op_fail(SPECDEC_ERR_CAPACITY, who, "the workspace is smaller than specdec_beam_select_workspace says, or not 8-byte aligned");
    BeamArgs a;
    const int nv = vectors((long long)B * K, V, e);
    a.logits = d_logits; a.s_row = op_stride(stride, B * K); a.V = V;
    a.scores = d_scores; a.finished = d_finished; a.norm = d_norm;
    a.end_token = end_token; a.B = B; a.K = K; a.n = n; a.stretches = stretches(nv, V, e);
    a.out_scores = d_out_scores; a.out_parent = d_out_parent; a.out_token = d_out_token;
    a.sums = (float2*)d_workspace; a.lists = (u64*)(a.sums + (long long)B * K * a.stretches);
    const cudaStream_t st = (cudaStream_t)stream;
    return op_done(who, dtype == SPECDEC_DTYPE_F32 ? run<float>(a, nv, st) : dtype == SPECDEC_DTYPE_BF16 ? run<__nv_bfloat16>(a, nv, st) : run<__half>(a, nv, st));
}

}  // extern "C"
