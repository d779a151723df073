// Pages of a K/V cache in the caller's memory: reserve, append, compact, release, fork (contract: specdec.h).
//
// Bookkeeping is a table of pages a sequence and a reference count a page; a free page is one whose count is 0, and the lowest free ones
// are given out first, so that no call's result depends on the order in which CTAs run: reference counts are sums of integers, and everything
// else is written by one CTA.  A call that cannot get all its pages changes nothing.
//
// The data are moved as 16-byte pieces, every piece read once and written once; what bounds large moves is HBM, a decoding step's the five launches behind one another.
// 8 prompts forked into 4 branches each, 32 layers of pages of 128 tokens (81 MB read, the other three times from L2, 326 MB written): 74 us, 65 of them the copy.  32 sentences
// of 26 new tokens, 6 layers of 8 heads of 64 in bf16: fork, reserve, append (20 MB) and compact 26 us together.
#include <cuda_runtime.h>
#include <stdint.h>

#include "op_error.cuh"

namespace sd {
namespace {

constexpr int CP_ALLOC_THREADS = 1024;

struct Cache {                                            // specdec_cache with strides in bytes and a token's row in 16-byte pieces
    char* kv;
    int* table; int* length; int* held; int* refs; int* status; int* scratch;
    long long s_layer, s_side, s_page, s_token, s_head;
    int n_pages, n_seqs, max_pages, page_shift;
    int heads, chunks;                                    // a token's row: heads (1 where they are contiguous) x chunks
    __device__ __forceinline__ bool seq_ok(int s) const { return (unsigned)s < (unsigned)n_seqs; }
    __device__ __forceinline__ bool page_ok(int p) const { return (unsigned)p < (unsigned)n_pages; }
    __device__ __forceinline__ int held_of(int s) const { return min(max(held[s], 0), max_pages); }
    // scratch: [0] whether the call got its pages, then per entry of the call the rank of its first new page, [n_pages] the pages given
    // out, per sequence the tickets of compact; fork: per pair source page / tokens / length, and the sources' tables
    __device__ __forceinline__ int* sc_ok() const { return scratch; }
    __device__ __forceinline__ int* sc_first() const { return scratch + 16; }
    __device__ __forceinline__ int* sc_pages() const { return scratch + 16 + n_seqs; }
    __device__ __forceinline__ int* sc_ticket() const { return scratch + 16 + n_seqs + n_pages; }
    __device__ __forceinline__ int* sc_pair() const { return scratch + 16 + 2 * n_seqs + n_pages; }
    __device__ __forceinline__ int* sc_rows() const { return scratch + 16 + 4 * n_seqs + n_pages; }
};

__device__ __forceinline__ int4 ld16(const char* p) { return *reinterpret_cast<const int4*>(p); }
__device__ __forceinline__ void st16(char* p, int4 v) { *reinterpret_cast<int4*>(p) = v; }

// Inclusive sum over the CTA's 1024 threads; *total: the sum of all.
__device__ __forceinline__ int cta_scan(int v, int* warp_sums, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += u; }
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int w = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, w, o); if (lane >= o) w += u; }
        warp_sums[lane] = w;
    }
    __syncthreads();
    if (warp) v += warp_sums[warp - 1];
    *total = warp_sums[31];
    __syncthreads();
    return v;
}

// The lowest `want` free pages, in order, into sc_pages(); returns whether there are as many.  Each of the 32 warps counts and then lists the
// zeros of its own stretch of the reference counts.
__device__ bool find_pages(const Cache& c, int want, int* warp_sums) {
    if (want <= 0) return true;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = ((c.n_pages + 31) / 32 + 31) / 32 * 32;
    const int lo = min(warp * per, c.n_pages), hi = min(lo + per, c.n_pages);
    int n = 0;
#pragma unroll 8
    for (int p = lo + lane; p < hi; p += 32) n += __ldcg(c.refs + p) == 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    int total;
    const int upto = cta_scan(lane == 0 ? n : 0, warp_sums, &total);
    if (total < want) return false;
    int first = __shfl_sync(0xffffffffu, upto, 0) - n;
    for (int p0 = lo; p0 < hi && first < want; p0 += 128) {
        bool f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { const int p = p0 + 32 * j + lane; f[j] = p < hi && __ldcg(c.refs + p) == 0; }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned m = __ballot_sync(0xffffffffu, f[j]);
            const int r = first + __popc(m & ((1u << lane) - 1));
            if (f[j] && r < want) c.sc_pages()[r] = p0 + 32 * j + lane;
            first += __popc(m);
        }
    }
    __syncthreads();
    return true;
}

__global__ void __launch_bounds__(CP_ALLOC_THREADS) k_cache_reserve(Cache c, const int* seqs, int n, int n_tokens) {
    __shared__ int warp_sums[32];
    op_begin();
    int run = 0;
    bool full = false;
    for (int i0 = 0; i0 < n; i0 += CP_ALLOC_THREADS) {
        const int i = i0 + threadIdx.x;
        int need = 0, total;
        if (i < n) {
            const int s = seqs[i];
            if (c.seq_ok(s)) {
                const long long want = ((long long)max(c.length[s], 0) + n_tokens + (1 << c.page_shift) - 1) >> c.page_shift;
                full |= want > c.max_pages;
                need = (int)max(min(want, (long long)c.max_pages) - c.held_of(s), 0ll);
            } else {
                atomicOr(c.status, SPECDEC_CACHE_BAD_INDEX);
            }
        }
        const int upto = cta_scan(need, warp_sums, &total);
        if (i < n) c.sc_first()[i] = run + upto - need;
        run += total;
    }
    if (__syncthreads_or(full)) { if (threadIdx.x == 0) atomicOr(c.status, SPECDEC_CACHE_ROW_FULL); return; }
    if (!find_pages(c, run, warp_sums)) { if (threadIdx.x == 0) atomicOr(c.status, SPECDEC_CACHE_NO_PAGES); return; }
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < n; i += CP_ALLOC_THREADS / 32) {
        const int s = seqs[i];
        if (!c.seq_ok(s)) continue;
        const int first = c.sc_first()[i], need = (i + 1 < n ? c.sc_first()[i + 1] : run) - first, held = c.held_of(s);
        for (int j = lane; j < need && held + j < c.max_pages; j += 32) {
            const int p = c.sc_pages()[first + j];
            c.table[(long long)s * c.max_pages + held + j] = p;
            c.refs[p] = 1;
        }
        __syncwarp();
        if (lane == 0 && need) c.held[s] = held + need;
    }
}

__global__ void k_cache_release(Cache c, const int* seqs) {
    op_begin();
    const int s = seqs[blockIdx.x];
    if (!c.seq_ok(s)) { if (threadIdx.x == 0) atomicOr(c.status, SPECDEC_CACHE_BAD_INDEX); return; }
    const int held = c.held_of(s);
    for (int j = threadIdx.x; j < held; j += blockDim.x) {
        int* t = c.table + (long long)s * c.max_pages + j;
        if (c.page_ok(*t)) atomicAdd(c.refs + *t, -1);
        *t = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0) { c.held[s] = 0; c.length[s] = 0; }
}

// Where slot `pos` of sequence s is (bytes from the side's begin), or -1 where that is no page of the sequence's own.
__device__ __forceinline__ long long own_slot(const Cache& c, int s, int pos) {
    const int i = pos >> c.page_shift;
    if (pos < 0 || i >= c.held_of(s)) return -1;
    const int p = c.table[(long long)s * c.max_pages + i];
    if (!c.page_ok(p) || c.refs[p] != 1) return -1;
    return p * c.s_page + (pos & ((1 << c.page_shift) - 1)) * c.s_token;
}

struct AppendArgs {
    const char* k; const char* v;
    long long s_layer, s_seq, s_token, s_head;            // bytes
    const int* seqs; const int* count;
    int layer, T, heads, chunks;                          // heads = 1 where both sides' heads are contiguous
    long long cache_s_head;
};
// One CTA a token and layer; a thread copies one piece of the keys and one of the values at a time.
__global__ void k_cache_append(Cache c, AppendArgs a) {
    op_begin();
    const int t = blockIdx.x, i = blockIdx.y, s = a.seqs[i];
    if (a.count && t >= a.count[i]) return;
    const long long slot = c.seq_ok(s) ? own_slot(c, s, c.length[s] + t) : -1;
    if (slot < 0) { if (threadIdx.x == 0) atomicOr(c.status, c.seq_ok(s) ? SPECDEC_CACHE_UNRESERVED : SPECDEC_CACHE_BAD_INDEX); return; }
    const long long from = blockIdx.z * a.s_layer + i * a.s_seq + t * a.s_token;
    char* to = c.kv + (a.layer + blockIdx.z) * c.s_layer + slot;
    for (int u = threadIdx.x; u < a.heads * a.chunks; u += blockDim.x) {
        const int h = a.heads == 1 ? 0 : u / a.chunks;
        const int x = (u - h * a.chunks) * 16;
        const int4 k = ld16(a.k + from + h * a.s_head + x), v = ld16(a.v + from + h * a.s_head + x);
        char* p = to + h * a.cache_s_head + x;
        st16(p, k);
        st16(p + c.s_side, v);
    }
}

// CTA = (64 columns' worth of pieces of one layer and side, sequence).  A thread moves its piece of every token of the path, in the path's order and
// up to eight at a time, all eight read before the first is written: path[i] >= i, so a write goes to a slot whose own token was read before or is dropped.
// The CTA that finishes a sequence last moves its length and gives pages back.
// The whole path is checked before anything moves; addresses are at hand for CC_PATH of its tokens at a time.
constexpr int CC_PATH = 1024;
__global__ void __launch_bounds__(128) k_cache_compact(Cache c, const int* seqs, const int* path, int path_stride,
                                                       const int* n_path, int sides) {
    __shared__ long long from[CC_PATH], to[CC_PATH];
    __shared__ int s_last;
    op_begin();
    const int b = blockIdx.y, s = seqs[b], n = n_path[b];
    const int* pa = path + (long long)b * path_stride;
    if (!c.seq_ok(s)) { if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(c.status, SPECDEC_CACHE_BAD_INDEX); return; }
    const int len = c.length[s];
    int bad = n < 0 || n > path_stride ? SPECDEC_CACHE_BAD_INDEX : 0;
    if (!bad)
        for (int j = threadIdx.x; j < n; j += blockDim.x) {
            const int x = pa[j];
            if (x < j || (j && pa[j - 1] >= x)) { bad = SPECDEC_CACHE_BAD_INDEX; break; }
            const long long f = own_slot(c, s, len + x), t = own_slot(c, s, len + j);
            if (f < 0 || t < 0) bad = SPECDEC_CACHE_UNRESERVED;
            if (j < CC_PATH) { from[j] = f; to[j] = t; }
        }
    const bool index = __syncthreads_or(bad & SPECDEC_CACHE_BAD_INDEX), slot = __syncthreads_or(bad & SPECDEC_CACHE_UNRESERVED);
    if (index || slot) { if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(c.status, index ? SPECDEC_CACHE_BAD_INDEX : SPECDEC_CACHE_UNRESERVED); return; }
    const int per = c.heads * c.chunks;
    for (int n0 = 0; n0 < n; n0 += CC_PATH) {
        const int m = min(n - n0, CC_PATH);
        if (n0) {
            __syncthreads();                              // the last ones' addresses have been used
            for (int j = threadIdx.x; j < m; j += blockDim.x) { from[j] = own_slot(c, s, len + pa[n0 + j]); to[j] = own_slot(c, s, len + n0 + j); }
            __syncthreads();
        }
        for (long long u = (long long)blockIdx.x * blockDim.x + threadIdx.x; u < (long long)sides * per; u += (long long)gridDim.x * blockDim.x) {
            const int side = (int)(u / per), r = (int)(u % per), h = c.heads == 1 ? 0 : r / c.chunks;
            char* base = c.kv + (side >> 1) * c.s_layer + (side & 1) * c.s_side + h * c.s_head + (r - h * c.chunks) * 16;
            for (int j0 = 0; j0 < m; j0 += 8) {
                int4 x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j0 + j < m) x[j] = ld16(base + from[j0 + j]);
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j0 + j < m && from[j0 + j] != to[j0 + j]) st16(base + to[j0 + j], x[j]);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicInc((unsigned*)c.sc_ticket() + b, gridDim.x - 1) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    const int held = c.held_of(s), keep = (len + n + (1 << c.page_shift) - 1) >> c.page_shift;
    for (int j = keep + threadIdx.x; j < held; j += blockDim.x) {
        int* t = c.table + (long long)s * c.max_pages + j;
        if (c.page_ok(*t)) atomicAdd(c.refs + *t, -1);
        *t = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0) { c.length[s] = len + n; c.held[s] = min(held, keep); }
}

// fork, 1 of 2: one CTA a pair.  The source's table as it is now; references of the pages that will be shared and, until the copy is done, of the page to be copied
// (so that nobody is given it); the destination's old pages lose theirs.  The CTA that is through last gives a new page to each pair that copies one.
__global__ void __launch_bounds__(CP_ALLOC_THREADS) k_fork_take(Cache c, const int* src, const int* dst) {
    __shared__ int warp_sums[32];
    __shared__ int s_last;
    op_begin();
    const int i = blockIdx.x, n = gridDim.x, s = src[i], d = dst[i];
    int* pair = c.sc_pair() + 2 * i;
    if (!c.seq_ok(s) || !c.seq_ok(d) || s == d) {
        if (threadIdx.x == 0) { pair[0] = -1; if (s != d || !c.seq_ok(s)) atomicOr(c.status, SPECDEC_CACHE_BAD_INDEX); }
    } else {
        const int pt = 1 << c.page_shift, len = min(max(c.length[s], 0), c.held_of(s) << c.page_shift), used = (len + pt - 1) / pt;
        for (int j = threadIdx.x; j < used; j += blockDim.x) {
            const int p = c.table[(long long)s * c.max_pages + j];
            c.sc_rows()[(long long)i * c.max_pages + j] = p;
            if (c.page_ok(p)) atomicAdd(c.refs + p, 1);
        }
        for (int j = threadIdx.x; j < c.held_of(d); j += blockDim.x) {
            const int p = c.table[(long long)d * c.max_pages + j];
            if (c.page_ok(p)) atomicAdd(c.refs + p, -1);
        }
        if (threadIdx.x == 0) { pair[0] = len; pair[1] = (len & (pt - 1)) != 0; }
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicInc((unsigned*)c.sc_ticket(), n - 1) == (unsigned)n - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    int run = 0;
    for (int i0 = 0; i0 < n; i0 += CP_ALLOC_THREADS) {
        const int j = i0 + threadIdx.x;
        int total;
        const int need = j < n && __ldcg(c.sc_pair() + 2 * j) >= 0 ? __ldcg(c.sc_pair() + 2 * j + 1) : 0;
        const int upto = cta_scan(need, warp_sums, &total);
        if (j < n) c.sc_first()[j] = run + upto - need;
        run += total;
    }
    const bool ok = find_pages(c, run, warp_sums);
    if (ok) for (int r = threadIdx.x; r < run; r += CP_ALLOC_THREADS) c.refs[c.sc_pages()[r]] = 1;
    if (threadIdx.x == 0) { *c.sc_ok() = ok; if (!ok) atomicOr(c.status, SPECDEC_CACHE_NO_PAGES); }
}
// 2 of 2: CTAs (share of the copy, pair) copy the tokens of the last page; the first of a pair writes its table.  Without pages the first
// part is undone.  CONTIG: a page's tokens are one stretch of memory.
template <bool CONTIG>
__global__ void __launch_bounds__(256) k_fork_copy(Cache c, const int* dst, int sides, int splits) {
    op_begin();
    const int i = blockIdx.y, d = dst[i], len = c.sc_pair()[2 * i];
    if (len < 0) return;
    const bool ok = *c.sc_ok();
    const int pt = 1 << c.page_shift, full = len >> c.page_shift, part = len & (pt - 1), used = full + (part != 0);
    const int* row = c.sc_rows() + (long long)i * c.max_pages;
    const int page = ok && part ? c.sc_pages()[c.sc_first()[i]] : -1;
    const int from = part ? row[full] : -1;
    if (ok && part && c.page_ok(from)) {
        const int side = blockIdx.x / splits, split = blockIdx.x % splits;
        char* base = c.kv + (side >> 1) * c.s_layer + (side & 1) * c.s_side;
        const char* a = base + from * c.s_page;
        char* b = base + page * c.s_page;
        const int per = c.heads * c.chunks, all = part * per;
        const int lo = (int)((long long)all * split / splits), hi = (int)((long long)all * (split + 1) / splits);
        auto at = [&](int u) -> long long {
            if (CONTIG) return (long long)u * 16;
            const int t = u / per, r = u - t * per, h = r / c.chunks;
            return t * c.s_token + h * c.s_head + (r - h * c.chunks) * 16;
        };
        for (int u0 = lo + threadIdx.x; u0 < hi; u0 += 4 * 256) {
            int4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) if (u0 + j * 256 < hi) x[j] = ld16(a + at(u0 + j * 256));
#pragma unroll
            for (int j = 0; j < 4; ++j) if (u0 + j * 256 < hi) st16(b + at(u0 + j * 256), x[j]);
        }
    }
    if (blockIdx.x) return;
    int* table = c.table + (long long)d * c.max_pages;
    const int held = c.held_of(d);
    if (!ok) {
        for (int j = threadIdx.x; j < used; j += blockDim.x) if (c.page_ok(row[j])) atomicAdd(c.refs + row[j], -1);
        for (int j = threadIdx.x; j < held; j += blockDim.x) if (c.page_ok(table[j])) atomicAdd(c.refs + table[j], 1);
        return;
    }
    __syncthreads();                                      // every thread has read held[d]
    for (int j = threadIdx.x; j < max(used, held); j += blockDim.x) table[j] = j < full ? row[j] : j < used ? page : -1;
    if (threadIdx.x == 0) {
        c.length[d] = len;
        c.held[d] = used;
        if (part && c.page_ok(from)) atomicAdd(c.refs + from, -1);
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The cache as the kernels take it; a message if it is none.
const char* view(const specdec_cache* c, Cache& v) {
    if (!c || !c->d_kv || !c->d_table || !c->d_length || !c->d_held || !c->d_refs || !c->d_status || !c->d_scratch) return "a pointer is NULL";
    const int e = op_elem_bytes(c->dtype);
    if (!e) return "unknown dtype";
    if (c->n_layers < 1 || c->n_heads < 1 || c->head_dim < 1 || c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1) return "a size is below 1";
    if (c->page_tokens < 1 || (c->page_tokens & (c->page_tokens - 1))) return "page_tokens is not a power of two";
    if ((long long)c->max_pages * c->page_tokens > 0x7fffffffLL - 65536) return "a sequence could pass 2^31 tokens";
    const long long st[5] = {op_stride(c->stride_layer, c->n_layers), c->stride_side, op_stride(c->stride_page, c->n_pages), op_stride(c->stride_token, c->page_tokens),
                             op_stride(c->stride_head, c->n_heads)};
    if (!aligned16(c->d_kv) || (long long)c->head_dim * e % 16) return "d_kv or head_dim is not a multiple of 16 bytes";
    for (long long s : st) if (s < 0 || s * e % 16) return "a stride is negative or not a multiple of 16 bytes";
    v.kv = (char*)c->d_kv;
    v.table = c->d_table; v.length = c->d_length; v.held = c->d_held; v.refs = c->d_refs; v.status = c->d_status; v.scratch = c->d_scratch;
    v.s_layer = st[0] * e; v.s_side = st[1] * e; v.s_page = st[2] * e; v.s_token = st[3] * e; v.s_head = st[4] * e;
    v.n_pages = c->n_pages; v.n_seqs = c->n_seqs; v.max_pages = c->max_pages;
    v.page_shift = __builtin_ctz(c->page_tokens);
    v.heads = c->n_heads; v.chunks = c->head_dim * e / 16;
    if (v.heads == 1 || v.s_head == v.chunks * 16LL) { v.chunks *= v.heads; v.heads = 1; }
    return nullptr;
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_cache_scratch(int n_seqs, int max_pages, int n_pages) {
    if (n_seqs < 1 || max_pages < 1 || n_pages < 1) return op_bad("cache_scratch", "a size is below 1");
    return 16 + 4LL * n_seqs + n_pages + (long long)n_seqs * max_pages;
}

int specdec_cache_reserve(const specdec_cache* c, const int32_t* d_seqs, int n, int n_tokens, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad("cache_reserve", why);
    if ((n && !d_seqs) || n < 0 || n > c->n_seqs || n_tokens < 0) return op_bad("cache_reserve", "d_seqs is NULL, n not in 0..n_seqs or n_tokens negative");
    if (n == 0) return SPECDEC_OK;
    return op_done("cache_reserve", op_launch(k_cache_reserve, dim3(1), CP_ALLOC_THREADS, 0, (cudaStream_t)stream, 1, v, d_seqs, n, n_tokens));
}

int specdec_cache_release(const specdec_cache* c, const int32_t* d_seqs, int n, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad("cache_release", why);
    if ((n && !d_seqs) || n < 0 || n > c->n_seqs) return op_bad("cache_release", "d_seqs is NULL or n not in 0..n_seqs");
    if (n == 0) return SPECDEC_OK;
    return op_done("cache_release", op_launch(k_cache_release, dim3(n), 256, 0, (cudaStream_t)stream, 1, v, d_seqs));
}

int specdec_cache_append(const specdec_cache* c, const int32_t* d_seqs, int n, int layer, int n_layers, const void* d_k, const void* d_v, int T,
                         long long stride_layer, long long stride_seq, long long stride_token, long long stride_head,
                         const int32_t* d_count, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad("cache_append", why);
    const int e = op_elem_bytes(c->dtype);
    if ((n && T && (!d_seqs || !d_k || !d_v)) || n < 0 || n > c->n_seqs || n > 65535 || T < 0 || layer < 0 || n_layers < 1 || n_layers > 65535 || layer > c->n_layers - n_layers)
        return op_bad("cache_append", "a pointer is NULL, or n, T or the layers are out of range");
    const long long st[4] = {op_stride(stride_layer, n_layers), op_stride(stride_seq, n), op_stride(stride_token, T), op_stride(stride_head, c->n_heads)};
    for (long long s : st) if (s * e % 16) return op_bad("cache_append", "a stride is not a multiple of 16 bytes");
    if (!aligned16(d_k) || !aligned16(d_v)) return op_bad("cache_append", "d_k or d_v is not 16-byte aligned");
    if (n == 0 || T == 0) return SPECDEC_OK;
    AppendArgs a{(const char*)d_k, (const char*)d_v, st[0] * e, st[1] * e, st[2] * e, st[3] * e, d_seqs, d_count, layer, T, c->n_heads, c->head_dim * e / 16, v.s_head};
    if (v.heads == 1 && (c->n_heads == 1 || a.s_head == a.chunks * 16LL)) { a.chunks *= a.heads; a.heads = 1; }
    const int all = a.heads * a.chunks, threads = all <= 32 ? 32 : all <= 64 ? 64 : all <= 128 ? 128 : 256;
    return op_done("cache_append", op_launch(k_cache_append, dim3(T, n, n_layers), threads, 0, (cudaStream_t)stream, 1, v, a));
}

int specdec_cache_compact(const specdec_cache* c, const int32_t* d_seqs, int n, const int32_t* d_path, int path_stride,
                          const int32_t* d_n_path, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad("cache_compact", why);
    if ((n && (!d_seqs || !d_path || !d_n_path)) || n < 0 || n > c->n_seqs || n > 65535 || path_stride < 1)
        return op_bad("cache_compact", "a pointer is NULL, n not in 0..n_seqs or path_stride below 1");
    if (n == 0) return SPECDEC_OK;
    const int sides = 2 * c->n_layers;
    const long long ctas = ((long long)sides * v.heads * v.chunks + 127) / 128;
    return op_done("cache_compact", op_launch(k_cache_compact, dim3((unsigned)(ctas < 1024 ? ctas : 1024), n), 128, 0, (cudaStream_t)stream, 1, v, d_seqs, d_path, path_stride, d_n_path, sides));
}

int specdec_cache_fork(const specdec_cache* c, const int32_t* d_src, const int32_t* d_dst, int n, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad("cache_fork", why);
    if ((n && (!d_src || !d_dst)) || n < 0 || n > c->n_seqs || n > 65535) return op_bad("cache_fork", "a pointer is NULL or n not in 0..n_seqs");
    if (n == 0) return SPECDEC_OK;
    const cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = op_launch(k_fork_take, dim3(n), CP_ALLOC_THREADS, 0, st, 1, v, d_src, d_dst);
    if (e != cudaSuccess) return op_done("cache_fork", e);
    const int sides = 2 * c->n_layers;
    const long long most = (long long)c->page_tokens * v.heads * v.chunks;             // pieces of a side's page
    const int splits = most <= 4096 ? 1 : most >= 32768 ? 8 : (int)(most / 4096);
    const bool contig = v.heads == 1 && v.s_token == v.chunks * 16LL;
    return op_done("cache_fork", op_launch(contig ? k_fork_copy<true> : k_fork_copy<false>, dim3(sides * splits, n), 256, 0, st, 1, v, d_dst, sides, splits));
}

}  // extern "C"
