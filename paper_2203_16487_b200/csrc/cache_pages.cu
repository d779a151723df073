// Pages of a K/V cache in the caller's memory, of 16- or 32-bit elements or of 4-bit codes and their scales: reserve, append, compact, release, fork, reorder (contract: specdec.h).
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

#include "fp4.cuh"
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
    char* sc;                                             // 4 bits: the scales, strides in bytes, a token and head's in 4-byte pieces
    long long c_layer, c_side, c_page, c_token, c_head;
    int c_heads, c_chunks;
    __device__ __forceinline__ bool seq_ok(int s) const { return (unsigned)s < (unsigned)n_seqs; }
    __device__ __forceinline__ bool page_ok(int p) const { return (unsigned)p < (unsigned)n_pages; }
    __device__ __forceinline__ int held_of(int s) const { return min(max(held[s], 0), max_pages); }
    // scratch: [0] whether the call got its pages, then per entry of the call the rank of its first new page, [n_pages] the pages given
    // out, per sequence the tickets of compact; fork, reorder: per pair length and whether its last page is copied (or goes on), and the sources' tables; reorder: the entries
    // that copy
    __device__ __forceinline__ int* sc_ok() const { return scratch; }
    __device__ __forceinline__ int* sc_first() const { return scratch + 16; }
    __device__ __forceinline__ int* sc_pages() const { return scratch + 16 + n_seqs; }
    __device__ __forceinline__ int* sc_ticket() const { return scratch + 16 + n_seqs + n_pages; }
    __device__ __forceinline__ int* sc_pair() const { return scratch + 16 + 2 * n_seqs + n_pages; }
    __device__ __forceinline__ int* sc_jobs() const { return scratch + 16 + 4 * n_seqs + n_pages; }
    __device__ __forceinline__ int* sc_rows() const { return scratch + 16 + 5 * n_seqs + n_pages; }
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

// Where slot `pos` of sequence s is, or -1 where that is no page of the sequence's own: bytes from the side's begin, or (FP4) the slot's number among all pages' slots.
template <bool FP4 = false>
__device__ __forceinline__ long long own_slot(const Cache& c, int s, int pos) {
    const int i = pos >> c.page_shift;
    if (pos < 0 || i >= c.held_of(s)) return -1;
    const int p = c.table[(long long)s * c.max_pages + i];
    if (!c.page_ok(p) || c.refs[p] != 1) return -1;
    const int t = pos & ((1 << c.page_shift) - 1);
    return FP4 ? ((long long)p << c.page_shift) + t : p * c.s_page + t * c.s_token;
}
// Bytes from a side's begin to slot `slot` of the codes, and of the scales.
__device__ __forceinline__ long long code_at(const Cache& c, long long slot) { return (slot >> c.page_shift) * c.s_page + (slot & ((1 << c.page_shift) - 1)) * c.s_token; }
__device__ __forceinline__ long long scale_at(const Cache& c, long long slot) { return (slot >> c.page_shift) * c.c_page + (slot & ((1 << c.page_shift) - 1)) * c.c_token; }

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
template <bool FP4>
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
            const long long f = own_slot<FP4>(c, s, len + x), t = own_slot<FP4>(c, s, len + j);
            if (f < 0 || t < 0) bad = SPECDEC_CACHE_UNRESERVED;
            if (j < CC_PATH) { from[j] = f; to[j] = t; }
        }
    const bool index = __syncthreads_or(bad & SPECDEC_CACHE_BAD_INDEX), slot = __syncthreads_or(bad & SPECDEC_CACHE_UNRESERVED);
    if (index || slot) { if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(c.status, index ? SPECDEC_CACHE_BAD_INDEX : SPECDEC_CACHE_UNRESERVED); return; }
    const int codes = c.heads * c.chunks, per = codes + (FP4 ? c.c_heads * c.c_chunks : 0);
    for (int n0 = 0; n0 < n; n0 += CC_PATH) {
        const int m = min(n - n0, CC_PATH);
        if (n0) {
            __syncthreads();                              // the last ones' addresses have been used
            for (int j = threadIdx.x; j < m; j += blockDim.x) { from[j] = own_slot<FP4>(c, s, len + pa[n0 + j]); to[j] = own_slot<FP4>(c, s, len + n0 + j); }
            __syncthreads();
        }
        auto move = [&](auto piece, char* base, auto at) {
            for (int j0 = 0; j0 < m; j0 += 8) {
                decltype(piece) x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j0 + j < m) x[j] = *reinterpret_cast<const decltype(piece)*>(base + at(from[j0 + j]));
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j0 + j < m && from[j0 + j] != to[j0 + j]) *reinterpret_cast<decltype(piece)*>(base + at(to[j0 + j])) = x[j];
            }
        };
        for (long long u = (long long)blockIdx.x * blockDim.x + threadIdx.x; u < (long long)sides * per; u += (long long)gridDim.x * blockDim.x) {
            const int side = (int)(u / per), r = (int)(u % per);
            if (FP4 && r >= codes) {                      // a piece of the scales
                const int x = r - codes, h = x / c.c_chunks;
                move(0, c.sc + (side >> 1) * c.c_layer + (side & 1) * c.c_side + h * c.c_head + (x - h * c.c_chunks) * 4, [&](long long slot) { return scale_at(c, slot); });
                continue;
            }
            const int h = c.heads == 1 ? 0 : r / c.chunks;
            move(int4(), c.kv + (side >> 1) * c.s_layer + (side & 1) * c.s_side + h * c.s_head + (r - h * c.chunks) * 16, [&](long long slot) { return FP4 ? code_at(c, slot) : slot; });
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

// A page's share of a copy, by a CTA of 256: the pieces [lo, hi) of a layer and side, of `per` pieces a token, four of a thread's on their way at a time.
template <typename P, typename At>
__device__ __forceinline__ void copy_pieces(const char* a, char* b, int lo, int hi, At at) {
    for (int u0 = lo + threadIdx.x; u0 < hi; u0 += 4 * 256) {
        P x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) if (u0 + j * 256 < hi) x[j] = *reinterpret_cast<const P*>(a + at(u0 + j * 256));
#pragma unroll
        for (int j = 0; j < 4; ++j) if (u0 + j * 256 < hi) *reinterpret_cast<P*>(b + at(u0 + j * 256)) = x[j];
    }
}
// How a page lies: whole (its tokens are one stretch of memory), by token and head, or in 4 bits (a head's tokens are one stretch of codes and one of scales).
enum { PAGE_WHOLE, PAGE_ROWS, PAGE_FP4 };
// Part `split` of `splits` of the first `part` tokens of one layer and side, page `from` to page `to`.
template <int LIES>
__device__ __forceinline__ void copy_part(const Cache& c, int side, int from, int to, int part, int split, int splits) {
    auto share = [&](long long all, int i) { return (int)(all * i / splits); };
    char* base = c.kv + (side >> 1) * c.s_layer + (side & 1) * c.s_side;
    const int per = c.heads * c.chunks, all = part * per;
    copy_pieces<int4>(base + from * c.s_page, base + to * c.s_page, share(all, split), share(all, split + 1), [&](int u) -> long long {
        if (LIES == PAGE_WHOLE) return (long long)u * 16;
        if (LIES == PAGE_FP4) { const int row = part * c.chunks, h = u / row; return h * c.s_head + (u - h * row) * 16LL; }
        const int t = u / per, r = u - t * per, h = r / c.chunks;
        return t * c.s_token + h * c.s_head + (r - h * c.chunks) * 16;
    });
    if constexpr (LIES == PAGE_FP4) {
        char* scales = c.sc + (side >> 1) * c.c_layer + (side & 1) * c.c_side;
        const int row = part * c.c_chunks, n = c.c_heads * row;
        copy_pieces<int>(scales + from * c.c_page, scales + to * c.c_page, share(n, split), share(n, split + 1), [&](int u) -> long long { const int h = u / row; return h * c.c_head + (u - h * row) * 4LL; });
    }
}

// 2 of 2: CTAs (share of the copy, pair) copy the tokens of the last page; the first of a pair writes its table.  Without pages the first
// part is undone.
template <int LIES>
__global__ void __launch_bounds__(256) k_fork_copy(Cache c, const int* dst, int sides, int splits) {
    op_begin();
    const int i = blockIdx.y, d = dst[i], len = c.sc_pair()[2 * i];
    if (len < 0) return;
    const bool ok = *c.sc_ok();
    const int pt = 1 << c.page_shift, full = len >> c.page_shift, part = len & (pt - 1), used = full + (part != 0);
    const int* row = c.sc_rows() + (long long)i * c.max_pages;
    const int page = ok && part ? c.sc_pages()[c.sc_first()[i]] : -1;
    const int from = part ? row[full] : -1;
    if (ok && part && c.page_ok(from)) copy_part<LIES>(c, blockIdx.x / splits, from, page, part, blockIdx.x % splits, splits);
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

// reorder.  Entries are the beams of groups of `beams` sequences; entry i's parent is the entry of its group that parents[i] names, itself where that, or a sequence number, is none
// (BAD_INDEX), nobody where parents[i] is -1.
struct Beams { const int* seqs; const int* parents; int n, beams; };
constexpr int NOBODY = -1, NO_ENTRY = -2;                 // no parent: pages given back; no such sequence: nothing is done
__device__ __forceinline__ int parent_of(const Cache& c, const Beams& b, int i, bool* bad = nullptr) {
    if (!c.seq_ok(b.seqs[i])) { if (bad) *bad = true; return NO_ENTRY; }
    const int p = b.parents[i], g = i - i % b.beams;
    if (p == -1) return NOBODY;
    if (p < 0 || p >= b.beams || !c.seq_ok(b.seqs[g + p])) { if (bad) *bad = true; return i; }
    return g + p;
}
__device__ __forceinline__ int committed(const Cache& c, int s) { return min(max(c.length[s], 0), c.held_of(s) << c.page_shift); }

// 1 of 2: one CTA an entry.  References move from the sequence's old pages to its parent's, whose table is noted.  A parent's last, partly filled page goes on with one child (the parent
// itself if it is one, else the first), the others copy it to pages that the CTA that is through last gives out: those of beams that nobody continues are free by then.
__global__ void __launch_bounds__(CP_ALLOC_THREADS) k_reorder_take(Cache c, Beams b) {
    __shared__ int warp_sums[32];
    __shared__ int s_last;
    op_begin();
    const int i = blockIdx.x;
    bool bad = false;
    const int p = parent_of(c, b, i, &bad), pt = 1 << c.page_shift;
    int* pair = c.sc_pair() + 2 * i;                      // tokens (-1: nothing to do), whether the last page is copied
    if (bad && threadIdx.x == 0) atomicOr(c.status, SPECDEC_CACHE_BAD_INDEX);
    if (p == NO_ENTRY) {
        if (threadIdx.x == 0) { pair[0] = -1; pair[1] = 0; }
    } else {
        const int d = b.seqs[i], len = p == NOBODY ? 0 : committed(c, b.seqs[p]), full = len >> c.page_shift, used = full + ((len & (pt - 1)) != 0);
        bool first = true;                                // of p's children
        if (p >= 0 && p != i) {
            const int g = i - i % b.beams;
            bool mine = true;
            for (int j = g + threadIdx.x; j < g + b.beams; j += blockDim.x)
                if ((j < i || j == p) && parent_of(c, b, j) == p) mine = false;
            first = __syncthreads_and(mine);
        }
        const bool copies = used > full && !first;
        if (p != i) {
            const int s = p == NOBODY ? d : b.seqs[p], take = copies ? full : used;
            for (int j = threadIdx.x; j < used; j += blockDim.x) {
                const int x = c.table[(long long)s * c.max_pages + j];
                c.sc_rows()[(long long)i * c.max_pages + j] = x;
                if (j < take && c.page_ok(x)) atomicAdd(c.refs + x, 1);
            }
        }
        for (int j = (p == i ? used : 0) + threadIdx.x; j < c.held_of(d); j += blockDim.x) {
            const int x = c.table[(long long)d * c.max_pages + j];
            if (c.page_ok(x)) atomicAdd(c.refs + x, -1);
        }
        if (threadIdx.x == 0) { pair[0] = len; pair[1] = copies; }
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicInc((unsigned*)c.sc_ticket(), b.n - 1) == (unsigned)b.n - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    int run = 0;
    for (int i0 = 0; i0 < b.n; i0 += CP_ALLOC_THREADS) {
        const int j = i0 + threadIdx.x;
        int total;
        const int need = j < b.n ? __ldcg(c.sc_pair() + 2 * j + 1) : 0;
        const int upto = cta_scan(need, warp_sums, &total);
        if (j < b.n) c.sc_first()[j] = run + upto - need;
        if (need) c.sc_jobs()[run + upto - need] = j;
        run += total;
    }
    const bool ok = find_pages(c, run, warp_sums);
    if (ok) for (int r = threadIdx.x; r < run; r += CP_ALLOC_THREADS) c.refs[c.sc_pages()[r]] = 1;
    if (threadIdx.x == 0) { c.sc_ok()[0] = ok; c.sc_ok()[1] = ok ? run : 0; if (!ok) atomicOr(c.status, SPECDEC_CACHE_NO_PAGES); }
}
constexpr int REORDER_ONE = 160 * 1024;
// ... where counts and tables fit into the shared memory of one CTA: everything but the copies.  Nothing is written until it is known that there are pages enough.
__global__ void __launch_bounds__(CP_ALLOC_THREADS) k_reorder_one(Cache c, Beams b) {
    extern __shared__ int one_smem[];
    __shared__ int warp_sums[32], s_seq[CP_ALLOC_THREADS], s_held[CP_ALLOC_THREADS], s_len[CP_ALLOC_THREADS], s_up[CP_ALLOC_THREADS], s_used[CP_ALLOC_THREADS], s_full[CP_ALLOC_THREADS],
        s_new[CP_ALLOC_THREADS];                          // (n <= 1024) up: as parent_of has it; full: place of the page that is copied, -1: none; new: the pages given out
    int* refs = one_smem;
    int* rows = refs + c.n_pages;                         // [n][max_pages]: the tables as they were
    op_begin();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, pt = 1 << c.page_shift, cells = b.n * c.max_pages;
    bool bad = false;
    if (tid < b.n) {
        s_up[tid] = parent_of(c, b, tid, &bad);
        const int s = b.seqs[tid];
        s_seq[tid] = s;
        s_held[tid] = 0;
        if (c.seq_ok(s)) { s_held[tid] = c.held_of(s); s_len[tid] = committed(c, s); }
    }
#pragma unroll 4
    for (int p = tid; p < c.n_pages; p += CP_ALLOC_THREADS) refs[p] = c.refs[p];
    if (__syncthreads_or(bad) && tid == 0) atomicOr(c.status, SPECDEC_CACHE_BAD_INDEX);
#pragma unroll 4
    for (int x = tid; x < cells; x += CP_ALLOC_THREADS) {
        const int i = x / c.max_pages, j = x - i * c.max_pages;
        rows[x] = j < s_held[i] ? c.table[(long long)s_seq[i] * c.max_pages + j] : -1;
    }
    int copy = 0;                                         // whether entry tid copies its parent's last page
    if (tid < b.n) {
        const int p = s_up[tid], len = p >= 0 ? s_len[p] : 0, g = tid - tid % b.beams;
        bool first = true;
        if (p >= 0 && p != tid) for (int j = g; j < g + b.beams; ++j) first &= !((j < tid || j == p) && s_up[j] == p);
        copy = (len & (pt - 1)) && !first;
        s_used[tid] = (len + pt - 1) >> c.page_shift;
        s_full[tid] = copy ? len >> c.page_shift : -1;
    }
    __syncthreads();
    for (int x = tid; x < cells; x += CP_ALLOC_THREADS) { // references: from the old pages to the parent's
        const int i = x / c.max_pages, j = x - i * c.max_pages, p = s_up[i];
        if (p == NO_ENTRY) continue;
        if (j < s_held[i] && (p != i || j >= s_used[i]) && c.page_ok(rows[x])) atomicAdd(refs + rows[x], -1);
        if (p >= 0 && p != i && j < s_used[i] && j != s_full[i]) { const int y = rows[p * c.max_pages + j]; if (c.page_ok(y)) atomicAdd(refs + y, 1); }
    }
    __syncthreads();
    // The lowest free pages: each warp counts, then lists, those of its own stretch.  One scan for both counts: copies, and (lane 0) free pages.
    const int per = ((c.n_pages + 31) / 32 + 31) / 32 * 32, lo = min(warp * per, c.n_pages), hi = min(lo + per, c.n_pages);
    int n = 0;
    for (int p = lo + lane; p < hi; p += 32) n += refs[p] == 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    int all;
    const int upto = cta_scan(copy << 20 | (lane == 0 ? n : 0), warp_sums, &all);
    const int total = all >> 20, rank = (upto >> 20) - copy, free_pages = all & 0xfffff;
    const bool ok = free_pages >= total;
    if (tid == 0) { c.sc_ok()[1] = ok ? total : 0; if (!ok) atomicOr(c.status, SPECDEC_CACHE_NO_PAGES); }
    if (!ok) return;
    int at = (__shfl_sync(0xffffffffu, upto, 0) & 0xfffff) - n;
    for (int p0 = lo; p0 < hi && at < total; p0 += 32) {
        const int p = p0 + lane;
        const bool f = p < hi && refs[p] == 0;
        const unsigned m = __ballot_sync(0xffffffffu, f);
        const int r = at + __popc(m & ((1u << lane) - 1));
        if (f && r < total) { c.sc_pages()[r] = p; s_new[r] = p; refs[p] = 1; }
        at += __popc(m);
    }
    __syncthreads();
    if (copy) {                                           // entry tid's new page, and what is copied to it
        const int p = s_up[tid];
        c.sc_pair()[2 * rank] = rows[p * c.max_pages + s_full[tid]]; c.sc_pair()[2 * rank + 1] = s_len[p] & (pt - 1);
        c.table[(long long)s_seq[tid] * c.max_pages + s_full[tid]] = s_new[rank];
    }
    for (int p = tid; p < c.n_pages; p += CP_ALLOC_THREADS) c.refs[p] = refs[p];
    if (tid < b.n && s_up[tid] != NO_ENTRY) { c.held[s_seq[tid]] = s_used[tid]; c.length[s_seq[tid]] = s_up[tid] == NOBODY ? 0 : s_len[s_up[tid]]; }
    for (int x = tid; x < cells; x += CP_ALLOC_THREADS) { // the tables
        const int i = x / c.max_pages, j = x - i * c.max_pages, p = s_up[i], used = s_used[i];
        if (p == NO_ENTRY || j == s_full[i] || j >= max(used, s_held[i]) || (p == i && j < used)) continue;
        c.table[(long long)s_seq[i] * c.max_pages + j] = j < used ? rows[p * c.max_pages + j] : -1;
    }
}

// 2 of 2: CTAs that stay.  The entries' tables (without pages: the references undone), unless k_reorder_one has written them; then copies, 256 pieces (4 KB) of a layer and side, of 4 bits
// of one head, a warp.
template <int LIES, bool ONE>
__global__ void __launch_bounds__(256, 4) k_reorder_copy(Cache c, Beams b, int sides) {
    op_begin();
    const int jobs = c.sc_ok()[1], pt = 1 << c.page_shift;
    if constexpr (!ONE) {
        const bool ok = c.sc_ok()[0];
        for (int i = blockIdx.x; i < b.n; i += gridDim.x) {
            const int len = c.sc_pair()[2 * i];
            if (len < 0) continue;
            const int d = b.seqs[i], full = len >> c.page_shift, used = full + ((len & (pt - 1)) != 0), held = c.held_of(d), p = parent_of(c, b, i);
            const bool copies = c.sc_pair()[2 * i + 1];
            const int* row = c.sc_rows() + (long long)i * c.max_pages;
            int* table = c.table + (long long)d * c.max_pages;
            if (!ok) {
                if (p != i) for (int j = threadIdx.x; j < (copies ? full : used); j += blockDim.x) if (c.page_ok(row[j])) atomicAdd(c.refs + row[j], -1);
                for (int j = (p == i ? used : 0) + threadIdx.x; j < held; j += blockDim.x) if (c.page_ok(table[j])) atomicAdd(c.refs + table[j], 1);
                continue;
            }
            const int page = copies ? c.sc_pages()[c.sc_first()[i]] : -1;
            __syncthreads();                              // every thread has read held[d]
            for (int j = (p == i ? used : 0) + threadIdx.x; j < max(used, held); j += blockDim.x) table[j] = j >= used ? -1 : j == full && copies ? page : row[j];
            if (threadIdx.x == 0) { c.length[d] = len; c.held[d] = used; }
        }
    }
    const int segments = LIES == PAGE_FP4 ? c.heads : 1, per = LIES == PAGE_FP4 ? c.chunks : c.heads * c.chunks, shares = (pt * per + 255) / 256, a_job = sides * segments * shares;
    const long long all = (long long)jobs * a_job;
    for (long long w = blockIdx.x * 8 + (threadIdx.x >> 5); w < all; w += gridDim.x * 8) {
        const int job = (int)(w / a_job), r = (int)(w - (long long)job * a_job), share = r % shares, q = r / shares, h = q % segments, side = q / segments;
        int from, part;
        if (ONE) { from = c.sc_pair()[2 * job]; part = c.sc_pair()[2 * job + 1]; }
        else {
            const int i = c.sc_jobs()[job], len = c.sc_pair()[2 * i];
            from = c.sc_rows()[(long long)i * c.max_pages + (len >> c.page_shift)]; part = len & (pt - 1);
        }
        const int to = c.sc_pages()[job];
        if (!c.page_ok(from) || share * 256 >= part * per) continue;
        // eight pieces of a lane and (4 bits) four of scales, all read before the first is written
        char* base = c.kv + (side >> 1) * c.s_layer + (side & 1) * c.s_side + (LIES == PAGE_FP4 ? h * c.s_head : 0);
        const int lane = threadIdx.x & 31, lo = share * 256 + lane, hi = min(part * per, share * 256 + 256);
        auto at = [&](int u) -> long long {
            if (LIES != PAGE_ROWS) return (long long)u * 16;
            const int t = u / per, x = u - t * per, g = x / c.chunks;
            return t * c.s_token + g * c.s_head + (x - g * c.chunks) * 16;
        };
        int4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) if (lo + j * 32 < hi) x[j] = ld16(base + from * c.s_page + at(lo + j * 32));
        if constexpr (LIES == PAGE_FP4) {
            char* scales = c.sc + (side >> 1) * c.c_layer + (side & 1) * c.c_side + h * c.c_head;
            const int s_lo = share * 128 + lane, s_hi = min(part * c.c_chunks, share * 128 + 128);         // (of the tokens whose codes this share has: two scales' pieces for four of codes, or one for two)
            int y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) if (s_lo + j * 32 < s_hi) y[j] = *reinterpret_cast<const int*>(scales + from * c.c_page + (s_lo + j * 32) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) if (s_lo + j * 32 < s_hi) *reinterpret_cast<int*>(scales + to * c.c_page + (s_lo + j * 32) * 4) = y[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) if (lo + j * 32 < hi) st16(base + to * c.s_page + at(lo + j * 32), x[j]);
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
// The same of a cache in 4 bits.
const char* view(const specdec_packed_cache* f, Cache& v) {
    if (const char* why = fp4_why_not(f)) return why;
    const specdec_cache* c = &f->codes;
    if (!c->d_refs || !c->d_held || !c->d_scratch) return "a pointer is NULL";
    v.kv = (char*)c->d_kv; v.sc = (char*)f->d_scales;
    v.table = c->d_table; v.length = c->d_length; v.held = c->d_held; v.refs = c->d_refs; v.status = c->d_status; v.scratch = c->d_scratch;
    v.s_layer = op_stride(c->stride_layer, c->n_layers); v.s_side = c->stride_side; v.s_page = op_stride(c->stride_page, c->n_pages); v.s_token = c->head_dim / 2;
    v.s_head = op_stride(c->stride_head, c->n_heads);
    v.c_layer = op_stride(f->scale_stride_layer, c->n_layers); v.c_side = f->scale_stride_side; v.c_page = op_stride(f->scale_stride_page, c->n_pages); v.c_token = c->head_dim / 16;
    v.c_head = op_stride(f->scale_stride_head, c->n_heads);
    v.n_pages = c->n_pages; v.n_seqs = c->n_seqs; v.max_pages = c->max_pages;
    v.page_shift = __builtin_ctz(c->page_tokens);
    v.heads = v.c_heads = c->n_heads; v.chunks = c->head_dim / 32; v.c_chunks = c->head_dim / 64;
    return nullptr;
}
int lies(const specdec_cache*, const Cache& v) { return v.heads == 1 && v.s_token == v.chunks * 16LL ? PAGE_WHOLE : PAGE_ROWS; }
int lies(const specdec_packed_cache*, const Cache&) { return PAGE_FP4; }
const specdec_cache& sizes(const specdec_cache* c) { return *c; }
const specdec_cache& sizes(const specdec_packed_cache* f) { return f->codes; }
// CTAs that share a layer and side of a page's copy.
int copy_splits(const specdec_cache& c, const Cache& v) {
    const long long most = (long long)c.page_tokens * v.heads * v.chunks;              // pieces of a side's page
    return most <= 4096 ? 1 : most >= 32768 ? 8 : (int)(most / 4096);
}

// The calls, of either cache.
template <typename C> int reserve(const char* who, const C* c, const int32_t* d_seqs, int n, int n_tokens, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad(who, why);
    if ((n && !d_seqs) || n < 0 || n > v.n_seqs || n_tokens < 0) return op_bad(who, "d_seqs is NULL, n not in 0..n_seqs or n_tokens negative");
    if (n == 0) return SPECDEC_OK;
    return op_done(who, op_launch(k_cache_reserve, dim3(1), CP_ALLOC_THREADS, 0, (cudaStream_t)stream, 1, v, d_seqs, n, n_tokens));
}
template <typename C> int release(const char* who, const C* c, const int32_t* d_seqs, int n, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad(who, why);
    if ((n && !d_seqs) || n < 0 || n > v.n_seqs) return op_bad(who, "d_seqs is NULL or n not in 0..n_seqs");
    if (n == 0) return SPECDEC_OK;
    return op_done(who, op_launch(k_cache_release, dim3(n), 256, 0, (cudaStream_t)stream, 1, v, d_seqs));
}
template <bool FP4, typename C>
int compact(const char* who, const C* c, const int32_t* d_seqs, int n, const int32_t* d_path, int path_stride, const int32_t* d_n_path, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad(who, why);
    if ((n && (!d_seqs || !d_path || !d_n_path)) || n < 0 || n > v.n_seqs || n > 65535 || path_stride < 1)
        return op_bad(who, "a pointer is NULL, n not in 0..n_seqs or path_stride below 1");
    if (n == 0) return SPECDEC_OK;
    const int sides = 2 * sizes(c).n_layers;
    const long long ctas = ((long long)sides * (v.heads * v.chunks + (FP4 ? v.c_heads * v.c_chunks : 0)) + 127) / 128;
    return op_done(who, op_launch(k_cache_compact<FP4>, dim3((unsigned)(ctas < 1024 ? ctas : 1024), n), 128, 0, (cudaStream_t)stream, 1, v, d_seqs, d_path, path_stride, d_n_path, sides));
}
template <typename C> int fork(const char* who, const C* c, const int32_t* d_src, const int32_t* d_dst, int n, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad(who, why);
    if ((n && (!d_src || !d_dst)) || n < 0 || n > v.n_seqs || n > 65535) return op_bad(who, "a pointer is NULL or n not in 0..n_seqs");
    if (n == 0) return SPECDEC_OK;
    const cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = op_launch(k_fork_take, dim3(n), CP_ALLOC_THREADS, 0, st, 1, v, d_src, d_dst);
    if (e != cudaSuccess) return op_done(who, e);
    const int sides = 2 * sizes(c).n_layers, splits = copy_splits(sizes(c), v), l = lies(c, v);
    return op_done(who, op_launch(l == PAGE_WHOLE ? k_fork_copy<PAGE_WHOLE> : l == PAGE_ROWS ? k_fork_copy<PAGE_ROWS> : k_fork_copy<PAGE_FP4>, dim3(sides * splits, n), 256, 0, st, 1, v, d_dst,
                                  sides, splits));
}
template <typename C> int reorder(const char* who, const C* c, const int32_t* d_seqs, const int32_t* d_parents, int n, int beams, void* stream) {
    Cache v;
    if (const char* why = view(c, v)) return op_bad(who, why);
    if ((n && (!d_seqs || !d_parents)) || n < 0 || n > v.n_seqs || beams < 1 || n % beams) return op_bad(who, "a pointer is NULL, n not in 0..n_seqs or no multiple of beams, or beams below 1");
    if (n == 0) return SPECDEC_OK;
    const cudaStream_t st = (cudaStream_t)stream;
    const Beams b{d_seqs, d_parents, n, beams};
    const int sides = 2 * sizes(c).n_layers, l = lies(c, v);
    // In one CTA where counts and tables fit its shared memory: with the copies 128 entries of 1400 pages 11.3 us instead of 12.3, 32 entries of 230 15.4 instead of 17.5.
    const long long bytes = 4 * ((long long)v.n_pages + (long long)n * v.max_pages);
    const bool one = n <= CP_ALLOC_THREADS && beams <= 64 && bytes <= REORDER_ONE;      // (at most 40960 pages: counts of 20 bits)
    if (one) if (const cudaError_t e = op_allow<k_reorder_one>(REORDER_ONE)) return op_done(who, e);
    const cudaError_t e = one ? op_launch(k_reorder_one, dim3(1), CP_ALLOC_THREADS, (size_t)bytes, st, 1, v, b) : op_launch(k_reorder_take, dim3(n), CP_ALLOC_THREADS, 0, st, 1, v, b);
    if (e != cudaSuccess) return op_done(who, e);
    const long long pieces = (long long)sizes(c).page_tokens * (l == PAGE_FP4 ? v.chunks : v.heads * v.chunks), items = (long long)n * sides * (l == PAGE_FP4 ? v.heads : 1) * ((pieces + 255) / 256);
    const long long ctas = (items + 7) / 8, most = 4 * 148;                            // (how many copies there are is known on the device)
    auto k = one ? (l == PAGE_WHOLE ? k_reorder_copy<PAGE_WHOLE, true> : l == PAGE_ROWS ? k_reorder_copy<PAGE_ROWS, true> : k_reorder_copy<PAGE_FP4, true>)
                 : l == PAGE_WHOLE ? k_reorder_copy<PAGE_WHOLE, false> : l == PAGE_ROWS ? k_reorder_copy<PAGE_ROWS, false> : k_reorder_copy<PAGE_FP4, false>;
    return op_done(who, op_launch(k, dim3((unsigned)(ctas < most ? ctas : most)), 256, 0, st, 1, v, b, sides));
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

long long specdec_cache_scratch(int n_seqs, int max_pages, int n_pages) {
    if (n_seqs < 1 || max_pages < 1 || n_pages < 1) return op_bad("cache_scratch", "a size is below 1");
    return 16 + 5LL * n_seqs + n_pages + (long long)n_seqs * max_pages;
}

int specdec_cache_reserve(const specdec_cache* c, const int32_t* d_seqs, int n, int n_tokens, void* stream) { return reserve("cache_reserve", c, d_seqs, n, n_tokens, stream); }
int specdec_packed_cache_reserve(const specdec_packed_cache* c, const int32_t* d_seqs, int n, int n_tokens, void* stream) { return reserve("packed_cache_reserve", c, d_seqs, n, n_tokens, stream); }
int specdec_cache_release(const specdec_cache* c, const int32_t* d_seqs, int n, void* stream) { return release("cache_release", c, d_seqs, n, stream); }
int specdec_packed_cache_release(const specdec_packed_cache* c, const int32_t* d_seqs, int n, void* stream) { return release("packed_cache_release", c, d_seqs, n, stream); }
int specdec_cache_compact(const specdec_cache* c, const int32_t* d_seqs, int n, const int32_t* d_path, int path_stride, const int32_t* d_n_path, void* stream) {
    return compact<false>("cache_compact", c, d_seqs, n, d_path, path_stride, d_n_path, stream);
}
int specdec_packed_cache_compact(const specdec_packed_cache* c, const int32_t* d_seqs, int n, const int32_t* d_path, int path_stride, const int32_t* d_n_path, void* stream) {
    return compact<true>("packed_cache_compact", c, d_seqs, n, d_path, path_stride, d_n_path, stream);
}
int specdec_cache_fork(const specdec_cache* c, const int32_t* d_src, const int32_t* d_dst, int n, void* stream) { return sd::fork("cache_fork", c, d_src, d_dst, n, stream); }
int specdec_packed_cache_fork(const specdec_packed_cache* c, const int32_t* d_src, const int32_t* d_dst, int n, void* stream) { return sd::fork("packed_cache_fork", c, d_src, d_dst, n, stream); }
int specdec_cache_reorder(const specdec_cache* c, const int32_t* d_seqs, const int32_t* d_parents, int n, int beams, void* stream) {
    return reorder("cache_reorder", c, d_seqs, d_parents, n, beams, stream);
}
int specdec_packed_cache_reorder(const specdec_packed_cache* c, const int32_t* d_seqs, const int32_t* d_parents, int n, int beams, void* stream) {
    return reorder("packed_cache_reorder", c, d_seqs, d_parents, n, beams, stream);
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

}  // extern "C"
