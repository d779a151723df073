// Attention of drafted trees over the caller's paged cache: what its kernels share (contract: specdec.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "op_error.cuh"

namespace sd {

// Rows of one K/V head: query row r = t * group + (head within the group), cut into tiles of a kernel's ROWS; the keys of a sequence are its
// length committed tokens and n nodes behind them, cut into `splits` runs of blocks of TA_BLOCK keys.
constexpr int TA_BLOCK = 64;
struct TreeAttn {
    const char* q; char* out; const char* k; const char* v;
    long long q_sb, q_st, q_sh, o_sb, o_st, o_sh, s_page, s_token, s_head;             // bytes
    const int* table; const int* length; const int* held; const int* seqs; const int* n_nodes;
    const uint32_t* mask; long long mask_sb;                                           // words
    int n_pages, n_seqs, max_pages, page_shift, max_length;
    int T, words, group, kv_heads, dim, B;
    int tiles, splits, min_blocks;                                                     // row tiles; splits at most, and blocks a split takes at least
    float scale;                                                                       // times log2(e)
    float* part; float2* part_ml;                                                      // [b, kv head, tile, split, row]: output [dim] and (maximum, sum)
    int q_vec, out_vec;                                                                // whether q / out allow 16-byte accesses
};

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
// Blocks per split and splits in use for a sequence.
__device__ __forceinline__ int ta_per_split(const TreeAttn& a, int blocks) { return max((blocks + a.splits - 1) / a.splits, a.min_blocks); }
__device__ __forceinline__ int ta_used(const TreeAttn& a, int keys, int& per) {
    const int blocks = (keys + TA_BLOCK - 1) / TA_BLOCK;
    per = ta_per_split(a, blocks);
    return (blocks + per - 1) / per;
}

// What the queries of a row tile see of the nodes: their mask rows, cut at n, in shared memory; and the nodes that any of them sees.
// 32 keys from key k0 on as bits: committed ones all, nodes by the row's words.
__device__ __forceinline__ uint32_t ta_window(const uint32_t* row, int words, int base) {      // base = k0 - length
    if (base <= -32) return 0xffffffffu;
    if (base < 0) return ((1u << -base) - 1u) | (words ? row[0] << -base : 0u);
    const int w = base >> 5, s = base & 31;
    const uint32_t a = w < words ? row[w] : 0u, b = w + 1 < words ? row[w + 1] : 0u;
    return __funnelshift_r(a, b, s);
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

}  // namespace sd
