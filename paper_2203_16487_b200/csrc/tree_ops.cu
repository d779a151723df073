// Trees of drafted tokens: ancestor bits and depths, and the walk along the sampled tokens (contract: specdec.h).
//
// One CTA a tree, everything in shared memory.  Both are chains of dependent look-ups, a few microseconds however small the tree is; what
// bounds them is the latency of the launch and of one read from memory.
#include <cuda_runtime.h>
#include <stdint.h>

#include "op_error.cuh"

namespace sd {
namespace {

constexpr int TO_MAX = 1024;

// One CTA a tree.  Rows of bits in shared memory: node i begins with itself and a pointer to its parent; every round takes over the row that the pointer leads to
// and then that node's pointer, so a chain of d nodes takes log2 d rounds.  (Rows are updated in place: one that is read while it grows holds more ancestors, never
// anything else.)  128 trees of 256 nodes: 6.0 us, a launch by itself some 4; with a warp a node that walks to the root 18.
__global__ void k_tree_ancestors(const int* parents, const int* n_nodes, int T, uint32_t* mask, int* depth) {
    extern __shared__ uint32_t ta_rows[];                 // [T][pitch], then two sets of pointers [T]
    const int b = blockIdx.x, W = (T + 31) / 32, pitch = W | 1;
    volatile uint32_t* rows = ta_rows;
    int* jump = reinterpret_cast<int*>(ta_rows + T * pitch);
    op_begin();
    const int n = max(min(n_nodes ? n_nodes[b] : T, T), 0);
    for (int i = threadIdx.x; i < T; i += blockDim.x) {
        const int p = parents[(long long)b * T + i];
        jump[i] = i < n && p >= 0 && p < i ? p : -1;
        for (int w = 0; w < W; ++w) rows[i * pitch + w] = i < n && w == i >> 5 ? 1u << (i & 31) : 0u;
    }
    bool more = true;
    for (int at = 0; more; at ^= 1) {
        const int* from = jump + at * T;
        int* to = jump + (at ^ 1) * T;
        __syncthreads();
        more = false;
        for (int i = threadIdx.x; i < T; i += blockDim.x) {
            const int p = from[i], q = p < 0 ? -1 : from[p];
            to[i] = q;
            more |= q >= 0;
            if (p >= 0)
#pragma unroll 4
                for (int w = 0; w <= p >> 5; ++w) rows[i * pitch + w] |= rows[p * pitch + w];
        }
        more = __syncthreads_or(more);
    }
    for (int i = threadIdx.x; i < T; i += blockDim.x) {
        int d = -1;
        for (int w = 0; w < W; ++w) {
            const uint32_t x = rows[i * pitch + w];
            d += __popc(x);
            if (mask) mask[((long long)b * T + i) * W + w] = x;
        }
        if (depth) depth[(long long)b * T + i] = d;
    }
}

// Thread i: whether node i is the first child of its parent that carries the parent's sampled token; next[parent] = that child.  The chain from the root is
// then walked by one thread, a read of shared memory a step.  128 trees of 256 nodes: 4.2 us.
__global__ void k_tree_accept(const int* parents, const int* tokens, const int* sampled,
                              const int* n_nodes, int T, int* path, int* n_path, int* emitted) {
    __shared__ int next[TO_MAX], walk[TO_MAX], smp[TO_MAX];
    __shared__ int s_n;
    const int b = blockIdx.x;
    op_begin();
    const long long row = (long long)b * T;
    const int n = max(min(n_nodes ? n_nodes[b] : T, T), 0);
    for (int i = threadIdx.x; i < n; i += blockDim.x) { next[i] = TO_MAX; smp[i] = sampled[row + i]; }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int p = parents[row + i];
        if (p >= 0 && p < i && tokens[row + i] == smp[p]) atomicMin(next + p, i);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int k = 0;
        if (n > 0)
            for (int i = 0; i < TO_MAX; i = next[i]) walk[k++] = i;
        s_n = k;
        n_path[b] = k;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < T; i += blockDim.x) {
        path[row + i] = i < s_n ? walk[i] : -1;
        emitted[row + i] = i < s_n ? smp[walk[i]] : -1;
    }
}

int check(const char* who, int B, int T, bool pointers) {
    if ((B && !pointers) || B < 0 || B > 65535 || T < 1) return op_bad(who, "a pointer is NULL, B not in 0..65535 or T below 1");
    if (T > TO_MAX) return op_fail(SPECDEC_ERR_CAPACITY, who, "trees have at most 1024 nodes");
    return SPECDEC_OK;
}

}  // namespace
}  // namespace sd

using namespace sd;

extern "C" {

int specdec_tree_ancestors(const int32_t* d_parents, const int32_t* d_n_nodes, int B, int T, uint32_t* d_mask, int32_t* d_depth, void* stream) {
    if (int rc = check("tree_ancestors", B, T, d_parents && (d_mask || d_depth))) return rc;
    if (B == 0) return SPECDEC_OK;
    if (const cudaError_t e = op_allow<k_tree_ancestors>(TO_MAX * (TO_MAX / 32 + 1 + 2) * 4)) return op_done("tree_ancestors", e);
    const int threads = T <= 32 ? 32 : T <= 64 ? 64 : T <= 128 ? 128 : 256;
    return op_done("tree_ancestors", op_launch(k_tree_ancestors, dim3(B), threads, (size_t)T * ((((T + 31) / 32) | 1) + 2) * 4, (cudaStream_t)stream, 1, d_parents, d_n_nodes, T, d_mask, d_depth));
}

int specdec_tree_accept(const int32_t* d_parents, const int32_t* d_tokens, const int32_t* d_sampled, const int32_t* d_n_nodes, int B, int T,
                        int32_t* d_path, int32_t* d_n_path, int32_t* d_emitted, void* stream) {
    if (int rc = check("tree_accept", B, T, d_parents && d_tokens && d_sampled && d_path && d_n_path && d_emitted)) return rc;
    if (B == 0) return SPECDEC_OK;
    const int threads = T <= 64 ? 64 : T <= 256 ? 128 : 256;
    return op_done("tree_accept", op_launch(k_tree_accept, dim3(B), threads, 0, (cudaStream_t)stream, 1, d_parents, d_tokens, d_sampled, d_n_nodes, T, d_path, d_n_path, d_emitted));
}

}  // extern "C"
