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

// A warp per node walks to the root once, setting bits in a row that its lanes hold (lane w: word w): as many steps as the node is deep.
__global__ void k_tree_ancestors(const int* __restrict__ parents, const int* __restrict__ n_nodes, int T, uint32_t* __restrict__ mask, int* __restrict__ depth) {
    __shared__ int par[TO_MAX];
    const int b = blockIdx.y, W = (T + 31) / 32, lane = threadIdx.x & 31;
    const int n = min(n_nodes ? n_nodes[b] : T, T);
    const int hi = min((int)(blockIdx.x + 1) * (int)(blockDim.x >> 5), T);             // nodes beyond this CTA's are nobody's ancestors here
    for (int i = threadIdx.x; i < hi; i += blockDim.x) {
        const int p = parents[(long long)b * T + i];
        par[i] = p >= 0 && p < i ? p : -1;
    }
    __syncthreads();
    const int i = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (i >= T) return;
    uint32_t bits = 0;
    int d = -1;
    if (i < n)
        for (int j = i; j >= 0; j = par[j]) {
            if (lane == j >> 5) bits |= 1u << (j & 31);
            ++d;
        }
    if (mask && lane < W) mask[((long long)b * T + i) * W + lane] = bits;
    if (depth && lane == 0) depth[(long long)b * T + i] = d;
}

// Thread i: whether node i is the first child of its parent that carries the parent's sampled token; next[parent] = that child.  The chain from the root is
// then walked by one thread.
__global__ void k_tree_accept(const int* __restrict__ parents, const int* __restrict__ tokens, const int* __restrict__ sampled,
                              const int* __restrict__ n_nodes, int T, int* __restrict__ path, int* __restrict__ n_path, int* __restrict__ emitted) {
    __shared__ int next[TO_MAX], walk[TO_MAX], smp[TO_MAX];
    __shared__ int s_n;
    const int b = blockIdx.x;
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
    const int warps = T < 8 ? T : 8;
    k_tree_ancestors<<<dim3((T + warps - 1) / warps, B), warps * 32, 0, (cudaStream_t)stream>>>(d_parents, d_n_nodes, T, d_mask, d_depth);
    return op_launched("tree_ancestors");
}

int specdec_tree_accept(const int32_t* d_parents, const int32_t* d_tokens, const int32_t* d_sampled, const int32_t* d_n_nodes, int B, int T,
                        int32_t* d_path, int32_t* d_n_path, int32_t* d_emitted, void* stream) {
    if (int rc = check("tree_accept", B, T, d_parents && d_tokens && d_sampled && d_path && d_n_path && d_emitted)) return rc;
    if (B == 0) return SPECDEC_OK;
    const int threads = T <= 64 ? 64 : T <= 256 ? 128 : 256;
    k_tree_accept<<<B, threads, 0, (cudaStream_t)stream>>>(d_parents, d_tokens, d_sampled, d_n_nodes, T, d_path, d_n_path, d_emitted);
    return op_launched("tree_accept");
}

}  // extern "C"
