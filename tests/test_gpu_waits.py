"""A bounded wait that runs out, on a barrier that nothing arrives at: what it leaves in the word that it reports to."""
import os
import subprocess

import pytest

from paper_2203_16487_b200 import build

pytestmark = pytest.mark.gpu

PROGRAM = r"""
#include <cstdio>
#include "barriers.cuh"

template <bool GATHERS> __global__ void k_wait(int* word, int* answer) {
    __shared__ __align__(8) uint64_t bar;
    __shared__ int abort_flag;
    if (threadIdx.x == 0) { sd::mbar_init(sd::smem_u32(&bar), 1); abort_flag = 0; }
    __syncthreads();
    const bool got = sd::mbar_wait_warp<GATHERS>(sd::smem_u32(&bar), 0, &abort_flag, word, 16);
    if (threadIdx.x == 0) *answer = got;
}

int main() {
    int *d, h[2];
    if (cudaMalloc(&d, 8) != cudaSuccess) return 1;
    for (int gathers = 0; gathers < 2; ++gathers) {
        h[0] = 5; h[1] = 7;                              // a word in which something stands already
        cudaMemcpy(d, h, 8, cudaMemcpyHostToDevice);
        if (gathers) k_wait<true><<<1, 32>>>(d, d + 1);
        else k_wait<false><<<1, 32>>>(d, d + 1);
        if (cudaMemcpy(h, d, 8, cudaMemcpyDeviceToHost) != cudaSuccess) return 2;
        printf("%d %d\n", h[0], h[1]);
    }
    return 0;
}
"""


def test_a_wait_that_runs_out_reports_as_its_word_is_read(tmp_path):
    """A handle's word holds the last code, a cache's status gathers bits."""
    src, exe = tmp_path / "wait.cu", tmp_path / "wait"
    src.write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    r = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", build.CSRC, "-o", str(exe), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.split() == ["16", "0", "21", "0"], r
