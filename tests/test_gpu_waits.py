"""The bounded wait of a whole warp gives all lanes one answer.  A barrier's phase ends
after some of the lanes have reached their limit (an own limit and flag for each lane here, so that
it happens every time; in a product's kernel it takes a phase that ends just then)."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include "tc_ptx.cuh"
using namespace moara;

// out[form * 32 + lane]: what lane got from the wait of one lane (0), of a warp (1), of a warp with
// cluster scope (2)
__global__ void k_waits(int* out, int* status, long long lower, long long upper, long long delay) {
    __shared__ uint64_t bars[3];
    __shared__ int flags[32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int form = 0; form < 3; ++form) {
        uint64_t& bar = bars[form];
        if (threadIdx.x < 32) flags[lane] = 0;
        if (threadIdx.x == 0) {
            ptx::mbar_init(ptx::smem_u32(&bar), 1);
            ptx::fence_barrier_init();
        }
        __syncthreads();
        if (warp == 1) {
            const long long t0 = clock64();
            while (clock64() - t0 < delay) {}
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&bar));
        } else {
            const long long limit = lane & 1 ? upper : lower;
            const uint32_t b = ptx::smem_u32(&bar);
            const bool got = form == 0   ? ptx::mbar_wait(b, 0, flags + lane, status, -7, limit)
                             : form == 1 ? ptx::mbar_wait_warp(b, 0, flags + lane, status, -7, limit)
                                         : ptx::mbar_wait_cluster_warp(b, 0, flags + lane, status, -7, limit);
            out[form * 32 + lane] = got;
        }
        __syncthreads();
    }
}

extern "C" int run(int* out, int* status, long long lower, long long upper, long long delay) {
    k_waits<<<1, 64>>>(out, status, lower, upper, delay);
    return cudaDeviceSynchronize();
}
"""


def test_lanes_of_a_warp_agree(tmp_path):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    (tmp_path / "w.cu").write_text(SRC)
    so = tmp_path / "w.so"
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2609_15037_gb300", "csrc"), str(tmp_path / "w.cu"), "-o", str(so)], check=True)
    run = ctypes.CDLL(str(so)).run
    run.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_longlong] * 3
    out = torch.full((96,), -1, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    # a limit of 1,000 clocks for the even lanes, and the phase's end behind 20 million (10 ms)
    assert run(out.data_ptr(), status.data_ptr(), 1000, 1 << 30, 20000000) == 0
    got = out.cpu().numpy().reshape(3, 32)
    assert np.array_equal(got[0], np.arange(32) % 2)        # lanes by themselves part
    assert not got[1:].any() and status.item() == -7
    # long limits for all: every lane sees the phase end
    assert run(out.data_ptr(), status.data_ptr(), 1 << 30, 1 << 30, 20000) == 0
    assert (out == 1).all()
