"""The mark that a bounded wait leaves when it runs out."""
from __future__ import annotations

import os
import subprocess
from pathlib import Path

import pytest
import torch

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

# One warp waits for a barrier at which nobody arrives: for a second, as the kernels' waits do, and then goes on.
SOURCE = r"""
#include "step_common.cu"
#include "step_tcgen05.cuh"
__global__ void wait_in_vain(int* fault, int* after) {
    __shared__ uint64_t bar;
    __shared__ int gave_up;
    const uint32_t at = halos_step::smem_u32(&bar);
    if (threadIdx.x == 0) {
        halos_step::bar_init(at, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        gave_up = 0;
    }
    __syncthreads();
    const halos_step::Waits W{&gave_up, fault};
    W.wait_warp(at, 0);
    W.wait_warp(at, 0);  // returns at once
    if (threadIdx.x == 0) *after = gave_up;
}
#define CHECK(c) if (!(c)) { printf("line %d: %s", __LINE__, halos_step_error()); return 1; }
int main() {
    using namespace halos_step;
    int *mark = nullptr, *after = nullptr, gave_up = 0;
    int32_t fault = 7;
    CHECK(enter(0) == HALOS_OK && fault_mark(&mark) == HALOS_OK && cudaMalloc(&after, sizeof(int)) == cudaSuccess);
    CHECK(halos_step_fault(0, &fault) == HALOS_OK && fault == 0);
    wait_in_vain<<<1, 32>>>(mark, after);
    CHECK(cudaDeviceSynchronize() == cudaSuccess);
    CHECK(cudaMemcpy(&gave_up, after, sizeof(int), cudaMemcpyDeviceToHost) == cudaSuccess && gave_up == 1);
    CHECK(enter(0) == HALOS_ERR_CUDA);
    CHECK(halos_step_fault(0, &fault) == HALOS_OK && fault == 1);
    CHECK(enter(0) == HALOS_OK);
    printf("ok");
    return 0;
}
"""


def test_the_mark_is_read_after_what_any_stream_has_been_given():
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    step.fault()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)      # a tenth of a second
        done.record()
    assert not step.fault()
    assert done.query()


def test_a_wait_that_runs_out_ends_and_is_an_error_of_the_next_call(tmp_path):
    src, exe = tmp_path / "wait.cu", tmp_path / "wait"
    src.write_text(SOURCE)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", str(ROOT / "include"),
                    "-I", str(ROOT / "paper_2506_04531_b200" / "csrc"), "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.stdout == "ok", r.stdout
