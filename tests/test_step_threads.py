"""Host code of the local step's operators that several threads enter at once."""
from __future__ import annotations

import os
import subprocess
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent

# The kernel's limit is set through a stand-in that lets the threads meet where they would do harm: the larger request has been set when
# the smaller one comes, and returns after it.
SHARED_MEMORY = r"""
#include <cuda_runtime.h>
#include <stdio.h>
#include <atomic>
#include <chrono>
#include <thread>
static std::atomic<int> limit{0}, larger_is_set{0};
static cudaError_t set_limit(const void*, cudaFuncAttribute, int bytes) {
    limit = bytes;
    if (bytes == 100) {
        larger_is_set = 1;
        std::this_thread::sleep_for(std::chrono::milliseconds(300));
    }
    return cudaSuccess;
}
template <typename K> static cudaError_t set_limit_of(K* kernel, cudaFuncAttribute what, int bytes) { return set_limit((const void*)kernel, what, bytes); }
#define cudaFuncSetAttribute set_limit_of
#include "step_common.cuh"
namespace halos_step {
int fail(int status, const char*) { return status; }
int cuda_status(cudaError_t e, const char*) { return e == cudaSuccess ? HALOS_OK : HALOS_ERR_CUDA; }
int current_device() { return 0; }
}
__global__ void kernel() {}
int main() {
    static halos_step::Allowed allowed;
    std::thread larger([] { halos_step::allow_smem(kernel, 100, allowed); });
    std::thread smaller([] {
        while (!larger_is_set) std::this_thread::yield();
        halos_step::allow_smem(kernel, 60, allowed);
    });
    larger.join(), smaller.join();
    if (halos_step::allow_smem(kernel, 100, allowed)) return 2;  // what a later call asks for
    printf("%d", (int)limit);
    return 0;
}
"""


def test_a_kernel_keeps_the_most_shared_memory_that_any_thread_asked_for(tmp_path):
    src, exe = tmp_path / "limit.cu", tmp_path / "limit"
    src.write_text(SHARED_MEMORY)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", str(ROOT / "include"), "-I", str(ROOT / "paper_2506_04531_b200" / "csrc"),
                    "-o", str(exe), str(src)], check=True)
    assert int(subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout) == 100
