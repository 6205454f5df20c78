"""What the host makes of the mark that a bounded wait leaves when it runs out, with stand-ins for the CUDA runtime."""
from __future__ import annotations

import os
import subprocess
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent

SOURCE = r"""
#include <cuda_runtime.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
static int synchronised = 0, allocations = 0, mode_now = 0;
static cudaError_t set_device(int) { return cudaSuccess; }
static cudaError_t attribute(int* n, cudaDeviceAttr, int) { *n = 148; return cudaSuccess; }
static cudaError_t host_alloc(void** p, size_t bytes, unsigned) {
    if (mode_now != cudaStreamCaptureModeRelaxed) return cudaErrorStreamCaptureUnsupported;
    ++allocations, *p = malloc(bytes), memset(*p, 255, bytes);
    return cudaSuccess;
}
static cudaError_t exchange(cudaStreamCaptureMode* mode) { const int had = mode_now; mode_now = *mode, *mode = (cudaStreamCaptureMode)had; return cudaSuccess; }
static cudaError_t synchronise() { ++synchronised; return cudaSuccess; }
#define cudaSetDevice set_device
#define cudaDeviceGetAttribute attribute
#undef cudaHostAlloc
#define cudaHostAlloc host_alloc
#define cudaThreadExchangeStreamCaptureMode exchange
#define cudaDeviceSynchronize synchronise
#include "step_common.cu"
#define CHECK(c) if (!(c)) { printf("line %d", __LINE__); return 1; }
int main() {
    using namespace halos_step;
    int* mark = nullptr;
    int32_t fault = 7;
    CHECK(enter(3) == HALOS_OK && fault_mark(&mark) == HALOS_OK && *mark == 0);
    CHECK(halos_step_fault(3, &fault) == HALOS_OK && fault == 0 && synchronised == 1);
    *mark = 1;                                                   // a wait on device 3 has run out
    CHECK(enter(3) == HALOS_ERR_CUDA && strstr(halos_step_error(), "wait of an earlier call"));
    CHECK(enter(3) == HALOS_ERR_CUDA);                           // every later call
    CHECK(enter(2) == HALOS_OK);                                 // other devices are well
    CHECK(halos_step_fault(2, &fault) == HALOS_OK && fault == 0);
    CHECK(halos_step_fault(3, &fault) == HALOS_OK && fault == 1);
    CHECK(enter(3) == HALOS_OK);                                 // it has been asked for
    CHECK(halos_step_fault(3, &fault) == HALOS_OK && fault == 0);
    CHECK(halos_step_fault(64, &fault) == HALOS_ERR_INVALID_ARG && halos_step_fault(3, nullptr) == HALOS_ERR_INVALID_ARG);
    CHECK(allocations == 1 && mode_now == 0);
    printf("ok");
    return 0;
}
"""


def test_a_wait_that_ran_out_is_an_error_of_the_next_call(tmp_path):
    src, exe = tmp_path / "fault.cu", tmp_path / "fault"
    src.write_text(SOURCE)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", str(ROOT / "include"),
                    "-I", str(ROOT / "paper_2506_04531_b200" / "csrc"), "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.stdout == "ok"
