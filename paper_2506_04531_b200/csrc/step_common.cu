// Host side that the operators of the local step share.
#include "step_common.cuh"

#include <atomic>
#include <stdio.h>

namespace halos_step {
namespace {
constexpr int kMaxDevices = 64;
thread_local char t_error[256] = "";
thread_local int t_device = 0;
std::atomic<int> g_sms[kMaxDevices];
__device__ int g_fault;
}  // namespace

int fail(int status, const char* text) {
    snprintf(t_error, sizeof t_error, "%s", text);
    return status;
}

int cuda_status(cudaError_t e, const char* where) {
    if (e == cudaSuccess) return HALOS_OK;
    snprintf(t_error, sizeof t_error, "%s: %s", where, cudaGetErrorString(e));
    (void)cudaGetLastError();
    return HALOS_ERR_CUDA;
}

int enter(int32_t device) {
    if (device < 0 || device >= kMaxDevices) return fail(HALOS_ERR_INVALID_ARG, "no such device");
    if (int rc = cuda_status(cudaSetDevice(device), "cudaSetDevice (there is no CPU path)")) return rc;
    t_device = device;
    if (!g_sms[device].load(std::memory_order_relaxed)) {
        int n = 0;
        if (int rc = cuda_status(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device), "multiprocessor count")) return rc;
        g_sms[device].store(n, std::memory_order_relaxed);
    }
    return HALOS_OK;
}

int fault_mark(int** mark) {
    static std::atomic<int*> known[kMaxDevices];
    *mark = known[t_device].load(std::memory_order_relaxed);
    if (*mark) return HALOS_OK;
    if (int rc = cuda_status(cudaGetSymbolAddress((void**)mark, g_fault), "fault mark")) return rc;
    known[t_device].store(*mark, std::memory_order_relaxed);
    return HALOS_OK;
}

int current_device() { return t_device; }

int sm_count(int32_t device) { return g_sms[device].load(std::memory_order_relaxed); }

}  // namespace halos_step

extern "C" const char* halos_step_error(void) { return halos_step::t_error; }

extern "C" int halos_step_fault(int32_t device, int32_t* fault) {
    using namespace halos_step;
    if (!fault) return fail(HALOS_ERR_INVALID_ARG, "fault: null pointer");
    if (int rc = enter(device)) return rc;
    // A copy alone would not wait for streams that do not synchronise with the default one.
    if (int rc = cuda_status(cudaDeviceSynchronize(), "fault mark")) return rc;
    return cuda_status(cudaMemcpyFromSymbol(fault, g_fault, sizeof(int)), "fault mark");
}
