// Host side that the operators of the local step share.
#include "step_common.cuh"

#include <atomic>
#include <mutex>
#include <stdio.h>

namespace halos_step {
namespace {
constexpr int kMaxDevices = 64;
thread_local char t_error[256] = "";
thread_local int t_device = 0;
std::atomic<int> g_sms[kMaxDevices];
// A word for each device, in host memory that kernels write to: every call looks at it without asking the device.  Never given back.
std::atomic<volatile int*> g_marks;
std::mutex g_making_marks;

int marks(volatile int** at) {
    *at = g_marks.load(std::memory_order_acquire);
    if (*at) return HALOS_OK;
    const std::lock_guard<std::mutex> alone(g_making_marks);
    *at = g_marks.load(std::memory_order_relaxed);
    if (*at) return HALOS_OK;
    // The first call may come while its stream is being captured, which an allocation has no part in.
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    if (int rc = cuda_status(cudaThreadExchangeStreamCaptureMode(&mode), "fault marks")) return rc;
    int* made = nullptr;
    const cudaError_t e = cudaHostAlloc((void**)&made, kMaxDevices * sizeof(int), cudaHostAllocPortable | cudaHostAllocMapped);
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    if (int rc = cuda_status(e, "fault marks")) return rc;
    for (int i = 0; i < kMaxDevices; ++i) made[i] = 0;
    *at = made;
    g_marks.store(made, std::memory_order_release);
    return HALOS_OK;
}

int make_current(int32_t device) {
    if (device < 0 || device >= kMaxDevices) return fail(HALOS_ERR_INVALID_ARG, "no such device");
    return cuda_status(cudaSetDevice(device), "cudaSetDevice (there is no CPU path)");
}
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
    if (int rc = make_current(device)) return rc;
    t_device = device;
    if (!g_sms[device].load(std::memory_order_relaxed)) {
        int n = 0;
        if (int rc = cuda_status(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device), "multiprocessor count")) return rc;
        g_sms[device].store(n, std::memory_order_relaxed);
    }
    volatile int* at = nullptr;
    if (int rc = marks(&at)) return rc;
    if (at[device]) return fail(HALOS_ERR_CUDA, "a bounded wait of an earlier call on this device ran out: what that call returned is undefined (halos_step_fault clears the mark)");
    return HALOS_OK;
}

int fault_mark(int** mark) {
    volatile int* at = nullptr;
    if (int rc = marks(&at)) return rc;
    *mark = const_cast<int*>(at) + t_device;  // one address on the host and on every device
    return HALOS_OK;
}

int current_device() { return t_device; }

int sm_count(int32_t device) { return g_sms[device].load(std::memory_order_relaxed); }

}  // namespace halos_step

extern "C" const char* halos_step_error(void) { return halos_step::t_error; }

extern "C" int halos_step_fault(int32_t device, int32_t* fault) {
    using namespace halos_step;
    if (!fault) return fail(HALOS_ERR_INVALID_ARG, "fault: null pointer");
    if (int rc = make_current(device)) return rc;
    volatile int* at = nullptr;
    if (int rc = marks(&at)) return rc;
    if (int rc = cuda_status(cudaDeviceSynchronize(), "fault mark")) return rc;
    *fault = at[device], at[device] = 0;
    return HALOS_OK;
}
