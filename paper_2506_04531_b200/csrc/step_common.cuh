// What the operators of the local step share: element types, wide loads and stores, error text.
#pragma once
#include "halos_step.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <atomic>
#include <mutex>
#include <stdint.h>

namespace halos_step {

int fail(int status, const char* text);                 // sets the thread's error text, returns status
int cuda_status(cudaError_t e, const char* where);      // HALOS_OK, or fail(HALOS_ERR_CUDA, ...)
int enter(int32_t device);                              // makes the device current; fails where a wait has run out on it
int sm_count(int32_t device);                           // of a device that enter() accepted
int fault_mark(int** mark);                             // where the current device's kernels say that a wait ran out: host memory

constexpr int kSharedPerSM = 228 * 1024;
int current_device();                                   // that enter() was last called with in this thread
// Lets a kernel have this much dynamic shared memory; each caller keeps what it was last allowed, per device.  One thread at a time sets and
// notes a limit, and it only grows: the limit that holds is never below the one that is noted.
struct Allowed {
    std::atomic<int> bytes[64];
    std::mutex changing;
};
template <typename K>
int allow_smem(K* kernel, int bytes, Allowed& allowed) {
    std::atomic<int>& had = allowed.bytes[current_device()];
    if (had.load(std::memory_order_acquire) >= bytes) return HALOS_OK;
    const std::lock_guard<std::mutex> alone(allowed.changing);
    if (had.load(std::memory_order_relaxed) >= bytes) return HALOS_OK;
    if (int rc = cuda_status(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes), "shared memory")) return rc;
    had.store(bytes, std::memory_order_release);
    return HALOS_OK;
}

// A kernel that may be started while the one before it in the stream still runs, and what it does before it touches what that one leaves: nothing
// of this waits for anything but that kernel's end.
template <typename... P, typename... A>
int launch_after(void (*kernel)(P...), dim3 grid, uint32_t threads, size_t shared, cudaStream_t st, const char* where, const A&... args) {
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization, early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = grid, config.blockDim = dim3(threads), config.dynamicSmemBytes = shared, config.stream = st, config.attrs = &early, config.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&config, kernel, args...), where);
}
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void say_fault(int* mark) { *const_cast<volatile int*>(mark) = 1; }

inline bool is_type(uint32_t t) { return t == HALOS_F32 || t == HALOS_BF16 || t == HALOS_F16; }

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Two neighbours as one 32-bit word, and back.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<uint64_t&>(r))
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 exp2_both(float2 x) { return make_float2(fast_exp2(x.x), fast_exp2(x.y)); }

}  // namespace halos_step
