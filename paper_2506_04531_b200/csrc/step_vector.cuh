// Neighbouring elements of a row as they are loaded, and as 32-bit floats.
#pragma once
#include "step_common.cuh"

namespace halos_step {

// N elements of T: 2, 4, 8, 16 or 32 bytes, in accesses of 16 bytes at most.
template <typename T, int N>
struct Words {
    static constexpr int kBytes = N * (int)sizeof(T);
    uint32_t w[kBytes >= 4 ? kBytes / 4 : 1];
};

template <typename T, int N>
__device__ __forceinline__ Words<T, N> load_words(const T* p) {
    Words<T, N> r;
    constexpr int B = Words<T, N>::kBytes;
    if constexpr (B == 2) r.w[0] = *reinterpret_cast<const uint16_t*>(p);
    if constexpr (B == 4) r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (B == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        r.w[0] = v.x, r.w[1] = v.y;
    }
    if constexpr (B >= 16) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            r.w[4 * i] = v.x, r.w[4 * i + 1] = v.y, r.w[4 * i + 2] = v.z, r.w[4 * i + 3] = v.w;
        }
    }
    return r;
}

template <typename T, int N>
__device__ __forceinline__ void store_words(T* p, const Words<T, N>& r) {
    constexpr int B = Words<T, N>::kBytes;
    if constexpr (B == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)r.w[0];
    if constexpr (B == 4) *reinterpret_cast<uint32_t*>(p) = r.w[0];
    if constexpr (B == 8) *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
    if constexpr (B >= 16) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
    }
}

template <typename T, int N>
__device__ __forceinline__ Words<T, N> no_words() {
    Words<T, N> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof r.w / 4); ++i) r.w[i] = 0;
    return r;
}

// One element on its own, for the ends of rows that vectors do not divide.
template <typename T, int N>
__device__ __forceinline__ void put_element(Words<T, N>& r, int e, T v) {
    if constexpr (sizeof(T) == 4) r.w[e] = __float_as_uint(to_f32(v));
    else {
        const uint32_t bits = *reinterpret_cast<const uint16_t*>(&v);
        r.w[e / 2] = e % 2 ? (r.w[e / 2] & 0xffffu) | bits << 16 : (r.w[e / 2] & 0xffff0000u) | bits;
    }
}

template <typename T, int N>
__device__ __forceinline__ void widen(const Words<T, N>& r, float (&v)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (N == 1) {
        v[0] = unpack2<T>(r.w[0]).x;
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 p = unpack2<T>(r.w[i]);
            v[2 * i] = p.x, v[2 * i + 1] = p.y;
        }
    }
}

template <typename T, int N>
__device__ __forceinline__ Words<T, N> narrow(const float (&v)[N]) {
    Words<T, N> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = __float_as_uint(v[i]);
    } else if constexpr (N == 1) {
        r.w[0] = pack2<T>(v[0], 0.f);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) r.w[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
    }
    return r;
}

// The same by pairs, for operations on two 32-bit floats at once.
template <typename T, int N>
__device__ __forceinline__ void widen(const Words<T, N>& r, float2 (&v)[N / 2]) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
        else v[i] = unpack2<T>(r.w[i]);
    }
}
template <typename T, int N>
__device__ __forceinline__ Words<T, N> narrow(const float2 (&v)[N / 2]) {
    Words<T, N> r;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        if constexpr (sizeof(T) == 4) r.w[2 * i] = __float_as_uint(v[i].x), r.w[2 * i + 1] = __float_as_uint(v[i].y);
        else r.w[i] = pack2<T>(v[i].x, v[i].y);
    }
    return r;
}

// Copies of 16 bytes, and of 4, into shared memory that nothing waits for until asked.
__device__ __forceinline__ void copy_16(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_4(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_copies(bool all_but_one) {
    if (all_but_one) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

inline uint32_t size_of(uint32_t type) { return type == HALOS_F32 ? 4 : 2; }

}  // namespace halos_step
