// Fifth-generation tensor cores, tensor memory, bulk copies and their barriers, as the attention kernels use them.
#pragma once
#include "step_common.cuh"

#include <cuda.h>

namespace halos_step {

// ---- warps that act as one ---------------------------------------------------------------------
// Copies and products are issued by one thread, but the warp goes through the loop together: what it computes is then the same in
// all lanes, which is where those instructions want their operands.
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.b32 %0, 1, 0, p; }" : "=r"(p));
    return p != 0;
}
template <typename V> __device__ __forceinline__ V uniform(V v) { return __shfl_sync(~0u, v, 0); }

// ---- barriers in shared memory -----------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Returns at the latest after a millisecond or so, and at once where the phase is over.
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3; selp.b32 %0, 1, 0, p; }"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
    return ok != 0;
}

__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.b32 %0, 1, 0, p; }"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

// Waits are bounded: one that runs out marks the CTA and *fault, and from then on every wait of the CTA returns at once.  All loops go on
// to their ends, within their buffers but with whatever is there, and before a CTA ends its copies and products in
// flight are waited for (again with a bound), so that tensor memory is given back and nothing hangs.
constexpr long long kWaitClocks = 2000000000ll;  // about a second
struct Waits {
    volatile int* gave_up;  // in shared memory
    int* fault;             // in host memory
    __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity) const {
        if (!bar_test(bar, parity)) wait_longer(bar, parity);
    }
    // For a warp whose next instruction is one for all its lanes together.
    __device__ __forceinline__ void wait_warp(uint32_t bar, uint32_t parity) const {
        wait(bar, parity);
        __syncwarp();
    }
    __device__ __noinline__ void wait_longer(uint32_t bar, uint32_t parity) const {
        const long long began = clock64();
        while (!*gave_up) {
            if (bar_try(bar, parity)) return;
            if (clock64() - began > kWaitClocks) {
                *gave_up = 1;
                say_fault(fault);
            }
        }
    }
    __device__ __noinline__ void drain(uint32_t bar, uint32_t parity) const {
        const long long began = clock64();
        while (!bar_try(bar, parity) && clock64() - began < kWaitClocks / 16) {}
    }
};

// ---- bulk copies -------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int d, int s, int h, int b) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(d), "r"(s), "r"(h), "r"(b) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory -----------------------------------------------------------------------------
template <int kColumns> __device__ __forceinline__ void tmem_alloc(uint32_t dst) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "n"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
template <int kColumns> __device__ __forceinline__ void tmem_free(uint32_t tmem) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kColumns));
}
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The registers of loads in flight go through the wait, so that nothing made of them can come before it.
#define HALOS_EIGHT(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
__device__ __forceinline__ void tmem_wait_loads16(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : HALOS_EIGHT(r, 0), HALOS_EIGHT(r, 8)::"memory");
}
__device__ __forceinline__ void tmem_wait_loads32(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : HALOS_EIGHT(r, 0), HALOS_EIGHT(r, 8), HALOS_EIGHT(r, 16), HALOS_EIGHT(r, 24)::"memory");
}
__device__ __forceinline__ void tmem_hold32(uint32_t* r) {  // for further registers of a wait just made
    asm volatile("" : HALOS_EIGHT(r, 0), HALOS_EIGHT(r, 8), HALOS_EIGHT(r, 16), HALOS_EIGHT(r, 24)::"memory");
}
#undef HALOS_EIGHT
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of this warp's 32 lanes: thread = lane, register = column.
__device__ __forceinline__ void tmem_load32(uint32_t* r, uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_load16(uint32_t* r, uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// 16 lanes by 32 columns: register 4 k + 2 i + e of a thread = lane t/4 + 8 i, column 8 k + 2 (t % 4) + e.
__device__ __forceinline__ void tmem_load_16x32(uint32_t* r, uint32_t at) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}
// 16 lanes by 32 columns: register 2 k + i of a thread = lane t/4 + 8 i, column 4 k + t % 4.
__device__ __forceinline__ void tmem_store_16x32(uint32_t at, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// ---- matrix products ---------------------------------------------------------------------------
// Operands in shared memory lie as the bulk copy's 128-byte swizzle leaves them: rows of 64 16-bit elements, blocks of 8
// rows (1024 bytes), sub-tiles of 64 columns one after another.
//
// As a "K-major" operand the 64 columns run along the summed dimension: 8-row blocks are 1024 bytes apart, and a
// step of 16 summed elements is 32 bytes.  As an "MN-major" operand the rows do: again 1024 bytes between
// blocks of 8 summed rows, a step of 16 is 2048 bytes, and the next 64 columns lie one sub-tile further.
constexpr uint32_t kOperandHigh = (2u << 29) | (1u << 14) | (1024 >> 4);
__device__ __forceinline__ uint32_t operand_low(uint32_t addr, uint32_t leading_bytes) { return ((addr & 0x3ffff) >> 4) | ((leading_bytes >> 4) << 16); }
__device__ __forceinline__ uint64_t operand(uint32_t low) { return ((uint64_t)kOperandHigh << 32) | low; }
template <typename T> struct MmaType;
template <> struct MmaType<__half> { static constexpr uint32_t id = 0; };
template <> struct MmaType<__nv_bfloat16> { static constexpr uint32_t id = 1; };
// 16-bit operands of one type, 32-bit sums; B transposed means MN-major.
template <typename T, int M, int N, bool kBTransposed>
__host__ __device__ constexpr uint32_t mma_shape() {
    return (1u << 4) | (MmaType<T>::id << 7) | (MmaType<T>::id << 10) | ((kBTransposed ? 1u : 0u) << 16) | ((uint32_t)(N / 8) << 17) |
           ((uint32_t)(M / 16) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
        ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
        ::"r"(d), "r"(a), "l"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}
// Arrives on the barrier once every product issued so far has been done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// D[128 x N] = A[128 x K] B[N x K]^T, both K-major in shared memory, with sub-tiles of kRowsA and kRowsB rows.
template <typename T, int N, int K, int kRowsA, int kRowsB>
__device__ __forceinline__ void product_ss(uint32_t d, uint32_t a, uint32_t b) {
    const uint32_t al = operand_low(a, 16), bl = operand_low(b, 16);
#pragma unroll
    for (int k = 0; k < K / 16; ++k)
        mma_ss(d, operand(al + (k / 4) * kRowsA * 8 + (k % 4) * 2), operand(bl + (k / 4) * kRowsB * 8 + (k % 4) * 2), mma_shape<T, 128, N, false>(), k > 0);
}
// D[128 x N] (+)= A[128 x K] B[K x N]: A in tensor memory, 32 summed elements every kApart columns (16: without gaps), B's K rows
// in shared memory.
template <typename T, int N, int K, int kApart>
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t b, bool add) {
    const uint32_t bl = operand_low(b, K * 128);
#pragma unroll
    for (int k = 0; k < K / 16; ++k)
        mma_ts(d, a + (k / 2) * kApart + (k % 2) * 8, operand(bl + k * 128), mma_shape<T, 128, N, true>(), add || k > 0);
}

}  // namespace halos_step
