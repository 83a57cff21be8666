// Shared by the kernels that use the tensor cores (train_ortho.cu, train_attention.cu): barriers in shared memory
// with bounded waits, operand descriptors, tensor memory.
#pragma once
#include "train_common.cuh"

namespace spb {

constexpr unsigned long long kWaitNs = 2000000000ull;  // a wait inside a kernel gives up after this

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// kSuspendNs: how long the hardware may let the thread sleep in one try; 0: its own limit.
template <uint32_t kSuspendNs = 0>
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    if constexpr (kSuspendNs > 0) {
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "n"(kSuspendNs)
            : "memory");
    } else {
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
    }
    return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Bounded: false once the time is up or another role of the CTA gave up.  For one lane.
template <uint32_t kSuspendNs = 0>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up,
                                         unsigned long long limit) {
    if (bar_try<kSuspendNs>(bar, parity)) return true;
    const unsigned long long until = now_ns() + limit;
    while (!bar_try<kSuspendNs>(bar, parity)) {
        if (*gave_up) return false;
        if (now_ns() > until) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}
// The same for a whole warp: all lanes get one answer.  Each by itself could see the time run out a look before or
// after another, and what follows a wait (elect, tensor memory) takes all lanes of the warp.
template <uint32_t kSuspendNs = 0>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up,
                                          unsigned long long limit) {
    if (__all_sync(kAllLanes, bar_try<kSuspendNs>(bar, parity))) return true;
    const unsigned long long until = now_ns() + limit;
    while (!__all_sync(kAllLanes, bar_try<kSuspendNs>(bar, parity))) {
        if (__any_sync(kAllLanes, *gave_up || now_ns() > until)) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
// Shared-memory operand of 128-byte swizzled rows.  K-major: groups of 8 rows `sbo` apart.  MN-major:
// blocks of 64 elements `lbo` apart, groups of 8 k `sbo` apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = __uint_as_float(r[i]);
}

}  // namespace spb
