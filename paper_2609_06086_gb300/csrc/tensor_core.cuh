// PTX that the kernels with tensor-core products share (wgrad.cu, attn.cu,
// attn_backward.cu): barriers in shared memory with bounded waits, register splits.
#pragma once
#include <cuda.h>

#include <mutex>

#include "common.cuh"
#include "wait_limit.h"

namespace pos {

__device__ __forceinline__ uint32_t smem_u32(const void *p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {  // own CTA
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}
constexpr uint32_t kTryNs = 1000000;  // a try sleeps for up to 1 ms
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity, uint32_t sleep = kTryNs) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(sleep)
        : "memory");
    return ok;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Waits for a phase, two seconds at most (WaitLimit); false: it did not come, or
// another wait of the block has already given up.
__device__ __forceinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    WaitLimit limit(now_ns());
    for (;;) {
        if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
        if (limit.reached(now_ns())) {
            *gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity, gave_up);
}
template <int R>
__device__ __forceinline__ void give_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void take_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);
// The driver's function that describes a tensor for copies into shared memory.
inline pos_status encode_fn(EncodeTiled *out) {
    static std::mutex mu;
    static EncodeTiled fn;
    std::lock_guard<std::mutex> lock(mu);
    if (!fn) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        POS_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000,
                                                  cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !f)
            return fail(POS_ECUDA, "the driver has no cuTensorMapEncodeTiled");
        fn = reinterpret_cast<EncodeTiled>(f);
    }
    *out = fn;
    return POS_OK;
}

}  // namespace pos
