// Shared-memory barriers, as the kernels that load by TMA use them: every wait is bounded.
#pragma once

#include <cuda_runtime.h>

namespace csd {
namespace ptx {

constexpr long long kWaitCycles = 4000000000ll;      // about two seconds

__device__ __forceinline__ unsigned int smem_u32(const void *p) { return static_cast<unsigned int>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(unsigned int bar, unsigned int count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned int bar, unsigned int bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(unsigned int bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(unsigned int bar, unsigned int parity)
{
    unsigned int ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0u;
}
// Bounded wait.  False if the wait ran out or another role of the CTA has given up.
__device__ __forceinline__ bool mbar_wait(unsigned int bar, unsigned int parity, volatile int *give_up)
{
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity)) {
        if (*give_up) return false;
        if (clock64() - t0 > kWaitCycles) {
            *give_up = 1;
            return false;
        }
    }
    return true;
}

}  // namespace ptx
}  // namespace csd
