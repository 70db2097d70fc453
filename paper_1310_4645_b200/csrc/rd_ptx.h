// Barriers in shared memory, and the limits of waits on them.
#ifndef RD_PTX_H_
#define RD_PTX_H_

#include <cuda_runtime.h>

#include <cstdint>

namespace rd {

constexpr long long kWaitCycles = 4000000000ll;     // a wait gives up after about two seconds of SM clock
constexpr long long kDrainCycles = 20000000ll;      // after that, copies in flight get ten milliseconds to land

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok;
}
// After a wait that gave up: lets the copies in flight land before the kernel ends.
static __device__ __noinline__ void drain()
{
    const long long t0 = clock64();
    while (clock64() - t0 < kDrainCycles) {}
}
}  // namespace rd

#endif  // RD_PTX_H_
