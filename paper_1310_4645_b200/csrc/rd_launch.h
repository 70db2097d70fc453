// Launches whose start overlaps the end of the kernel before them in the stream.
#ifndef RD_LAUNCH_H_
#define RD_LAUNCH_H_

#include <cuda_runtime.h>

namespace rd {

// First statement of every kernel launched below, before it touches memory: lets the next kernel's thread blocks come up and
// wait, and waits itself until the kernels before it are done.  Every one of them waits, so what is two kernels back is done too.
__device__ __forceinline__ void pdl_start()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// The same the other way round, for the first kernel of a call whose later ones include one that does not wait: nothing of the
// call starts before the stream's earlier work is done.
__device__ __forceinline__ void pdl_wait_first()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Both halves by themselves: for kernels of as many thread blocks as fit at once, each with a fixed share of the work.  Blocks of the
// next kernel that come up while such a kernel starts take room that some of its own blocks then wait for, and with them all of their
// share (norm gradient of 16384 x 4096 bf16 with its join: 240 us released at the start, B200).
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

inline cudaLaunchAttribute pdl_attribute()
{
    cudaLaunchAttribute a{};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    return a;
}

template <typename... P, typename... A> cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, cudaStream_t stream, A &&...args)
{
    cudaLaunchConfig_t c{};
    cudaLaunchAttribute pdl = pdl_attribute();
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.stream = stream;
    c.attrs = &pdl;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, P(args)...);
}

}  // namespace rd

#endif  // RD_LAUNCH_H_
