// Kernels that may begin while the previous kernel of their stream ends.
//
// A small call spends as long on being launched and setting up (barriers, tensor memory) as on its work.  These kernels are
// launched with the programmatic attribute: their CTAs may start as soon as every CTA of the previous kernel has said so or
// ended, and wait in after_previous() until that kernel is complete and its writes are visible.  Nothing of the call's
// operands may be touched before it.  Kernels that never say anything (all others) are waited for as ever.
#pragma once
#include <cuda_runtime.h>

namespace dr {

inline cudaLaunchAttribute overlap_attribute()
{
    cudaLaunchAttribute a{};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    return a;
}
__device__ __forceinline__ void after_previous()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

}  // namespace dr
