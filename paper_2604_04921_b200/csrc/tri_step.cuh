// Device-side definitions shared by the kernels of the decode step (append, attend).
#pragma once
#include "tri_common.cuh"

namespace tri {

// Programmatic dependent launch: waits for the kernels this launch depends on; lets a launch that depends on this kernel begin.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
__device__ __forceinline__ void grid_dependents_launch() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

}  // namespace tri
