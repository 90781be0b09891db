// Device-side definitions shared by the kernels of the decode step (append, attend).
#pragma once
#include "tri_common.cuh"

namespace tri {

// Programmatic dependent launch: waits for the kernels this launch depends on; lets a launch that depends on this kernel begin.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
__device__ __forceinline__ void grid_dependents_launch() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

// Lengths, groups and page ids.  A kernel that begins before its predecessor has ended reads nothing through the read-only path
// (__ldg): such a load promises that the data stay as they are from the kernel's first instruction on, so that the compiler may
// move it before the wait.  This one stays where it is written.  (Plain loads stay behind the wait, too, but cost the prefix kernel
// 3 us of 68 in shared_32_of_32k and 3 of 109 in shared_64_of_6_paged, two cases of perf/operators.py.)
__device__ __forceinline__ int32_t ld_here(const int32_t *p)
{
    int32_t x;
    asm volatile("ld.global.s32 %0, [%1];\n" : "=r"(x) : "l"(p) : "memory");
    return x;
}
// For what was written before the predecessor began, in a kernel that does not wait for that one.  The predecessor's blocks let
// it begin behind their own wait, so all earlier kernels have ended and what they wrote is performed, in L2 at the latest.  Both
// loads are answered by L2, not by a line that the multiprocessor still holds from before; behind the acquiring one (and a
// barrier of the block, for its other threads) the same goes for weak loads.  For shared_32_of_32k and shared_64_of_6_paged (68
// and 109 us) a fence in the acquiring load's place measured the same, strong loads throughout the same and 4 us more, waiting
// in front 10 us more in both.
__device__ __forceinline__ int32_t ld_acquire(const int32_t *p)
{
    int32_t x;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];\n" : "=r"(x) : "l"(p) : "memory");
    return x;
}
__device__ __forceinline__ int32_t ld_relaxed(const int32_t *p)
{
    int32_t x;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];\n" : "=r"(x) : "l"(p) : "memory");
    return x;
}

// row_offset() with such a load of the page id.
__device__ __forceinline__ int64_t step_row_offset(const View &w, int l, int s, int h, int n)
{
    const int64_t unit = (int64_t)l * w.stride_layer + (int64_t)h * w.stride_head;
    if (!w.paged) return unit + (int64_t)s * w.stride_seq + (int64_t)n * w.stride_tok;
    const int pg = w.page_shift >= 0 ? n >> w.page_shift : n / w.page_size;
    const int page = ld_here(w.page_table + (int64_t)s * w.max_pages_per_seq + pg);
    if (w.n_pages > 0 && (page < 0 || page >= w.n_pages)) return -1;
    return unit + (int64_t)page * w.stride_page + (int64_t)(n - pg * w.page_size) * w.stride_slot;
}

}  // namespace tri
