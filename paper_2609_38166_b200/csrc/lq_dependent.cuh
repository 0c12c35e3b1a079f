#pragma once

namespace lq {

// Programmatic dependent launch: a kernel launched with the stream-serialization attribute may become resident
// before the kernel ahead of it has finished; this is where it waits for that kernel's completion and writes
// (a no-op for an ordinary launch).
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace lq
