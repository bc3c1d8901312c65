// heddle_launch.cuh -- the device side of programmatic dependent launches.
#pragma once

namespace hd {

// A kernel launched so may start while the previous kernel of its stream still
// runs, once every CTA of that one has called allow_dependents (or exited);
// await_previous returns when the previous kernel has completed and its writes
// are visible (at once when the kernel was launched the ordinary way).  What
// the previous kernels write is read by ordinary loads and bulk copies only:
// the wait does not order the read-only path (__ldg).
__device__ __forceinline__ void allow_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

}  // namespace hd
