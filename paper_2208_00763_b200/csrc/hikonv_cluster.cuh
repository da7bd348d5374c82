// Barriers of thread-block clusters.
#pragma once

namespace hikonv {

// Not the .aligned forms: those want all threads of a warp at the instruction together, and the code in front of them has branches that the
// threads of a warp take apart.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

}  // namespace hikonv
