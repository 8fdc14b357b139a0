// Workgroups of a launch that count themselves in, so that the last one can go on with what all of them left.
#pragma once
#include "common.hpp"

namespace scmoe {

// Another number, never zero, for every call that uses one (call_number).
unsigned long long next_call();

// Marks workgroup `mine` of `all` as done and says whether all are (called by one whole wave; its earlier stores have been
// performed).  The last one to be marked sees all marks; others may as well.  A mark is the number of the call (call_number),
// another one for every call, because the memory is the caller's and not cleared: whatever lies there counts as a mark only if
// it is that number, which for other data has a probability of 2^-64 a mark and which no other call of the process has.
// A replayed graph has the same number again, so whoever saw all marks clears them.
__device__ __forceinline__ bool all_arrived(unsigned long long* marks, unsigned long long call, int mine, int all) {
  const int lane = threadIdx.x & 63;
  if (lane == 0) __hip_atomic_store(marks + mine, call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  bool there = true;
  for (int i = lane; i < all; i += 64) there = there && __hip_atomic_load(marks + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == call;
  return __all(there);
}

}  // namespace scmoe
