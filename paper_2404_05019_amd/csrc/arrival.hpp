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

// Data handed from one workgroup to another inside a launch: device scope, past the caches that are not shared.
template <typename V>
__device__ __forceinline__ void leave(V* p, V v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V>
__device__ __forceinline__ V left_there(const V* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The same for a whole workgroup that has left its part: true in every thread of the last one (of several, if so), which clears the
// marks.  `flag` is one int of LDS.
__device__ __forceinline__ bool last_to_arrive(unsigned long long* marks, unsigned long long call, int mine, int all, int* flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // what this wave left is where every workgroup sees it
  __syncthreads();                                        // ... and every wave's
  if (threadIdx.x < 64) {
    const bool there = all_arrived(marks, call, mine, all);
    if (threadIdx.x == 0) *flag = there;
  }
  __syncthreads();
  if (*flag == 0) return false;                           // (two may find all the others done: they write the same)
  for (int i = threadIdx.x; i < all; i += blockDim.x) leave(marks + i, 0ull);
  return true;
}

// Sum over `n` parts, `stride` floats apart, of the two floats at each; in their order, N loads in flight together (the last of them
// again where there are no more: a loop over a remainder would wait for each).  A load past the caches costs also where it is repeated:
// with N to fit 512 rows of 512 took 9.2 us a call, with 32 for any number 10.5.
template <int N>
__device__ __forceinline__ void add_left(const float* part, int n, int64_t stride, float2& v) {
  unsigned long long q[N];
#pragma unroll
  for (int i = 0; i < N; ++i) q[i] = left_there(reinterpret_cast<const unsigned long long*>(part + min(i, n - 1) * stride));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v.x += i < n ? __uint_as_float(static_cast<uint32_t>(q[i])) : 0.0f;
    v.y += i < n ? __uint_as_float(static_cast<uint32_t>(q[i] >> 32)) : 0.0f;
  }
}

constexpr int MOST_LEFT = 32;          // parts that sum_left takes

// MOST: the largest n of the caller's, 8 or MOST_LEFT.
template <int MOST>
__device__ __forceinline__ float2 sum_left(const float* part, int n, int64_t stride) {
  static_assert(MOST == 8 || MOST == MOST_LEFT);
  float2 v = make_float2(0.0f, 0.0f);
  if (n <= 4) add_left<4>(part, n, stride, v);
  else if (MOST == 8 || n <= 8) add_left<8>(part, n, stride, v);
  else if (n <= 16) add_left<16>(part, n, stride, v);
  else add_left<MOST>(part, n, stride, v);
  return v;
}

__device__ __forceinline__ void leave2(float* p, float x, float y) {
  leave(reinterpret_cast<unsigned long long*>(p), static_cast<unsigned long long>(__float_as_uint(y)) << 32 | __float_as_uint(x));
}

}  // namespace scmoe
