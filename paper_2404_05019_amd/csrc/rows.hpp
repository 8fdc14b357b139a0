// Rows of activations as 16-byte pieces in registers, and sums over the lanes of a wave: shared by the kernels
// that walk rows (layer norm, gradients of the gate and of the output decode).
#pragma once
#include "common.hpp"
#include "mfma_common.hpp"

namespace scmoe {

// 16 bytes of a row: 8 bf16 or 4 fp32 values.
template <bool BF16>
__device__ __forceinline__ void unpack16(const uint4& q, float* v) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  if (BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  }
}

// Rounded to nearest even where the type has fewer bits.
template <bool BF16>
__device__ __forceinline__ uint4 pack16(const float* v) {
  if (BF16) return make_uint4(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7]));
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

__device__ __forceinline__ uint4 load16(const unsigned char* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void store16(unsigned char* p, const uint4& q) { *reinterpret_cast<uint4*>(p) = q; }

__device__ __forceinline__ uint4 zero_unless(bool keep, const uint4& q) {
  return make_uint4(keep ? q.x : 0u, keep ? q.y : 0u, keep ? q.z : 0u, keep ? q.w : 0u);
}

// Sum over the 64 lanes, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Between a wave's LDS writes and its reads of what other lanes of it wrote (the LDS serves a wave in order; this
// keeps the compiler to that order).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace scmoe
