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

// STREAM: past what the caches keep for others (no other use is expected before newer data take its place).
template <bool STREAM = false>
__device__ __forceinline__ uint4 load16(const unsigned char* p) {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  if (!STREAM) return *reinterpret_cast<const uint4*>(p);
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool STREAM = false>
__device__ __forceinline__ void store16(unsigned char* p, const uint4& q) {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  if (!STREAM) *reinterpret_cast<uint4*>(p) = q;
  else __builtin_nontemporal_store(u32x4_t{q.x, q.y, q.z, q.w}, reinterpret_cast<u32x4_t*>(p));
}

// Calls that move more than the 256 MB that the device's last cache holds use streaming loads and stores (a copy of 1 GB ran at 5.8 TB/s
// without and 6.3 with them).  us a call without / with them:
//                                                              128 MB          256 MB          320 MB          512 MB
//   norm of 1024 columns, residual, bf16                    23.7 / 25.0     43.8 / 46.9     64.9 / 57.4     99.3 / 92.3
//   its gradient, fp32                                      27.8 / 28.3     48.2 / 50.2     66.7 / 61.5      104 / 94.3
//   decode's gradient of 2048 columns, one choice, bf16     23.8 / 25.1     43.9 / 50.9     63.8 / 63.5      107 / 103
//   gate's gradient with encode of 1024, bf16, 8 experts    31.7 / 34.7     53.7 / 58.0     74.0 / 70.6      120 / 108
//                                             32 experts    40.6 / 45.5     66.8 / 69.3     85.9 / 82.5      129 / 121
//                                             64 experts    74.5 / 78.0      129 / 129       156 / 154       233 / 230
//                                       fp32, 64 experts    64.8 / 67.3      100 / 100       121 / 119       172 / 170
// Not built with them: norm and its gradient with less than a wave a row (up to 32 pieces of 16 bytes), the decode's gradient up to 128
// pieces.  Those would gain 3 to 9 % past 256 MB (384 MB of rows of 128 in bf16: norm 74.3 / 69.5, its gradient 78.7 / 73.2, decode's
// gradient 82.3 / 77.7).
inline bool streams_past_caches(int64_t bytes) { return bytes > (static_cast<int64_t>(256) << 20); }

__device__ __forceinline__ uint4 zero_unless(bool keep, const uint4& q) {
  return make_uint4(keep ? q.x : 0u, keep ? q.y : 0u, keep ? q.z : 0u, keep ? q.w : 0u);
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over L neighbouring lanes (16, 32 or all 64 of the wave, all of them active), in every one of them: within rows of 16 lanes by the
// vector unit's lane moves (neighbour, pair, mirrored 8, mirrored 16), which cost no trip to the LDS, then over the rows.
template <int L = 64>
__device__ __forceinline__ float wave_sum(float v) {
  static_assert(L == 16 || L == 32 || L == 64);
  v = dpp_add<0xB1>(v);
  v = dpp_add<0x4E>(v);
  v = dpp_add<0x141>(v);
  v = dpp_add<0x140>(v);
  if (L == 16) return v;
  if (L == 32) return v + __shfl_xor(v, 16, 64);
  const int b = __float_as_int(v);
  const float r0 = __int_as_float(__builtin_amdgcn_readlane(b, 0)), r1 = __int_as_float(__builtin_amdgcn_readlane(b, 16));
  const float r2 = __int_as_float(__builtin_amdgcn_readlane(b, 32)), r3 = __int_as_float(__builtin_amdgcn_readlane(b, 48));
  return (r0 + r1) + (r2 + r3);
}

// Waits for every load in flight, ahead of stores: where what was loaded ahead is due in the next turn of a loop, the wait the compiler
// puts there would be one for the stores as well (one counter has both, and a store under a condition cannot be counted off).
__device__ __forceinline__ void loads_have_arrived() {
  __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
}

// Between a wave's LDS writes and its reads of what other lanes of it wrote (the LDS serves a wave in order; this
// keeps the compiler to that order).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace scmoe
