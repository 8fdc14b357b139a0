// Activation checkpoints in 8 bits: how a row is laid out, and a value's way there and back.
//
// A row of w columns: w codes of one byte (4 bits of exponent, 3 of mantissa), then ceil(w / 32) bytes of scale, one for every 32
// columns.  A block's scale is the least power of two s, of at least 2^-126, with max |x| <= 448 s, stored as its exponent plus 127,
// so x / s and code * s are exact: all that is lost is the rounding of the code, half of 2^-3 of the value (or half of
// 2^-9 s for small ones; s is under max |x| / 224).  A block with an infinity or NaN: scale byte 255, all its codes NaN.
#pragma once
#include "common.hpp"

namespace scmoe {

constexpr int CKPT_BLOCK = 32;
constexpr int64_t ckpt_bytes(int64_t w) { return w + (w + CKPT_BLOCK - 1) / CKPT_BLOCK; }      // of a row
inline bool ckpt_view_ok(const void* p, int64_t ld, int64_t w) { return aligned16(p) && ld >= ckpt_bytes(w) && ld % 16 == 0; }

// Scale byte of a block from the bits of its largest magnitude (an integer comparison orders magnitudes, infinities and NaN).
// 448 = 1.75 * 2^8: the exponent less 8, and one more where the mantissa is above 1.75.
__device__ __forceinline__ uint32_t ckpt_scale_byte(uint32_t most) {
  const int e = static_cast<int>(most >> 23);
  if (e == 255) return 255;
  const int b = e - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < 1 ? 1 : b;
}
// 1 / s; a block without finite scale: NaN, which makes every code one.
__device__ __forceinline__ float ckpt_inverse(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7fc00000u : (254u - byte) << 23); }
__device__ __forceinline__ float ckpt_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four codes, first in the low byte.
__device__ __forceinline__ uint32_t ckpt_encode4(float a, float b, float c, float d, float inverse) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, r, true);
  return static_cast<uint32_t>(r);
}
__device__ __forceinline__ void ckpt_decode4(uint32_t codes, float scale, float* v) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  v[0] = lo[0] * scale;
  v[1] = lo[1] * scale;
  v[2] = hi[0] * scale;
  v[3] = hi[1] * scale;
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// What a kernel of this library asks of both (checkpoint.hip): rows of activations into checkpoint rows and back.  n_rows: how many of
// max_rows, on the device (nullptr: all).
int checkpoint_pack(const void* x, int64_t ldx, int dtype, const int32_t* n_rows, int64_t max_rows, int width, void* q, int64_t ldq, hipStream_t stream);
int checkpoint_unpack(const void* q, int64_t ldq, const int32_t* n_rows, int64_t max_rows, int width, void* x, int64_t ldx, int dtype, hipStream_t stream);

}  // namespace scmoe
