// Adds up the partial sums that the workgroups of a gradient kernel leave in the workspace.  A second launch in
// place of floating-point atomics: the order of the sum is fixed, so the gradient has the same bits in every run.
#include "common.hpp"

namespace scmoe {

constexpr int SUM_SLICES = 64;   // threads that share a column group, each with every 64th part
constexpr int SUM_QUADS = 4;     // 16-byte column groups per workgroup: 64 bytes of every part

// parts: [n][stride] fp32, stride a multiple of 4.  Columns [0, na) go to a, columns [na, na + nb) to b.
__global__ __launch_bounds__(SUM_SLICES * SUM_QUADS) void sum_parts_kernel(const float* __restrict__ parts, int n, int64_t stride,
                                                                           float* __restrict__ a, int64_t na, float* __restrict__ b,
                                                                           int64_t nb) {
  __shared__ float4 s[SUM_SLICES * SUM_QUADS / 64][SUM_QUADS];
  const int quad = threadIdx.x % SUM_QUADS, slice = threadIdx.x / SUM_QUADS;
  const int64_t col = (static_cast<int64_t>(blockIdx.x) * SUM_QUADS + quad) * 4;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (col < stride) {
#pragma unroll 8
    for (int i = slice; i < n; i += SUM_SLICES) {
      const float4 q = *reinterpret_cast<const float4*>(parts + i * stride + col);
      v.x += q.x;
      v.y += q.y;
      v.z += q.z;
      v.w += q.w;
    }
  }
  // over the 16 slices of a wave, whose lanes of a quad are 4 apart, then over the waves
#pragma unroll
  for (int off = SUM_QUADS; off < 64; off <<= 1) {
    v.x += __shfl_xor(v.x, off, 64);
    v.y += __shfl_xor(v.y, off, 64);
    v.z += __shfl_xor(v.z, off, 64);
    v.w += __shfl_xor(v.w, off, 64);
  }
  if ((threadIdx.x & 63) < SUM_QUADS) s[threadIdx.x >> 6][quad] = v;
  __syncthreads();
  if (threadIdx.x >= 4 * SUM_QUADS) return;
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * SUM_QUADS * 4) + threadIdx.x;
  float r = 0.0f;
#pragma unroll
  for (int w = 0; w < SUM_SLICES * SUM_QUADS / 64; ++w) r += reinterpret_cast<const float*>(s[w])[threadIdx.x];
  if (c < na) {
    if (a != nullptr) a[c] = r;
  } else if (c < na + nb) {
    if (b != nullptr) b[c - na] = r;
  }
}

int sum_parts(const float* parts, int n, int64_t stride, float* a, int64_t na, float* b, int64_t nb, hipStream_t stream) {
  const int64_t quads = (na + nb + 3) / 4;
  dim3 grid(static_cast<unsigned>((quads + SUM_QUADS - 1) / SUM_QUADS)), block(SUM_SLICES * SUM_QUADS);
  hipLaunchKernelGGL(sum_parts_kernel, grid, block, 0, stream, parts, n, stride, a, na, b, nb);
  return launch_status();
}

}  // namespace scmoe
