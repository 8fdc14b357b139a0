// The gated feed-forward block for a few rows (decode steps): bound by streaming the weights.
//
// A wave has one column of the output: [g; u] of one feature, or one column of y, for up to FEW_ROWS rows of a segment.  Its 64 lanes read
// whole rows of weights, 1 KiB a load, eight loads in flight (matrix tiles read 64 bytes of 16 rows at a time, and a product of
// one row and 2048 columns has 128 of them, half of the compute units); the products are dot products of pairs on the vector ALUs, summed
// in fp32 over the lane's places, then over the lanes.  One row of d = 2048, F = 8192: 101 MB of weights in 22.7 us, 4.4 TB/s (36.1 us by matrix
// tiles).
#include "gated_tiles.hpp"

namespace scmoe {

constexpr int FEW_ROWS = 4, FEW_WAVES = 8, FEW_LOADS = 4;

struct FewArgs {
  const unsigned char* A; int64_t lda;          // rows, stride in bytes
  const unsigned char* W; int64_t ldw;          // [E, (2) N, K], stride in bytes
  unsigned char* C; int64_t ldc;
  unsigned char* pre; int64_t ldpre;            // g and u, where they are kept (nullptr: not)
  const int32_t* offsets;
  int E, N, K;
};

// One pair (bf16) or one element (fp32) of a 16-byte piece times another's, added to a sum.
template <bool F32>
__device__ __forceinline__ float few_dot(const g_u32x4& a, const g_u32x4& b, float s) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (F32) {
      s = fmaf(__uint_as_float(a[q]), __uint_as_float(b[q]), s);
    } else {
#if defined(__HIP_DEVICE_COMPILE__)
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, static_cast<uint32_t>(a[q])), __builtin_bit_cast(bf16x2_t, static_cast<uint32_t>(b[q])), s, false);
#endif
    }
  }
  return s;
}

// GATE: W has 2 N rows an expert, those of g first; C = act(g) u.  ACT as in gated_kernel.
template <bool F32, bool GATE, int ACT>
__global__ __launch_bounds__(64 * FEW_WAVES) void gated_few_kernel(const FewArgs p) {
  constexpr int EB = F32 ? 4 : 2, PARTS = GATE ? 2 : 1, U = FEW_LOADS * 2 / PARTS;      // U: pieces of a row in flight
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = blockIdx.x * FEW_WAVES + wave;

  // ---- which segment: 64 at a time, one per lane ---------------------------------------------
  int e = -1, row0 = 0, rows = 0, left = blockIdx.y;
  for (int e0 = 0; e0 < p.E && e < 0; e0 += 64) {
    const int q = e0 + lane;
    const int s = p.offsets[q < p.E ? q : p.E], t = p.offsets[q + 1 < p.E ? q + 1 : p.E];
    const int tiles = (t - s + FEW_ROWS - 1) / FEW_ROWS;         // (0 past the last segment)
    int incl = tiles;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int up = __shfl_up(incl, off, 64);
      if (lane >= off) incl += up;
    }
    const unsigned long long hit = __ballot(incl > left);
    if (hit != 0) {
      const int at = __builtin_ctzll(hit);
      e = e0 + at;
      const int first = __builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(tiles, at);
      row0 = __builtin_amdgcn_readlane(s, at) + (left - first) * FEW_ROWS;
      rows = min(__builtin_amdgcn_readlane(t, at) - row0, FEW_ROWS);
    } else {
      left -= __builtin_amdgcn_readlane(incl, 63);
    }
  }
  if (e < 0 || n >= p.N) return;

  const unsigned char* w[PARTS];
#pragma unroll
  for (int t = 0; t < PARTS; ++t) w[t] = p.W + (static_cast<int64_t>(e) * PARTS * p.N + static_cast<int64_t>(t) * p.N + n) * p.ldw;
  const unsigned char* x[FEW_ROWS];
#pragma unroll
  for (int r = 0; r < FEW_ROWS; ++r) x[r] = p.A + static_cast<int64_t>(row0 + (r < rows ? r : rows - 1)) * p.lda;
  float sum[PARTS][FEW_ROWS];
#pragma unroll
  for (int t = 0; t < PARTS; ++t)
#pragma unroll
    for (int r = 0; r < FEW_ROWS; ++r) sum[t][r] = 0.0f;
  const uint32_t bytes = static_cast<uint32_t>(p.K) * EB;
  auto body = [&](auto rows_c) {
    constexpr int R = decltype(rows_c)::value;
    for (uint32_t k = 0; k < bytes; k += U * 1024) {
      g_u32x4 wv[PARTS][U], xv[R][U];
      // (past a row's end: zeros)
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const uint32_t at = k + i * 1024 + lane * 16, off = at < bytes ? at : BUFFER_NOWHERE;
#pragma unroll
        for (int t = 0; t < PARTS; ++t) wv[t][i] = buffer_get<g_u32x4>(w[t], off, 0);
#pragma unroll
        for (int r = 0; r < R; ++r) xv[r][i] = buffer_get<g_u32x4>(x[r], off, 0);
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int t = 0; t < PARTS; ++t)
#pragma unroll
          for (int r = 0; r < R; ++r) sum[t][r] = few_dot<F32>(wv[t][i], xv[r][i], sum[t][r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float v[PARTS];
#pragma unroll
      for (int t = 0; t < PARTS; ++t) v[t] = wave_sum<64>(sum[t][r]);
      if (lane == 0 && r < rows) {
        auto put = [&](unsigned char* base, int64_t ld, int col, float y) {
          unsigned char* const to = base + static_cast<int64_t>(row0 + r) * ld + static_cast<int64_t>(col) * EB;
          if constexpr (F32) *reinterpret_cast<float*>(to) = y;
          else *reinterpret_cast<uint16_t*>(to) = f32_to_bf16(y);
        };
        if constexpr (GATE) {
          put(p.C, p.ldc, n, gated_act<F32, ACT>(v[0]) * v[PARTS - 1]);
          if (p.pre != nullptr) {
            put(p.pre, p.ldpre, n, v[0]);
            put(p.pre, p.ldpre, p.N + n, v[PARTS - 1]);
          }
        } else {
          put(p.C, p.ldc, n, v[0]);
        }
      }
    }
  };
  if (rows == 1) body(std::integral_constant<int, 1>{});
  else if (rows == 2) body(std::integral_constant<int, 2>{});
  else body(std::integral_constant<int, FEW_ROWS>{});
}

template <bool F32, bool GATE>
static int launch_few(const GatedArgs& a, int keep, int64_t max_rows, hipStream_t stream) {
  constexpr int EB = F32 ? 4 : 2;
  const GatedJob& j = a.j[0];
  FewArgs f{};
  f.A = j.A; f.lda = j.lda * EB;
  f.W = j.B; f.ldw = j.ldb * EB;
  f.C = j.C; f.ldc = j.ldc * EB;
  if (GATE && keep == KEEP_FULL) { f.pre = a.pre; f.ldpre = a.ldpre * EB; }
  f.offsets = a.offsets; f.E = a.E; f.N = j.N; f.K = j.Kd;
  const int64_t tiles = max_rows / FEW_ROWS + (a.E < max_rows ? a.E : max_rows);
  const dim3 grid(static_cast<unsigned>((j.N + FEW_WAVES - 1) / FEW_WAVES), static_cast<unsigned>(tiles)), block(64 * FEW_WAVES);
  if (!GATE || a.act == SCMOE_SILU) hipLaunchKernelGGL((gated_few_kernel<F32, GATE, SCMOE_SILU>), grid, block, 0, stream, f);
  else if (a.act == SCMOE_GELU_TANH) hipLaunchKernelGGL((gated_few_kernel<F32, GATE, SCMOE_GELU_TANH>), grid, block, 0, stream, f);
  else hipLaunchKernelGGL((gated_few_kernel<F32, GATE, SCMOE_GELU_ERF>), grid, block, 0, stream, f);
  return launch_status();
}

int launch_gated_few(const GatedArgs& a, int mode, int keep, int64_t max_rows, int dtype, hipStream_t stream) {
  if (mode == G_GATE) return dtype == SCMOE_BF16 ? launch_few<false, true>(a, keep, max_rows, stream) : launch_few<true, true>(a, keep, max_rows, stream);
  return dtype == SCMOE_BF16 ? launch_few<false, false>(a, keep, max_rows, stream) : launch_few<true, false>(a, keep, max_rows, stream);
}

}  // namespace scmoe
