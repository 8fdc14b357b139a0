// Gradient of the output decode, y = c0 base + c1 sum_j w_j y_perm[r_j] (+ residual, whose gradient is dy itself):
//
//   dy_perm[r_j] = c1 w_j dy,  dw_j = c1 <dy, y_perm[r_j]>,  dbase = c0 dy,  dc0 = <dy, base>,  dc1 = sum_j w_j <dy, y_perm[r_j]>
//
// Every packed row belongs to one (token, choice), so a token's wave writes its rows without atomics.  Bound by HBM: dy
// is read once for all of them.  Products and sums in fp32.  32768 tokens of 2048 in bf16, one choice: 69 us, 5.8 TB/s; 3001 of 768
// in fp32, two choices, coefficients: 12 us, 5.5 TB/s.
#include "rows.hpp"

namespace scmoe {

struct CombineGradArgs {
  const unsigned char* dy; int64_t lddy;       // strides in bytes
  const unsigned char* yp; int64_t ldyp;       // nullptr: neither dw nor dcoef is wanted
  const int32_t* dst_row; const float* gate_w;
  const unsigned char* base; int64_t ldbase;   // nullptr: no dc0
  const float* coef;                           // [T][2]; nullptr: 1, 1
  int T, pieces;
  unsigned char* dyp; int64_t lddyp;           // nullptr: not wanted; so are the others
  float* dgate_w;
  unsigned char* dbase; int64_t lddbase;
  float* dcoef;                                // [T][2]
};

// A token belongs to L lanes of a wave; PER pieces of 16 bytes per lane are in flight at a time.
template <bool BF16, int K, int L, int PER, bool ST>
__global__ __launch_bounds__(256) void combine_backward_kernel(CombineGradArgs a) {
  constexpr int NV = BF16 ? 8 : 4, TOK = 256 / L;
  const int lane = threadIdx.x % L;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * TOK + threadIdx.x / L; t < a.T; t += static_cast<int64_t>(gridDim.x) * TOK) {
    int64_t r[K];
    float w[K], dot[K + 1];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      r[j] = a.dst_row[t * K + j];
      w[j] = r[j] >= 0 ? a.gate_w[t * K + j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j <= K; ++j) dot[j] = 0.0f;
    const float c0 = a.coef == nullptr ? 1.0f : a.coef[2 * t], c1 = a.coef == nullptr ? 1.0f : a.coef[2 * t + 1];
    const unsigned char* dyr = a.dy + t * a.lddy;
    for (int p0 = lane; p0 < a.pieces; p0 += PER * L) {
      uint4 g[PER], y[K][PER], b[PER];
      int64_t at[PER];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        at[p] = static_cast<int64_t>(min(p0 + p * L, a.pieces - 1)) * 16;
        g[p] = load16<ST>(dyr + at[p]);
      }
      if (a.yp != nullptr) {
#pragma unroll
        for (int j = 0; j < K; ++j)
          if (r[j] >= 0) {
#pragma unroll
            for (int p = 0; p < PER; ++p) y[j][p] = load16<ST>(a.yp + r[j] * a.ldyp + at[p]);
          }
      }
      if (a.base != nullptr) {
#pragma unroll
        for (int p = 0; p < PER; ++p) b[p] = load16<ST>(a.base + t * a.ldbase + at[p]);
      }
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        if (p0 + p * L >= a.pieces) continue;
        float v[NV], u[NV], o[NV];
        unpack16<BF16>(g[p], v);
        if (a.base != nullptr) {
          unpack16<BF16>(b[p], u);
#pragma unroll
          for (int i = 0; i < NV; ++i) dot[K] = fmaf(v[i], u[i], dot[K]);
        }
        if (a.dbase != nullptr) {
#pragma unroll
          for (int i = 0; i < NV; ++i) o[i] = c0 * v[i];
          store16<ST>(a.dbase + t * a.lddbase + at[p], pack16<BF16>(o));
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
          if (r[j] < 0) continue;
          if (a.yp != nullptr) {
            unpack16<BF16>(y[j][p], u);
#pragma unroll
            for (int i = 0; i < NV; ++i) dot[j] = fmaf(v[i], u[i], dot[j]);
          }
          if (a.dyp != nullptr) {
            const float f = c1 * w[j];
#pragma unroll
            for (int i = 0; i < NV; ++i) o[i] = f * v[i];
            store16<ST>(a.dyp + r[j] * a.lddyp + at[p], pack16<BF16>(o));
          }
        }
      }
    }
    if (a.yp == nullptr && a.base == nullptr) continue;
#pragma unroll
    for (int j = 0; j <= K; ++j) dot[j] = wave_sum<L>(dot[j]);
    if (lane != 0) continue;
    float dc1 = 0.0f;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      if (a.dgate_w != nullptr) a.dgate_w[t * K + j] = r[j] >= 0 ? c1 * dot[j] : 0.0f;
      if (r[j] >= 0) dc1 = fmaf(w[j], dot[j], dc1);
    }
    if (a.dcoef != nullptr) {
      a.dcoef[2 * t] = dot[K];
      a.dcoef[2 * t + 1] = dc1;
    }
  }
}

constexpr int COMBINE_GRAD_MAX_GROUPS = 1 << 20;   // keeps the threads of a launch under 2^32

static int combine_backward(const CombineGradArgs& a, int dtype, int k, hipStream_t stream) {
  // Lanes of a wave share out several tokens whose rows one piece per lane covers (32768 tokens of 128, two each, bf16: 10.8 us with 16
  // lanes, 20.1 with 64), and wider rows keep no more pieces in flight than they have (32768 of 384, bf16: 15.7 us with one piece per
  // lane, 22.1 with four).  Several waves on a row gained nothing for any number of tokens.
  const int lanes = a.pieces <= 16 ? 16 : a.pieces <= 32 ? 32 : 64;
  const int64_t groups = (static_cast<int64_t>(a.T) + 256 / lanes - 1) / (256 / lanes);
  dim3 grid(static_cast<unsigned>(groups < COMBINE_GRAD_MAX_GROUPS ? groups : COMBINE_GRAD_MAX_GROUPS)), block(256);
  // (every item counts as kept)
  const int64_t rows = 1 + (a.base ? 1 : 0) + (a.dbase ? 1 : 0) + k * ((a.yp ? 1 : 0) + (a.dyp ? 1 : 0));
  const bool st = a.pieces > 128 && streams_past_caches(rows * a.T * a.pieces * 16);
#define SCMOE_COMBINE_GRAD_L(K, L, PER, ST)                                                                                    \
  do {                                                                                                                         \
    if (dtype == SCMOE_BF16) hipLaunchKernelGGL((combine_backward_kernel<true, K, L, PER, ST>), grid, block, 0, stream, a);    \
    else hipLaunchKernelGGL((combine_backward_kernel<false, K, L, PER, ST>), grid, block, 0, stream, a);                       \
  } while (0)
#define SCMOE_COMBINE_GRAD(K)                                                        \
  do {                                                                               \
    if (lanes == 16) SCMOE_COMBINE_GRAD_L(K, 16, 1, false);                          \
    else if (lanes == 32) SCMOE_COMBINE_GRAD_L(K, 32, 1, false);                     \
    else if (a.pieces <= 64) SCMOE_COMBINE_GRAD_L(K, 64, 1, false);                  \
    else if (a.pieces <= 128) SCMOE_COMBINE_GRAD_L(K, 64, 2, false);                 \
    else if (st) SCMOE_COMBINE_GRAD_L(K, 64, (K == 1 ? 4 : 2), true);                \
    else SCMOE_COMBINE_GRAD_L(K, 64, (K == 1 ? 4 : 2), false);                       \
  } while (0)
  static_assert(SCMOE_MAX_TOPK == 4, "one instantiation per k below");
  switch (k) {
    case 1: SCMOE_COMBINE_GRAD(1); break;
    case 2: SCMOE_COMBINE_GRAD(2); break;
    case 3: SCMOE_COMBINE_GRAD(3); break;
    default: SCMOE_COMBINE_GRAD(4); break;
  }
#undef SCMOE_COMBINE_GRAD
#undef SCMOE_COMBINE_GRAD_L
  return launch_status();
}

}  // namespace scmoe

extern "C" int scmoe_combine_backward(const void* dy, int64_t lddy, int32_t dtype, const void* y_perm, int64_t ldyp,
                                      const int32_t* dst_row, const float* gate_w, int32_t T, int32_t d, int32_t k, const void* base,
                                      int64_t ldbase, const float* coef, void* dy_perm, int64_t lddyp, float* dgate_w, void* dbase,
                                      int64_t lddbase, float* dcoef, void* stream) {
  using namespace scmoe;
  if (!dtype_ok(dtype)) return SCMOE_ERR_DTYPE;
  if (T < 0 || d <= 0 || d % 8 != 0) return SCMOE_ERR_SHAPE;
  if (k < 1 || k > SCMOE_MAX_TOPK) return SCMOE_ERR_ARG;
  if (T == 0) return SCMOE_OK;
  if (!dy || !dst_row || !gate_w) return SCMOE_ERR_NULL;
  if (!y_perm && (dgate_w || dcoef)) return SCMOE_ERR_NULL;
  if (dcoef && !base) return SCMOE_ERR_NULL;
  if (!view_ok(dy, lddy, d, dtype) || (y_perm && !view_ok(y_perm, ldyp, d, dtype)) || (base && !view_ok(base, ldbase, d, dtype)) ||
      (dy_perm && !view_ok(dy_perm, lddyp, d, dtype)) || (dbase && !view_ok(dbase, lddbase, d, dtype)))
    return SCMOE_ERR_SHAPE;
  const int eb = elem_bytes(dtype);
  CombineGradArgs a = {};
  a.dy = static_cast<const unsigned char*>(dy); a.lddy = lddy * eb;
  a.yp = dgate_w || dcoef ? static_cast<const unsigned char*>(y_perm) : nullptr; a.ldyp = ldyp * eb;
  a.dst_row = dst_row; a.gate_w = gate_w;
  a.base = dcoef ? static_cast<const unsigned char*>(base) : nullptr; a.ldbase = ldbase * eb;
  a.coef = coef;
  a.T = T; a.pieces = d * eb / 16;
  a.dyp = static_cast<unsigned char*>(dy_perm); a.lddyp = lddyp * eb;
  a.dgate_w = dgate_w;
  a.dbase = static_cast<unsigned char*>(dbase); a.lddbase = lddbase * eb;
  a.dcoef = dcoef;
  return combine_backward(a, dtype, k, static_cast<hipStream_t>(stream));
}
