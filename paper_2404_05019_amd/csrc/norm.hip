// Layer norm over the model width and its gradient.
//
//   mean = sum(h) / d,  rstd = (sum((h - mean)^2) / d + eps)^(-1/2),  xh = (h - mean) rstd,  y = xh gamma + beta
//   g = dy gamma:  dh = rstd (g - sum(g) / d - xh sum(g xh) / d);  dgamma = sum over rows of dy xh;  dbeta = sum of dy
//
// Bound by HBM: a row is read once, kept in registers (the squares are summed about the mean in a second walk over
// them, so that a large mean costs no digits) and written once.  All arithmetic in fp32.  32768 rows of 2048 in bf16 with
// residual and statistics: 91 us, 5.9 TB/s (a copy of 1 GB in the same way: 6.3); the gradient of 16384 rows of 1024 with the
// residual's: 28 us, 4.8 TB/s, and 4 us for adding up the parts.  A call of few rows is bound by its launch (3 us on the device).
#include "arrival.hpp"
#include "rows.hpp"

namespace scmoe {

struct NormArgs {
  const unsigned char* x; int64_t ldx;           // strides in bytes
  const unsigned char* residual; int64_t ldres;  // added to x; nullptr: none
  unsigned char* sum; int64_t ldsum;
  const float* gamma; const float* beta;         // nullptr: 1, 0
  float eps;
  int T, d;
  unsigned char* y; int64_t ldy;
  float* mean; float* rstd;                      // nullptr: not kept
};

struct NormGradArgs {
  const unsigned char* dy; int64_t lddy;         // strides in bytes
  const unsigned char* x; int64_t ldx;
  const float* gamma; const float* mean; const float* rstd;
  const unsigned char* dsum; int64_t lddsum;     // added to the gradient; nullptr: none
  int T, d;
  unsigned char* dx; int64_t lddx;
  float* parts; int64_t stride;                  // one part per workgroup: dgamma [d], dbeta [d]; nullptr: neither is wanted
  // In one launch (else both nullptr): the last workgroup adds up the parts.  One workgroup: marks is not used.
  float* dgamma; float* dbeta;
  int one_launch;
  unsigned long long* marks; unsigned long long call;   // (all_arrived)
};

// A row belongs to W waves, or to L lanes of one (16 and 32: narrow rows), a lane to V of its values (V / 8 or V / 4 pieces of 16
// bytes, L W pieces apart).  W = 1: several rows per workgroup and no barrier.
constexpr int norm_threads(int W) { return W == 1 ? 256 : 64 * W; }

// Sums of two values over the waves of a row.  Calls that follow each other use places `s` of their own: one barrier is enough.
template <int W, int L>
__device__ __forceinline__ void row_sums(float& a, float& b, float2 (&s)[W]) {
  a = wave_sum<L>(a);
  b = wave_sum<L>(b);
  if (W > 1) {
    if ((threadIdx.x & 63) == 0) s[threadIdx.x / 64 % W] = make_float2(a, b);
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float2 p = s[w];
      a += p.x;
      b += p.y;
    }
  }
}

template <bool BF16, int V, int W, bool ST, int L = 64>
__global__ __launch_bounds__(norm_threads(W)) void layer_norm_kernel(NormArgs a) {
  constexpr int NV = BF16 ? 8 : 4, P = V / NV, STEP = L * W, ROWS = W == 1 ? 256 / L : 1;
  __shared__ float2 s[2][W];
  const int lane = threadIdx.x % STEP;
  const int pieces = a.d / NV;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / STEP; row < a.T; row += static_cast<int64_t>(gridDim.x) * ROWS) {
    uint4 q[P];
#pragma unroll
    for (int p = 0; p < P; ++p) q[p] = load16<ST>(a.x + row * a.ldx + static_cast<int64_t>(min(lane + p * STEP, pieces - 1)) * 16);
    if (a.residual != nullptr) {
      uint4 r[P];
#pragma unroll
      for (int p = 0; p < P; ++p) r[p] = load16<ST>(a.residual + row * a.ldres + static_cast<int64_t>(min(lane + p * STEP, pieces - 1)) * 16);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float v[NV], u[NV];
        unpack16<BF16>(q[p], v);
        unpack16<BF16>(r[p], u);
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] += u[i];
        q[p] = pack16<BF16>(v);       // what is normed is what is stored: the backward pass reads the stored sum
        if (lane + p * STEP < pieces) store16<ST>(a.sum + row * a.ldsum + static_cast<int64_t>(lane + p * STEP) * 16, q[p]);
      }
    }
    float v[V];
    float sum = 0.0f, none = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      unpack16<BF16>(zero_unless(lane + p * STEP < pieces, q[p]), v + p * NV);
#pragma unroll
      for (int i = 0; i < NV; ++i) sum += v[p * NV + i];
    }
    row_sums<W, L>(sum, none, s[0]);
    const float inv = 1.0f / static_cast<float>(a.d);
    const float mean = sum * inv;
    float sq = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const bool in = lane + p * STEP < pieces;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float c = v[p * NV + i] - mean;
        v[p * NV + i] = c;
        sq += in ? c * c : 0.0f;
      }
    }
    row_sums<W, L>(sq, none, s[1]);
    const float rstd = 1.0f / sqrtf(sq * inv + a.eps);
    if (lane == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = lane + p * STEP;
      if (c >= pieces) continue;
      float o[NV];
#pragma unroll
      for (int i = 0; i < NV; i += 4) {
        const float4 g = a.gamma == nullptr ? make_float4(1.0f, 1.0f, 1.0f, 1.0f) : *reinterpret_cast<const float4*>(a.gamma + c * NV + i);
        const float4 b = a.beta == nullptr ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : *reinterpret_cast<const float4*>(a.beta + c * NV + i);
        const float* t = v + p * NV + i;
        o[i] = fmaf(t[0] * rstd, g.x, b.x);
        o[i + 1] = fmaf(t[1] * rstd, g.y, b.y);
        o[i + 2] = fmaf(t[2] * rstd, g.z, b.z);
        o[i + 3] = fmaf(t[3] * rstd, g.w, b.w);
      }
      store16<ST>(a.y + row * a.ldy + static_cast<int64_t>(c) * 16, pack16<BF16>(o));
    }
  }
}

// Of a row of the gradient: x, dy, dsum, and its mean and 1 / deviation.
template <int P>
struct NormGradRow {
  uint4 x[P], y[P], s[P];
  float mean, rstd;
};

template <int P, int STEP, bool ST, bool DSUM>
__device__ __forceinline__ void norm_grad_load(const NormGradArgs& a, int64_t row, int lane, int pieces, NormGradRow<P>& r) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t c = static_cast<int64_t>(min(lane + p * STEP, pieces - 1)) * 16;
    r.x[p] = load16<ST>(a.x + row * a.ldx + c);
    r.y[p] = load16<ST>(a.dy + row * a.lddy + c);
    if (DSUM && a.dsum != nullptr) r.s[p] = load16<ST>(a.dsum + row * a.lddsum + c);
  }
  r.mean = a.mean[row];
  r.rstd = a.rstd[row];
}

// gamma of the columns of piece c.
template <int NV>
__device__ __forceinline__ void norm_grad_gamma(const NormGradArgs& a, int c, float* g) {
#pragma unroll
  for (int i = 0; i < NV; i += 4) {
    const float4 t = a.gamma == nullptr ? make_float4(1.0f, 1.0f, 1.0f, 1.0f) : *reinterpret_cast<const float4*>(a.gamma + c * NV + i);
    g[i] = t.x;
    g[i + 1] = t.y;
    g[i + 2] = t.z;
    g[i + 3] = t.w;
  }
}

// Columns 4 i and on of [dgamma, dbeta] of the whole call.
__device__ __forceinline__ void norm_grad_put(const NormGradArgs& a, int i, const float4& v) {
  float* const to = 4 * i < a.d ? a.dgamma : a.dbeta;
  if (to == nullptr) return;
  const int c = 4 * i < a.d ? 4 * i : 4 * i - a.d;
  to[c] = v.x;
  to[c + 1] = v.y;
  to[c + 2] = v.z;
  to[c + 3] = v.w;
}

// ... of this workgroup's part.
__device__ __forceinline__ void norm_grad_leave(const NormGradArgs& a, int i, const float4& v) {
  float* const part = a.parts + blockIdx.x * a.stride + 4 * i;
  if (!a.one_launch) {
    *reinterpret_cast<float4*>(part) = v;
  } else if (gridDim.x == 1) {
    norm_grad_put(a, i, v);
  } else {
    leave2(part, v.x, v.y);
    leave2(part + 2, v.z, v.w);
  }
}

// A workgroup has R rows at a time, W waves each, and takes every gridDim.x-th group of R; a lane's columns are the same in all of
// them, so dgamma and dbeta are summed in registers and leave as one part per workgroup.  Where there are registers for it the
// next row is loaded before this one is worked on.
template <bool BF16, int V, int W, int R, bool ST, int L = 64>
__global__ __launch_bounds__(64 * W * R, 2) void layer_norm_backward_kernel(NormGradArgs a) {
  constexpr int NV = BF16 ? 8 : 4, P = V / NV, STEP = L * W, H = NV / 4, AREAS = W <= 2 ? 2 : 1, ROWS = R * (64 / L);
  constexpr bool AHEAD = P <= 2;
  // 32 values of x, of dy and of both sums leave no registers for gamma as well, in fp32 neither for dsum: they are read where they are
  // used (all kept, 2048 rows of 16384 with dsum took 200 us in place of 136 in fp32 and spilled in bf16 too)
  constexpr bool WIDE = V > 16, LATE = WIDE && !BF16;
  __shared__ float2 s[2][R][W];
  __shared__ int last_one;
  extern __shared__ __attribute__((aligned(16))) float4 cols[];  // R > 1: AREAS of [dgamma, dbeta][half][piece]
  const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W));   // of the R
  const int mine = L == 64 ? slot : static_cast<int>(threadIdx.x / STEP);     // this lane's row of the ROWS
  const int lane = threadIdx.x - mine * STEP;
  const int pieces = a.d / NV;
  const float inv = 1.0f / static_cast<float>(a.d);
  const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS, last = a.T - 1;
  int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + mine;
  NormGradRow<P> n;
  if (AHEAD) norm_grad_load<P, STEP, ST, !LATE>(a, row < a.T ? row : last, lane, pieces, n);
  float g[WIDE ? NV : V], ag[V], ab[V];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (!WIDE) norm_grad_gamma<NV>(a, min(lane + p * STEP, pieces - 1), g + p * NV);
#pragma unroll
    for (int i = 0; i < NV; ++i) ag[p * NV + i] = ab[p * NV + i] = 0.0f;
  }
  int turn = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * ROWS; first < a.T; first += step, row += step) {               // (as many turns for every wave of the workgroup)
    const bool live = row < a.T;
    NormGradRow<P> q;
    if (AHEAD) {
      q = n;
      norm_grad_load<P, STEP, ST, !LATE>(a, row + step < a.T ? row + step : last, lane, pieces, n);
    } else {
      norm_grad_load<P, STEP, ST, !LATE>(a, live ? row : last, lane, pieces, q);
    }
    if (!live) q.mean = q.rstd = 0.0f;                  // (a row that is there for the barrier adds zeros, whatever the last row holds)
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const bool in = live && lane + p * STEP < pieces;
      float x[NV], y[NV];
      const uint4 qx = zero_unless(in, q.x[p]), qy = zero_unless(in, q.y[p]);
      if (WIDE) {                                       // (one copy of them)
        q.x[p] = qx;
        q.y[p] = qy;
      }
      unpack16<BF16>(qx, x);
      unpack16<BF16>(qy, y);
      if (WIDE) norm_grad_gamma<NV>(a, min(lane + p * STEP, pieces - 1), g);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float xh = (x[i] - q.mean) * q.rstd, gy = y[i] * g[WIDE ? i : p * NV + i];
        s1 += gy;
        s2 = fmaf(gy, xh, s2);
        ag[p * NV + i] = fmaf(y[i], xh, ag[p * NV + i]);
        ab[p * NV + i] += y[i];
      }
    }
    row_sums<W, L>(s1, s2, s[turn][slot]);
    turn ^= 1;
    s1 *= inv;
    s2 *= inv;
    if (AHEAD) loads_have_arrived();
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = lane + p * STEP;
      float x[NV], y[NV], r[NV];
      unpack16<BF16>(q.x[p], x);
      unpack16<BF16>(q.y[p], y);
      if (WIDE) norm_grad_gamma<NV>(a, min(c, pieces - 1), g);
      if (LATE) {
        if (a.dsum != nullptr) q.s[p] = load16<ST>(a.dsum + (live ? row : last) * a.lddsum + static_cast<int64_t>(min(c, pieces - 1)) * 16);
      }
      if (a.dsum != nullptr) {
        unpack16<BF16>(q.s[p], r);
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) r[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float xh = (x[i] - q.mean) * q.rstd;
        r[i] = fmaf(q.rstd, (y[i] * g[WIDE ? i : p * NV + i] - s1) - xh * s2, r[i]);
      }
      if (live && c < pieces) store16<ST>(a.dx + row * a.lddx + static_cast<int64_t>(c) * 16, pack16<BF16>(r));
    }
  }
  if (a.parts == nullptr) return;
  const int half = a.d / 4;                             // float4 of dgamma; dbeta lies behind
  if (R > 1) {
    // The rows' waves hold sums of the same columns: every AREAS-th row's are added up in one area, in their order.  A lane's 4 or 8
    // columns lie in two halves, so that neighbouring lanes use neighbouring banks.
    float4* const area = cols + slot % AREAS * 2 * half;
    if (L < 64) {                                       // the rows of one wave first
#pragma unroll
      for (int off = L; off < 64; off <<= 1)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          ag[i] += __shfl_xor(ag[i], off, 64);
          ab[i] += __shfl_xor(ab[i], off, 64);
        }
    }
    for (int w = 0; w < (R + AREAS - 1) / AREAS; ++w) {
      if (slot / AREAS == w) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int c = lane + p * STEP;
          if (c >= pieces || (L < 64 && (threadIdx.x & 63) >= L)) continue;
#pragma unroll
          for (int h = 0; h < H; ++h) {
            const float* const u = ag + p * NV + 4 * h;
            const float* const v = ab + p * NV + 4 * h;
            float4 x = make_float4(u[0], u[1], u[2], u[3]), y = make_float4(v[0], v[1], v[2], v[3]);
            if (w > 0) {
              const float4 m = area[h * pieces + c], b = area[half + h * pieces + c];
              x = make_float4(m.x + x.x, m.y + x.y, m.z + x.z, m.w + x.w);
              y = make_float4(b.x + y.x, b.y + y.y, b.z + y.z, b.w + y.w);
            }
            area[h * pieces + c] = x;
            area[half + h * pieces + c] = y;
          }
        }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < 2 * half; i += 64 * W * R) {
      const int k = i < half ? i : i - half;
      const int at = i - k + (k % H) * pieces + k / H;
      float4 x = cols[at];
      if (AREAS > 1) {
        const float4 y = cols[2 * half + at];
        x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
      }
      norm_grad_leave(a, i, x);
    }
  } else {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = lane + p * STEP;
      if (c >= pieces) continue;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const float* const u = ag + p * NV + 4 * h;
        const float* const v = ab + p * NV + 4 * h;
        norm_grad_leave(a, c * H + h, make_float4(u[0], u[1], u[2], u[3]));
        norm_grad_leave(a, half + c * H + h, make_float4(v[0], v[1], v[2], v[3]));
      }
    }
  }
  if (!a.one_launch || gridDim.x == 1 || !last_to_arrive(a.marks, a.call, blockIdx.x, gridDim.x, &last_one)) return;
  for (int i = threadIdx.x; i < a.d; i += 64 * W * R) {
    const float2 v = sum_left<MOST_LEFT>(a.parts + 2 * i, gridDim.x, a.stride);
    float* const to = 2 * i < a.d ? a.dgamma : a.dbeta;
    if (to == nullptr) continue;
    to[2 * i < a.d ? 2 * i : 2 * i - a.d] = v.x;
    to[(2 * i < a.d ? 2 * i : 2 * i - a.d) + 1] = v.y;
  }
}

// Lanes of a row: fewer than a wave where one piece of 16 bytes per lane covers it.  32768 rows of 128 in bf16 with their residual: 9.1 us
// with 16 lanes and 13.0 with 64, the gradient 13.5 and 19.5.
static int norm_lanes(int d, int dtype) {
  const int pieces = d / vec_elems(dtype);
  return pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
}

// Rows of a workgroup of the backward kernel, eight waves in all.  (Twelve, three a SIMD, took 30.2 us in place of 28.5 for 16384
// rows of 1024: more of them wait for the last turn.)
static int norm_grad_rows(int d, int dtype) {
  const int lanes = norm_lanes(d, dtype);
  return lanes < 64 ? 8 * (64 / lanes) : d <= 1024 ? 8 : d <= 2048 ? 4 : d <= 4096 ? 2 : 1;
}

// One workgroup per compute unit, each with a part of 8 d bytes to leave, which a second launch adds up, but for calls of few rows:
//  - up to four groups of narrow rows, two of rows up to 8192 wide and one of wider ones are one workgroup's, which writes the sums itself;
//  - up to MOST_LEFT parts of a narrow row's columns, 64 KB in all, are added up by the last workgroup of the one launch.
// us a call in a replayed graph / called back to back from Python / waited for one by one, bf16 (fp32 alike), against two launches:
//   2 turns of one workgroup     64 columns 4.8 / 9.1 / 20.4 (6.3 / 12.0 / 22.6), 2048 6.0 / 9.1 / 21.6 (7.0 / 12.2 / 22.9)
//                                fp32: 8192 columns 6.4 / 8.4 / 21.4 (7.0 / 11.4 / 22.2), 16384 12.5 / 12.2 / 27.8 (10.8 / 11.3 / 26.0)
//   4 turns                      512 columns 6.1 / 9.1 / 21.9 (6.0 / 12.1 / 22.7), 1024 8.6 / 9.0 / 24.3 (7.2 / 12.2 / 23.0)
//   the last workgroup adds up   32 parts of 64 columns 7.9 / 8.2 / 23.3 (6.4 / 10.8 / 22.1), 16 of 512 7.9 / 8.1 / 23.2 (6.1 / 10.7 / 22.0),
//                                8 of 1024 9.9 / 9.5 / 25.1 (7.3 / 10.7 / 22.8), 4 of 2048 10.8 / 10.3 / 25.9 (7.0 / 10.8 / 22.5)
// The arrival costs the device up to 1.8 us and saves the host 2.6 for narrow rows; wider ones cost it more than the host saves.
constexpr int NORM_GRAD_NARROW = 512;
constexpr int64_t NORM_GRAD_ONE_LAUNCH = 64 << 10;

static int norm_grad_groups(int T, int d, int dtype, bool sums, bool* one_launch) {
  const int rows = norm_grad_rows(d, dtype);
  const int64_t most = (static_cast<int64_t>(T) + rows - 1) / rows, groups = most < num_cus() ? most : num_cus();
  *one_launch = false;
  if (!sums) return static_cast<int>(groups);          // (dx alone: 256 rows of 1024 in bf16 3.9 us, on 8 workgroups 7.3)
  const bool narrow = d <= NORM_GRAD_NARROW, single = most <= (narrow ? 4 : d <= 8192 ? 2 : 1);
  *one_launch = single || (narrow && most <= MOST_LEFT && most * 8 * d <= NORM_GRAD_ONE_LAUNCH);
  return single && groups > 1 ? 1 : static_cast<int>(groups);
}

static size_t norm_grad_bytes(int T, int d) {          // (fp32 has as many workgroups or more)
  bool one;
  const int groups = norm_grad_groups(T, d, SCMOE_F32, true, &one);
  return static_cast<size_t>(groups) * (8 * static_cast<size_t>(d) + 8);   // parts and marks
}

constexpr int64_t NORM_MAX_GROUPS = 1 << 20;   // keeps the threads of a launch under 2^32; more rows than that take turns

static int layer_norm(const NormArgs& a, int dtype, hipStream_t stream) {
  const int d = a.d;
  const int lanes = norm_lanes(d, dtype);
  if (lanes < 64) {
    const int rows = 256 / lanes;
    const int64_t groups = (static_cast<int64_t>(a.T) + rows - 1) / rows;
    dim3 grid(static_cast<unsigned>(groups < NORM_MAX_GROUPS ? groups : NORM_MAX_GROUPS)), block(256);
    if (dtype == SCMOE_BF16 && lanes == 16) hipLaunchKernelGGL((layer_norm_kernel<true, 8, 1, false, 16>), grid, block, 0, stream, a);
    else if (dtype == SCMOE_BF16) hipLaunchKernelGGL((layer_norm_kernel<true, 8, 1, false, 32>), grid, block, 0, stream, a);
    else if (lanes == 16) hipLaunchKernelGGL((layer_norm_kernel<false, 4, 1, false, 16>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((layer_norm_kernel<false, 4, 1, false, 32>), grid, block, 0, stream, a);
    return launch_status();
  }
  const bool st = streams_past_caches(static_cast<int64_t>(a.T) * d * elem_bytes(dtype) * (a.residual != nullptr ? 4 : 2));
#define SCMOE_NORM(V, W)                                                                                                  \
  do {                                                                                                                    \
    const int64_t groups = W == 1 ? (static_cast<int64_t>(a.T) + 3) / 4 : a.T;                                            \
    dim3 grid(static_cast<unsigned>(groups < NORM_MAX_GROUPS ? groups : NORM_MAX_GROUPS)), block(norm_threads(W));        \
    if (dtype == SCMOE_BF16 && st) hipLaunchKernelGGL((layer_norm_kernel<true, V, W, true>), grid, block, 0, stream, a);  \
    else if (dtype == SCMOE_BF16) hipLaunchKernelGGL((layer_norm_kernel<true, V, W, false>), grid, block, 0, stream, a);  \
    else if (st) hipLaunchKernelGGL((layer_norm_kernel<false, V, W, true>), grid, block, 0, stream, a);                   \
    else hipLaunchKernelGGL((layer_norm_kernel<false, V, W, false>), grid, block, 0, stream, a);                          \
  } while (0)
  if (d <= 512) SCMOE_NORM(8, 1);
  else if (d <= 1024) SCMOE_NORM(16, 1);
  else if (d <= 2048) SCMOE_NORM(32, 1);
  else if (d <= 4096) SCMOE_NORM(16, 4);
  else if (d <= 8192) SCMOE_NORM(32, 4);
  else SCMOE_NORM(32, 8);
#undef SCMOE_NORM
  return launch_status();
}

static int layer_norm_backward(const NormGradArgs& a, int dtype, int groups, hipStream_t stream) {
  const int d = a.d;
  const int lanes = norm_lanes(d, dtype);
  if (lanes < 64) {
    const size_t lds = a.parts != nullptr ? static_cast<size_t>(d) * 16 : 0;
    dim3 grid(groups), block(512);
    if (dtype == SCMOE_BF16 && lanes == 16) hipLaunchKernelGGL((layer_norm_backward_kernel<true, 8, 1, 8, false, 16>), grid, block, lds, stream, a);
    else if (dtype == SCMOE_BF16) hipLaunchKernelGGL((layer_norm_backward_kernel<true, 8, 1, 8, false, 32>), grid, block, lds, stream, a);
    else if (lanes == 16) hipLaunchKernelGGL((layer_norm_backward_kernel<false, 4, 1, 8, false, 16>), grid, block, lds, stream, a);
    else hipLaunchKernelGGL((layer_norm_backward_kernel<false, 4, 1, 8, false, 32>), grid, block, lds, stream, a);
    return launch_status();
  }
  const bool st = streams_past_caches(static_cast<int64_t>(a.T) * d * elem_bytes(dtype) * (a.dsum != nullptr ? 4 : 3));
#define SCMOE_NORM(V, W, R)                                                                                                             \
  do {                                                                                                                                  \
    const size_t lds = R > 1 && a.parts != nullptr ? static_cast<size_t>(d) * (W <= 2 ? 16 : 8) : 0;                                    \
    dim3 grid(groups), block(64 * W * R);                                                                                               \
    if (dtype == SCMOE_BF16 && st) hipLaunchKernelGGL((layer_norm_backward_kernel<true, V, W, R, true>), grid, block, lds, stream, a);  \
    else if (dtype == SCMOE_BF16) hipLaunchKernelGGL((layer_norm_backward_kernel<true, V, W, R, false>), grid, block, lds, stream, a);  \
    else if (st) hipLaunchKernelGGL((layer_norm_backward_kernel<false, V, W, R, true>), grid, block, lds, stream, a);                   \
    else hipLaunchKernelGGL((layer_norm_backward_kernel<false, V, W, R, false>), grid, block, lds, stream, a);                          \
  } while (0)
  if (d <= 512) SCMOE_NORM(8, 1, 8);
  else if (d <= 1024) SCMOE_NORM(16, 1, 8);
  else if (d <= 2048) SCMOE_NORM(16, 2, 4);
  else if (d <= 4096) SCMOE_NORM(16, 4, 2);
  else if (d <= 8192) SCMOE_NORM(16, 8, 1);
  else SCMOE_NORM(32, 8, 1);
#undef SCMOE_NORM
  return launch_status();
}

static int norm_shape(int dtype, int T, int d) {
  if (!dtype_ok(dtype)) return SCMOE_ERR_DTYPE;
  if (T < 0 || d <= 0 || d % 8 != 0 || d > SCMOE_MAX_NORM_WIDTH) return SCMOE_ERR_SHAPE;
  return SCMOE_OK;
}

}  // namespace scmoe

extern "C" int scmoe_layer_norm(const void* x, int64_t ldx, int32_t dtype, const void* residual, int64_t ldres, const float* gamma,
                                const float* beta, float eps, int32_t T, int32_t d, void* sum, int64_t ldsum, void* y, int64_t ldy,
                                float* mean, float* rstd, void* stream) {
  using namespace scmoe;
  if (const int st = norm_shape(dtype, T, d)) return st;
  if (!(eps > 0.0f) || isinf(eps)) return SCMOE_ERR_ARG;
  if (T == 0) return SCMOE_OK;
  if (!x || !y || (residual != nullptr) != (sum != nullptr)) return SCMOE_ERR_NULL;
  if (!view_ok(x, ldx, d, dtype) || !view_ok(y, ldy, d, dtype) || !aligned16(gamma) || !aligned16(beta)) return SCMOE_ERR_SHAPE;
  if (residual && (!view_ok(residual, ldres, d, dtype) || !view_ok(sum, ldsum, d, dtype))) return SCMOE_ERR_SHAPE;
  const int eb = elem_bytes(dtype);
  NormArgs a = {};
  a.x = static_cast<const unsigned char*>(x); a.ldx = ldx * eb;
  a.residual = static_cast<const unsigned char*>(residual); a.ldres = ldres * eb;
  a.sum = static_cast<unsigned char*>(sum); a.ldsum = ldsum * eb;
  a.gamma = gamma; a.beta = beta; a.eps = eps; a.T = T; a.d = d;
  a.y = static_cast<unsigned char*>(y); a.ldy = ldy * eb;
  a.mean = mean; a.rstd = rstd;
  return layer_norm(a, dtype, static_cast<hipStream_t>(stream));
}

extern "C" int scmoe_layer_norm_backward_workspace_bytes(int32_t T, int32_t d, size_t* out) {
  using namespace scmoe;
  if (!out) return SCMOE_ERR_NULL;
  if (const int st = norm_shape(SCMOE_F32, T, d)) return st;
  *out = norm_grad_bytes(T, d);
  return SCMOE_OK;
}

extern "C" int scmoe_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int32_t dtype, const float* gamma,
                                         const float* mean, const float* rstd, const void* dsum, int64_t lddsum, int32_t T, int32_t d,
                                         void* dx, int64_t lddx, float* dgamma, float* dbeta, void* workspace, size_t ws_bytes,
                                         void* stream) {
  using namespace scmoe;
  if (const int st = norm_shape(dtype, T, d)) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const bool sums = dgamma != nullptr || dbeta != nullptr;
  if (T == 0) return sums ? sum_parts(nullptr, 0, 0, dgamma, d, dbeta, d, hs) : SCMOE_OK;
  if (!dy || !x || !mean || !rstd || !dx || (sums && !workspace)) return SCMOE_ERR_NULL;
  if (!view_ok(dy, lddy, d, dtype) || !view_ok(x, ldx, d, dtype) || !view_ok(dx, lddx, d, dtype) || !aligned16(gamma)) return SCMOE_ERR_SHAPE;
  if (dsum && !view_ok(dsum, lddsum, d, dtype)) return SCMOE_ERR_SHAPE;
  if (sums && !aligned16(workspace)) return SCMOE_ERR_SHAPE;
  if (sums && ws_bytes < norm_grad_bytes(T, d)) return SCMOE_ERR_WORKSPACE;
  bool one;
  const int groups = norm_grad_groups(T, d, dtype, sums, &one);
  const int eb = elem_bytes(dtype);
  NormGradArgs a = {};
  a.dy = static_cast<const unsigned char*>(dy); a.lddy = lddy * eb;
  a.x = static_cast<const unsigned char*>(x); a.ldx = ldx * eb;
  a.gamma = gamma; a.mean = mean; a.rstd = rstd;
  a.dsum = static_cast<const unsigned char*>(dsum); a.lddsum = lddsum * eb;
  a.T = T; a.d = d;
  a.dx = static_cast<unsigned char*>(dx); a.lddx = lddx * eb;
  a.parts = sums ? static_cast<float*>(workspace) : nullptr;
  a.stride = 2 * static_cast<int64_t>(d);
  a.dgamma = dgamma; a.dbeta = dbeta;
  a.one_launch = one;
  if (sums && one && groups > 1) {
    a.marks = reinterpret_cast<unsigned long long*>(a.parts + groups * a.stride);
    a.call = next_call();
  }
  if (const int st = layer_norm_backward(a, dtype, groups, hs)) return st;
  return sums && !one ? sum_parts(a.parts, groups, a.stride, dgamma, d, dbeta, d, hs) : SCMOE_OK;
}
