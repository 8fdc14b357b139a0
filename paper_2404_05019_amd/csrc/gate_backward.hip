// The balance loss of a gate, and the gradient of the gate: of the loss and of the gate weights through the softmax and
// the gate product, and of the input encode.
//
//   loss       = coef E sum_e f_e P_e,  f_e = items of expert e / (k N),  P_e = mean of p[t,e] over the N counted tokens
//   slope[e]   = dloss / dp[t,e] = coef E f_e / N        (the counts have no gradient)
//   dl[t,e]    = p (g - sum_e' p g),  g = dloss slope[e] + the gradients of the full-softmax weights chosen there
//                + w_j (dw_j - sum_i w_i dw_i) where weights are a softmax over the chosen logits alone
//   dW_g = x^T dl,  dbias = sum_t dl,  dx = dl W_g^T + the encode's gradient rows gathered by dst_row
#include "rows.hpp"

namespace scmoe {

// ---- balance loss ---------------------------------------------------------------------------------

constexpr int LOSS_THREADS = 256;
constexpr int LOSS_MAX_GROUPS = 256;

// What a workgroup found: sums of p, items and (one number) counted tokens, EP experts wide.
struct LossArgs {
  const float* probs; const int32_t* idx; const uint8_t* mask;
  int T, E, k, EP;               // EP: power of two >= E
  float coef;
  float* part_p; int32_t* part_n;   // [groups][EP], [groups][EP + 1]
  int32_t* load; float* mean_prob; float* slope; float* loss;
};

// The lanes of a token are EP apart in thread index, lane e of a token reads p[t, e] and compares the token's choices
// with e: loads are consecutive, and the counts need no atomics.
__device__ __forceinline__ void loss_sums(const LossArgs& a, int block, int blocks, float& sum, int& items, int& tokens) {
  const int per = LOSS_THREADS / a.EP, e = threadIdx.x & (a.EP - 1), sub = threadIdx.x / a.EP;
  sum = 0.0f;
  items = tokens = 0;
  for (int64_t t0 = static_cast<int64_t>(block) * per; t0 < a.T; t0 += static_cast<int64_t>(blocks) * per) {
    const int64_t t = t0 + sub;
    if (t >= a.T || (a.mask != nullptr && a.mask[t] == 0)) continue;
    ++tokens;
    if (e < a.E) sum += a.probs[t * a.E + e];
    for (int j = 0; j < a.k; ++j) items += a.idx[t * a.k + j] == e ? 1 : 0;
  }
}

// Sums over the threads of a workgroup that have one expert, in the threads of the first EP.
__device__ __forceinline__ void loss_fold(int EP, float& sum, int& items, int& tokens) {
  __shared__ float sp[LOSS_THREADS];
  __shared__ int si[LOSS_THREADS], st[LOSS_THREADS];
  sp[threadIdx.x] = sum;
  si[threadIdx.x] = items;
  st[threadIdx.x] = tokens;
  __syncthreads();
  for (int half = LOSS_THREADS / 2; half >= EP; half >>= 1) {
    if (static_cast<int>(threadIdx.x) < half) {
      sp[threadIdx.x] += sp[threadIdx.x + half];
      si[threadIdx.x] += si[threadIdx.x + half];
      st[threadIdx.x] += st[threadIdx.x + half];
    }
    __syncthreads();
  }
  sum = sp[threadIdx.x];
  items = si[threadIdx.x];
  tokens = st[threadIdx.x];
}

// The first wave holds the sums of expert `lane`.
__device__ __forceinline__ void loss_finish(const LossArgs& a, float sum, int items, int tokens) {
  if (threadIdx.x >= 64) return;
  const int e = threadIdx.x;
  const bool in = e < a.E;
  const int n = __shfl(tokens, 0, 64);
  const float inv = n > 0 ? 1.0f / static_cast<float>(n) : 0.0f;   // nothing counted: loss and slopes are zero
  const float mean = in ? sum * inv : 0.0f;
  const float slope = in ? a.coef * a.E * (static_cast<float>(items) * inv / a.k) * inv : 0.0f;
  const float loss = wave_sum(n > 0 && in ? slope * static_cast<float>(n) * mean : 0.0f);
  if (in) {
    a.load[e] = items;
    a.mean_prob[e] = mean;
    a.slope[e] = slope;
  }
  if (e == 0) a.loss[0] = loss;
}

__global__ __launch_bounds__(LOSS_THREADS) void balance_loss_kernel(LossArgs a) {
  float sum;
  int items, tokens;
  loss_sums(a, blockIdx.x, gridDim.x, sum, items, tokens);
  loss_fold(a.EP, sum, items, tokens);
  if (gridDim.x == 1) {
    loss_finish(a, sum, items, tokens);
    return;
  }
  if (static_cast<int>(threadIdx.x) < a.EP) {
    a.part_p[blockIdx.x * a.EP + threadIdx.x] = sum;
    a.part_n[blockIdx.x * (a.EP + 1) + threadIdx.x] = items;
    if (threadIdx.x == 0) a.part_n[blockIdx.x * (a.EP + 1) + a.EP] = tokens;
  }
}

__global__ __launch_bounds__(LOSS_THREADS) void balance_loss_finish_kernel(LossArgs a, int groups) {
  const int per = LOSS_THREADS / a.EP, e = threadIdx.x & (a.EP - 1);
  float sum = 0.0f;
  int items = 0, tokens = 0;
  for (int i = threadIdx.x / a.EP; i < groups; i += per) {
    sum += a.part_p[i * a.EP + e];
    items += a.part_n[i * (a.EP + 1) + e];
    tokens += a.part_n[i * (a.EP + 1) + a.EP];
  }
  loss_fold(a.EP, sum, items, tokens);
  loss_finish(a, sum, items, tokens);
}

static int padded_experts(int E) {
  int ep = 1;
  while (ep < E) ep *= 2;
  return ep;
}

static int loss_groups(int T, int E) {
  const int per = LOSS_THREADS / padded_experts(E);
  const int64_t g = (static_cast<int64_t>(T) + 4 * per - 1) / (4 * per);
  return static_cast<int>(g < 1 ? 1 : g < LOSS_MAX_GROUPS ? g : LOSS_MAX_GROUPS);
}

static size_t loss_bytes(int T, int E) {
  return static_cast<size_t>(loss_groups(T, E)) * (2 * padded_experts(E) + 1) * 4;
}

// ---- gradient of the gate -------------------------------------------------------------------------

constexpr int GG_COLS = 128;     // columns of a workgroup: 8 per lane, 16 lanes
constexpr int GG_TOKENS = 16;    // tokens of a wave's step

struct GateGradArgs {
  const unsigned char* x; int64_t ldx;          // strides in bytes
  const float* Wg; const float* probs; const int32_t* idx; const float* gate_w; const float* dgate_w;
  const float* slope; const float* dloss; const uint8_t* mask;
  int T, d, E, k, normalize;
  const unsigned char* dxp; int64_t lddxp; const int32_t* dst_row;
  unsigned char* dx; int64_t lddx;
  float* parts; int64_t stride;                 // [splits][d E + E, padded to 4]; one split: dW_g and dbias themselves
  float* dWg; float* dbias;
  int splits;
};

// A workgroup has 128 columns and every `splits`-th group of 64 tokens, a wave 16 tokens of it.  Both products run on
// the fp32 matrix instruction (16 x 16 outputs, k = 4):
//   dx:   rows = tokens,  k = experts: lane (m, q) holds dl[token m, expert 4 s + q], which it computed
//   dW_g: rows = columns, k = tokens:  lane (m, q) holds x[token 4 q + s, columns 8 m + j] as it was loaded, and
//         dl[token 4 q + s, expert m] through LDS
// Column tile j of a lane's eight is column 8 m + j, so rows of x and dx are moved in 16-byte pieces and nothing is
// shuffled.  EC: groups of 16 experts.
template <bool BF16, int EC>
__global__ __launch_bounds__(256) void gate_backward_kernel(GateGradArgs a) {
  constexpr int EP = 16 * EC, S = 4 * EC, NV = BF16 ? 8 : 4, PP = 8 / NV, LD = EP + 4;
  __shared__ __attribute__((aligned(16))) float ws[EP * GG_COLS];        // W_g transposed: [expert][column]; later sums of dW_g
  __shared__ __attribute__((aligned(16))) float dls[4][GG_TOKENS * LD];  // dl of each wave's tokens
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m = lane & 15, q = lane >> 4;
  const int split = blockIdx.x % a.splits, c0 = (blockIdx.x / a.splits) * GG_COLS;
  const int cols = min(GG_COLS, a.d - c0);
  for (int i = tid; i < EP * GG_COLS; i += 256) {
    const int c = i / EP, e = i % EP;
    ws[e * GG_COLS + c] = c < cols && e < a.E ? a.Wg[static_cast<int64_t>(c0 + c) * a.E + e] : 0.0f;
  }
  __syncthreads();
  const int col = c0 + min(8 * m, cols - 8);          // this lane's columns (lanes past the end move what they do not use)
  const bool in = 8 * m < cols;
  float slope[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int e = 4 * s + q;
    slope[s] = a.slope != nullptr && e < a.E ? a.slope[e] * (a.dloss != nullptr ? a.dloss[0] : 1.0f) : 0.0f;
  }
  f32x4_t acc[EC][8];
  float db[S];
#pragma unroll
  for (int c = 0; c < EC; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[c][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < S; ++s) db[s] = 0.0f;

  for (int64_t t0 = (static_cast<int64_t>(split) * 4 + wave) * GG_TOKENS; t0 < a.T; t0 += static_cast<int64_t>(a.splits) * 4 * GG_TOKENS) {
    // x of tokens 4 q + s
    uint4 xq[4][PP];
    bool use[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int64_t t = t0 + 4 * q + s;
      const int64_t tc = t < a.T ? t : a.T - 1;
#pragma unroll
      for (int p = 0; p < PP; ++p) xq[s][p] = load16(a.x + tc * a.ldx + static_cast<int64_t>(col) * (BF16 ? 2 : 4) + 16 * p);
      use[s] = t < a.T && (a.mask == nullptr || a.mask[tc] != 0);
    }
    // dl of token m, experts 4 s + q
    float dl[S];
    {
      const int64_t t = t0 + m;
      const bool on = t < a.T && (a.mask == nullptr || a.mask[t] != 0);
      float p[S], g[S], own[S];
      float total = 0.0f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        p[s] = on && 4 * s + q < a.E ? a.probs[t * a.E + 4 * s + q] : 0.0f;
        g[s] = slope[s];
        own[s] = 0.0f;
      }
      if (on && a.dgate_w != nullptr) {
        float dot = 0.0f;
        if (a.normalize)
          for (int j = 0; j < a.k; ++j) {
            const int e = a.idx[t * a.k + j];
            if (e >= 0 && e < a.E) dot = fmaf(a.gate_w[t * a.k + j], a.dgate_w[t * a.k + j], dot);
          }
        for (int j = 0; j < a.k; ++j) {
          const int e = a.idx[t * a.k + j];
          const float dw = a.dgate_w[t * a.k + j];
          const float v = a.normalize ? a.gate_w[t * a.k + j] * (dw - dot) : dw;
#pragma unroll
          for (int s = 0; s < S; ++s)
            if (e == 4 * s + q) {
              if (a.normalize) own[s] += v;
              else g[s] += v;
            }
        }
      }
#pragma unroll
      for (int s = 0; s < S; ++s) total = fmaf(p[s], g[s], total);
      total += __shfl_xor(total, 16, 64);
      total += __shfl_xor(total, 32, 64);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        dl[s] = on ? fmaf(p[s], g[s] - total, own[s]) : 0.0f;
        db[s] += dl[s];
        dls[wave][m * LD + 4 * s + q] = dl[s];
      }
    }
    // dx
    f32x4_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float4 w0 = *reinterpret_cast<const float4*>(&ws[(4 * s + q) * GG_COLS + 8 * m]);
      const float4 w1 = *reinterpret_cast<const float4*>(&ws[(4 * s + q) * GG_COLS + 8 * m + 4]);
      const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(dl[s], w[j], o[j], 0, 0, 0);
    }
    // dW_g
    wave_lds_order();
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      float v[8];
#pragma unroll
      for (int p = 0; p < PP; ++p) unpack16<BF16>(zero_unless(use[s], xq[s][p]), v + p * NV);
#pragma unroll
      for (int c = 0; c < EC; ++c) {
        const float b = dls[wave][(4 * q + s) * LD + 16 * c + m];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], b, acc[c][j], 0, 0, 0);
      }
    }
    wave_lds_order();
    // lane (m, q) holds dx of tokens 4 q + i, columns 8 m + j
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = t0 + 4 * q + i;
      if (t >= a.T || !in) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = o[j][i];
      if (a.dst_row != nullptr) {
        for (int j = 0; j < a.k; ++j) {
          const int64_t r = a.dst_row[t * a.k + j];
          if (r < 0) continue;
#pragma unroll
          for (int p = 0; p < PP; ++p) {
            float u[NV];
            unpack16<BF16>(load16(a.dxp + r * a.lddxp + static_cast<int64_t>(col) * (BF16 ? 2 : 4) + 16 * p), u);
#pragma unroll
            for (int n = 0; n < NV; ++n) v[p * NV + n] += u[n];
          }
        }
      }
#pragma unroll
      for (int p = 0; p < PP; ++p) store16(a.dx + t * a.lddx + static_cast<int64_t>(col) * (BF16 ? 2 : 4) + 16 * p, pack16<BF16>(v + p * NV));
    }
  }

  // Sums of the four waves, in their order.
  __syncthreads();
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float* to = &ws[(8 * (4 * q + i) + j) * EP + 16 * c + m];   // column 8 (4 q + i) + j, expert 16 c + m
            *to = acc[c][j][i] + (w == 0 ? 0.0f : *to);
          }
#pragma unroll
      for (int s = 0; s < S; ++s) {
        float v = db[s];
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) v += __shfl_xor(v, off, 64);
        if (m == 0) dls[0][4 * s + q] = v + (w == 0 ? 0.0f : dls[0][4 * s + q]);
      }
    }
    __syncthreads();
  }
  float* dw = a.splits == 1 ? a.dWg : a.parts + split * a.stride;
  for (int i = tid; i < cols * a.E; i += 256) dw[static_cast<int64_t>(c0) * a.E + i] = ws[(i / a.E) * EP + i % a.E];
  if (c0 == 0) {
    float* to = a.splits == 1 ? a.dbias : a.parts + split * a.stride + static_cast<int64_t>(a.d) * a.E;
    if (to != nullptr)
      for (int i = tid; i < a.E; i += 256) to[i] = dls[0][i];
  }
}

// Two workgroups per compute unit where there are tokens for them.
static int gate_grad_splits(int T, int d) {
  const int blocks = (d + GG_COLS - 1) / GG_COLS;
  const int64_t groups = (static_cast<int64_t>(T) + 4 * GG_TOKENS - 1) / (4 * GG_TOKENS);
  const int want = (2 * num_cus() + blocks - 1) / blocks;
  return static_cast<int>(groups < 1 ? 1 : groups < want ? groups : want);
}

static int64_t gate_grad_stride(int d, int E) { return (static_cast<int64_t>(d) * E + E + 3) / 4 * 4; }

static size_t gate_grad_bytes(int T, int d, int E) {
  const int s = gate_grad_splits(T, d);
  return s == 1 ? 0 : static_cast<size_t>(s) * gate_grad_stride(d, E) * 4;
}

static int gate_backward(const GateGradArgs& a, int dtype, hipStream_t stream) {
  dim3 grid((a.d + GG_COLS - 1) / GG_COLS * a.splits), block(256);
#define SCMOE_GATE_GRAD(EC)                                                                                          \
  do {                                                                                                               \
    if (dtype == SCMOE_BF16) hipLaunchKernelGGL((gate_backward_kernel<true, EC>), grid, block, 0, stream, a);        \
    else hipLaunchKernelGGL((gate_backward_kernel<false, EC>), grid, block, 0, stream, a);                           \
  } while (0)
  if (a.E <= 16) SCMOE_GATE_GRAD(1);
  else if (a.E <= 32) SCMOE_GATE_GRAD(2);
  else SCMOE_GATE_GRAD(4);
#undef SCMOE_GATE_GRAD
  if (const int st = launch_status()) return st;
  if (a.splits == 1) return SCMOE_OK;
  return sum_parts(a.parts, a.splits, a.stride, a.dWg, static_cast<int64_t>(a.d) * a.E, a.dbias, a.E, stream);
}

}  // namespace scmoe

extern "C" int scmoe_balance_loss_workspace_bytes(int32_t T, int32_t E, size_t* out) {
  using namespace scmoe;
  if (!out) return SCMOE_ERR_NULL;
  if (T < 0 || E < 1 || E > SCMOE_MAX_EXPERTS) return SCMOE_ERR_SHAPE;
  *out = loss_bytes(T, E);
  return SCMOE_OK;
}

extern "C" int scmoe_balance_loss(const float* probs, const int32_t* expert_idx, const uint8_t* mask, int32_t T, int32_t E, int32_t k,
                                  float coef, int32_t* load, float* mean_prob, float* slope, float* loss, void* workspace,
                                  size_t ws_bytes, void* stream) {
  using namespace scmoe;
  if (T < 0 || E < 1 || E > SCMOE_MAX_EXPERTS) return SCMOE_ERR_SHAPE;
  if (k < 1 || k > SCMOE_MAX_TOPK) return SCMOE_ERR_ARG;
  if (k > E || static_cast<int64_t>(T) * k > 0x7fffffffLL) return SCMOE_ERR_SHAPE;   // counts are int32
  if (!load || !mean_prob || !slope || !loss || (T > 0 && (!probs || !expert_idx || !workspace))) return SCMOE_ERR_NULL;
  if (!aligned16(workspace)) return SCMOE_ERR_SHAPE;
  if (T > 0 && ws_bytes < loss_bytes(T, E)) return SCMOE_ERR_WORKSPACE;
  LossArgs a = {};
  a.probs = probs; a.idx = expert_idx; a.mask = mask;
  a.T = T; a.E = E; a.k = k; a.EP = padded_experts(E);
  a.coef = coef;
  const int groups = loss_groups(T, E);
  a.part_p = static_cast<float*>(workspace);
  a.part_n = reinterpret_cast<int32_t*>(a.part_p + groups * a.EP);
  a.load = load; a.mean_prob = mean_prob; a.slope = slope; a.loss = loss;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(balance_loss_kernel, dim3(groups), dim3(LOSS_THREADS), 0, hs, a);
  if (const int st = launch_status()) return st;
  if (groups == 1) return SCMOE_OK;
  hipLaunchKernelGGL(balance_loss_finish_kernel, dim3(1), dim3(LOSS_THREADS), 0, hs, a, groups);
  return launch_status();
}

extern "C" int scmoe_gate_backward_workspace_bytes(int32_t T, int32_t d, int32_t E, size_t* out) {
  using namespace scmoe;
  if (!out) return SCMOE_ERR_NULL;
  if (T < 0 || d <= 0 || d % 8 != 0 || E < 1 || E > SCMOE_MAX_EXPERTS) return SCMOE_ERR_SHAPE;
  *out = gate_grad_bytes(T, d, E);
  return SCMOE_OK;
}

extern "C" int scmoe_gate_backward(const void* x, int64_t ldx, int32_t dtype, const float* W_g, const float* probs,
                                   const int32_t* expert_idx, const float* gate_w, const float* dgate_w, const float* slope,
                                   const float* dloss, const uint8_t* mask, int32_t T, int32_t d, int32_t E, int32_t k,
                                   int32_t normalize, const void* dx_perm, int64_t ld_perm, const int32_t* dst_row, void* dx,
                                   int64_t lddx, float* dW_g, float* dbias, void* workspace, size_t ws_bytes, void* stream) {
  using namespace scmoe;
  if (!dtype_ok(dtype)) return SCMOE_ERR_DTYPE;
  if (T < 0 || d <= 0 || d % 8 != 0 || E < 1 || E > SCMOE_MAX_EXPERTS) return SCMOE_ERR_SHAPE;
  if (k < 1 || k > SCMOE_MAX_TOPK || (normalize != 0 && normalize != 1)) return SCMOE_ERR_ARG;
  if (k > E) return SCMOE_ERR_SHAPE;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (!dW_g) return SCMOE_ERR_NULL;
  if (T == 0) return sum_parts(nullptr, 0, 0, dW_g, static_cast<int64_t>(d) * E, dbias, E, hs);
  if (!x || !W_g || !probs || !dx || (!dgate_w && !slope) || (dgate_w && !expert_idx)) return SCMOE_ERR_NULL;
  if (dgate_w && normalize && !gate_w) return SCMOE_ERR_NULL;
  if ((dx_perm != nullptr) != (dst_row != nullptr)) return SCMOE_ERR_NULL;
  if (!view_ok(x, ldx, d, dtype) || !view_ok(dx, lddx, d, dtype) || (dx_perm && !view_ok(dx_perm, ld_perm, d, dtype))) return SCMOE_ERR_SHAPE;
  const size_t need = gate_grad_bytes(T, d, E);
  if (need && !workspace) return SCMOE_ERR_NULL;
  if (need && !aligned16(workspace)) return SCMOE_ERR_SHAPE;
  if (ws_bytes < need) return SCMOE_ERR_WORKSPACE;
  const int eb = elem_bytes(dtype);
  GateGradArgs a = {};
  a.x = static_cast<const unsigned char*>(x); a.ldx = ldx * eb;
  a.Wg = W_g; a.probs = probs; a.idx = expert_idx; a.gate_w = gate_w; a.dgate_w = dgate_w;
  a.slope = slope; a.dloss = dloss; a.mask = mask;
  a.T = T; a.d = d; a.E = E; a.k = k; a.normalize = normalize;
  a.dxp = static_cast<const unsigned char*>(dx_perm); a.lddxp = ld_perm * eb; a.dst_row = dst_row;
  a.dx = static_cast<unsigned char*>(dx); a.lddx = lddx * eb;
  a.splits = gate_grad_splits(T, d);
  a.parts = static_cast<float*>(workspace); a.stride = gate_grad_stride(d, E);
  a.dWg = dW_g; a.dbias = dbias;
  return gate_backward(a, dtype, hs);
}
