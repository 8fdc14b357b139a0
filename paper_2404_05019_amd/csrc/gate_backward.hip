// The gradient of the gate: of the gate weights and of the balance loss through the softmax and the gate product, and of the
// input encode.
//
//   dl[t,e]    = p (g - sum_e' p g),  g = dloss slope[e] + the gradients of the full-softmax weights chosen there
//                + w_j (dw_j - sum_i w_i dw_i) where weights are a softmax over the chosen logits alone
//   dW_g = x^T dl,  dbias = sum_t dl,  dx = dl W_g^T + the encode's gradient rows gathered by dst_row
//
// Bound by HBM where there are many tokens and up to 32 experts (32768 tokens of 2048, 16 experts, bf16, with the encode: 76 us for
// 410 MB, and 5 us for adding up the parts); by issue beyond (64 experts, two each: 222 us, where every column block works out
// dl of its tokens anew and the products take 31 us of matrix pipe); by the chain of one step and the kernel's start and end where there are
// few tokens (5003 of 1024, 32 experts: 23 us, of which the rows' loads 10, W_g 3, sums 2).
#include "arrival.hpp"
#include "rows.hpp"

namespace scmoe {

constexpr int GG_TOK = 16;       // tokens of a wave's step
static_assert(GG_TOK * SCMOE_MAX_TOPK <= 64, "one register holds a step's items");
constexpr int GATE_GRAD_FEW_PARTS = 8;   // that the last workgroup of a column block adds up (the rule: GATE_GRAD_ONE_LAUNCH)
static_assert(GATE_GRAD_FEW_PARTS <= MOST_LEFT);

struct GateGradArgs {
  const unsigned char* x; int64_t ldx;          // strides in bytes
  const float* Wg; const float* probs; const int32_t* idx; const float* gate_w; const float* dgate_w;
  const float* slope; const float* dloss; const uint8_t* mask;
  int T, d, E, k, normalize;
  int probs16, Wg16;                            // rows of probs, of W_g are 16-byte aligned
  const unsigned char* dxp; int64_t lddxp; const int32_t* dst_row;
  unsigned char* dx; int64_t lddx;
  float* parts; int64_t stride;                 // [splits][d E + E, padded to 4]; one split: dW_g and dbias themselves
  float* dWg; float* dbias;
  int splits;
  unsigned long long* marks; unsigned long long call;   // one launch: the last workgroup of a column block adds up its parts (nullptr: not)
};

// A workgroup has COLS columns and every `splits`-th group of 64 tokens, a wave 16 tokens of it at a time.  Outputs of both
// products are 16 x 16 tiles of the matrix instructions:
//   dx:   rows = tokens,  k = experts: lane (m, q) computes dl[token m, S consecutive experts] and holds it as operand
//   dW_g: rows = columns, k = tokens:  lane (m, q) holds x[tokens 4 q + i, columns NV m + j] as it was loaded, and
//         dl[tokens 4 q + i, expert m] through LDS
// Column tile j of a lane's NV is column NV m + j, so rows of x and dx are moved in pieces of 16 bytes (8 for bf16 beyond 32
// experts, whose accumulators leave room for two waves per SIMD only so: 4 tokens 12.6 -> 8.6 us, 32768 of 2048 217 -> 222) and nothing is
// shuffled.  fp32: the fp32 instruction (k = 4).  bf16: the bf16 ones (k = 16 and 32, 8 and 16 times the rate):
//   dx:   dl and W_g each as two bf16 parts, rounded, 2^-16 of the value; the product of the low parts is left out
//   dW_g: x is bf16; dl in three truncated parts, which hold its 24 bits exactly
// (all on the fp32 instruction, 32768 tokens of 2048 took 155 us in place of 89 at that stage.)  What the next step reads is loaded
// a step ahead, the encode's rows as soon as their places are known.  Two workgroups per compute unit: three took 90 and four 96 us
// in place of 82.
template <bool BF16, int EC>
struct GateGradCfg {
  static constexpr int EP = 16 * EC;                                 // experts, padded
  static constexpr int S = EP / 4;                                   // experts of a lane
  static constexpr int NV = BF16 && EC < 4 ? 8 : 4, COLS = 16 * NV, EB = BF16 ? 2 : 4;
  using Piece = std::conditional_t<NV * EB == 16, uint4, uint2>;     // a lane's columns of a row
  static constexpr int KB = EC == 4 ? 2 : 1;                         // bf16: k blocks of dx
  static constexpr int KS = EC == 1 ? 4 : 8;                         // and values of a lane in one
  static constexpr int LD = GG_TOK + 4;                              // floats per expert of the dl buffer
  static constexpr int W_BYTES = EP * COLS * 4;
  static constexpr int SUM_BYTES = (EC > 1 ? 2 : 1) * 4 * COLS * 16 * 4;   // dW_g of four waves, 16 experts, twice
  static constexpr int LDS = W_BYTES + 16 * EP * LD > SUM_BYTES ? W_BYTES + 16 * EP * LD : SUM_BYTES;
};

// A piece as fp32 values and back, 16 bytes or 8; its bytes in memory.
template <bool BF16>
__device__ __forceinline__ void unpack(const uint4& q, float* v) { unpack16<BF16>(q, v); }
template <bool BF16>
__device__ __forceinline__ void unpack(const uint2& q, float* v) {
  v[0] = __uint_as_float(q.x << 16);
  v[1] = __uint_as_float(q.x & 0xffff0000u);
  v[2] = __uint_as_float(q.y << 16);
  v[3] = __uint_as_float(q.y & 0xffff0000u);
}
template <bool BF16>
__device__ __forceinline__ void pack(const float* v, uint4& q) { q = pack16<BF16>(v); }
template <bool BF16>
__device__ __forceinline__ void pack(const float* v, uint2& q) { q = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])); }
__device__ __forceinline__ uint2 zero_unless(bool keep, const uint2& q) { return make_uint2(keep ? q.x : 0u, keep ? q.y : 0u); }
template <bool STREAM>
__device__ __forceinline__ void load_piece(const unsigned char* p, uint4& q) { q = load16<STREAM>(p); }
template <bool STREAM>
__device__ __forceinline__ void load_piece(const unsigned char* p, uint2& q) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  const u32x2_t v = STREAM ? __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p)) : *reinterpret_cast<const u32x2_t*>(p);
  q = make_uint2(v.x, v.y);
}
template <bool STREAM>
__device__ __forceinline__ void store_piece(unsigned char* p, const uint4& q) { store16<STREAM>(p, q); }
template <bool STREAM>
__device__ __forceinline__ void store_piece(unsigned char* p, const uint2& q) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  if (STREAM) __builtin_nontemporal_store(u32x2_t{q.x, q.y}, reinterpret_cast<u32x2_t*>(p));
  else *reinterpret_cast<u32x2_t*>(p) = u32x2_t{q.x, q.y};
}
// Columns 2 i and 2 i + 1 in bf16.
__device__ __forceinline__ uint32_t word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
__device__ __forceinline__ uint32_t word(const uint2& q, int i) { return i == 0 ? q.x : q.y; }

// Tokens of a step.
__device__ __forceinline__ int gate_grad_left(const GateGradArgs& a, int64_t t0) { return a.T - t0 < GG_TOK ? static_cast<int>(a.T - t0) : GG_TOK; }

// What a step reads, as it lies in memory: loaded a step ahead, so nothing here may be looked at (and waited for) before it is due.
template <bool BF16, int EC>
struct GateGradStep {
  typename GateGradCfg<BF16, EC>::Piece x[4];   // tokens 4 q + i
  float p[GateGradCfg<BF16, EC>::S];   // token m
  int idx, dst;                        // item `lane` of the step's 16 k
  float add, w;                        // its dgate_w, its gate_w
  uint32_t mask;                       // token m
};

template <bool BF16, int EC, int K, bool DISPATCH, bool ST>
__device__ __forceinline__ void gate_grad_load(const GateGradArgs& a, int64_t t0, int64_t col_byte, int lane, GateGradStep<BF16, EC>& n) {
  using C = GateGradCfg<BF16, EC>;
  const int m = lane & 15, q = lane >> 4;
  const int left = gate_grad_left(a, t0);
  const int mine = min(m, left - 1);
  n.mask = 1;
  if (a.mask != nullptr) n.mask = a.mask[t0 + mine];
  const int at = min(lane, left * K - 1);
  n.idx = n.dst = -1;
  n.add = n.w = 0.0f;
  if (DISPATCH) n.dst = a.dst_row[t0 * K + at];
  if (a.dgate_w != nullptr) {
    n.idx = a.idx[t0 * K + at];
    n.add = a.dgate_w[t0 * K + at];
    if (a.normalize) n.w = a.gate_w[t0 * K + at];
  }
  const float* row = a.probs + (t0 + mine) * a.E;
  if (a.probs16) {
#pragma unroll
    for (int s = 0; s < C::S; s += 4) {
      const float4 v = *reinterpret_cast<const float4*>(row + min(C::S * q + s, a.E - 4));
      n.p[s] = v.x;
      n.p[s + 1] = v.y;
      n.p[s + 2] = v.z;
      n.p[s + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int s = 0; s < C::S; ++s) n.p[s] = row[min(C::S * q + s, a.E - 1)];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) load_piece<ST>(a.x + (t0 + min(4 * q + i, left - 1)) * a.ldx + col_byte, n.x[i]);
}

template <int N>
union Bf16Parts {
  uint32_t w[N / 2];
  __bf16 __attribute__((ext_vector_type(N))) v;
  short __attribute__((ext_vector_type(N))) s;
};

template <int N>
__device__ __forceinline__ f32x4_t mfma_bf16(const Bf16Parts<N>& a, const Bf16Parts<N>& b, f32x4_t c) {
  if constexpr (N == 4) return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a.s, b.s, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}

// Two parts, rounded.
template <int N>
__device__ __forceinline__ void split2(const float* v, Bf16Parts<N>& hi, Bf16Parts<N>& lo) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    hi.w[i] = cvt_pk_bf16(v[2 * i], v[2 * i + 1]);
    lo.w[i] = cvt_pk_bf16(v[2 * i] - __uint_as_float(hi.w[i] << 16), v[2 * i + 1] - __uint_as_float(hi.w[i] & 0xffff0000u));
  }
}

// The high (low) halves of two words, the first one's in the low half.
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Three parts, truncated: their sum is the value.
__device__ __forceinline__ void split3(const float* v, Bf16Parts<4> (&part)[3]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      part[p].w[i] = high_halves(__float_as_uint(a), __float_as_uint(b));
      a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
      b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
    }
  }
}

// Rows of the encode's gradient for choice j of tokens 4 q + i, as far as they were kept.
template <int K, bool ST, typename Piece>
__device__ __forceinline__ uint32_t gate_grad_rows(const GateGradArgs& a, int64_t t0, int64_t col_byte, int lane, int dst, int j, Piece (&dp)[4]) {
  uint32_t have = 0;
  const int items = gate_grad_left(a, t0) * K;
  const unsigned char* at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int item = (4 * (lane >> 4) + i) * K + j, r = __shfl(dst, item, 64);
    const bool there = r >= 0 && item < items;
    have |= there ? 1u << i : 0u;
    // (no row: the x of the step's first token, which is there)
    at[i] = (there ? a.dxp + r * a.lddxp : a.x + t0 * a.ldx) + col_byte;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) load_piece<ST>(at[i], dp[i]);
  return have;
}

// Adds them to dx: lane (m, q) holds tokens 4 q + i, columns NV m + l.
template <bool BF16, int NV, typename Piece>
__device__ __forceinline__ void gate_grad_add(const Piece (&dp)[4], uint32_t have, f32x4_t (&o)[NV]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float u[NV];
    unpack<BF16>(zero_unless((have >> i & 1u) != 0, dp[i]), u);
#pragma unroll
    for (int l = 0; l < NV; ++l) o[l][i] += u[l];
  }
}

// K: experts per token.  DISPATCH: with the encode's rows.  ST: rows are moved past the caches (streams_past_caches); a choice at run time
// between the two kinds of store came out of the compiler as one, without the hint.
template <bool BF16, int EC, int K, bool DISPATCH, bool ST>
__global__ __launch_bounds__(256, 2) void gate_backward_kernel(GateGradArgs a) {
  using C = GateGradCfg<BF16, EC>;
  constexpr int EP = C::EP, S = C::S, LD = C::LD, NV = C::NV, COLS = C::COLS, KB = C::KB, KS = C::KS;
  constexpr bool SECOND = DISPATCH && K > 1 && (BF16 || EC < 4);   // (rows of the second choice early: fp32 beyond 32 experts has no registers left)
  constexpr int ITEMS = BF16 || EC < 4 || K < 4 ? K : 1;           // items of a token looked at together (as SECOND: registers)
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::LDS];
  __shared__ float dbs[4][EP];
  __shared__ int last_one;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, q = lane >> 4;
  float* const dls = reinterpret_cast<float*>(lds + C::W_BYTES) + wave * EP * LD;   // dl of this wave's tokens: [expert][token]
  // Consecutive workgroups go to the eight dies in turn: each die takes a run of (split, column block), so that the blocks of a
  // token's row, whose ends share cache lines and whose probabilities are the same, meet in one L2.
  const int blocks = (a.d + COLS - 1) / COLS;
  const int id = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  if (id >= a.splits * blocks) return;
  const int split = id / blocks, c0 = id % blocks * COLS;
  const int cols = min(COLS, a.d - c0);
  const bool in = NV * m < cols;                      // (lanes past the end move what they do not use)
  const int64_t col_byte = static_cast<int64_t>(c0 + min(NV * m, cols - NV)) * C::EB;
  const int64_t step = static_cast<int64_t>(a.splits) * 4 * GG_TOK;
  int64_t t0 = (static_cast<int64_t>(split) * 4 + wave) * GG_TOK;
  GateGradStep<BF16, EC> n;
  typename C::Piece dp[4];                                        // the encode's rows of the first choice
  uint32_t have = 0;
  if (t0 < a.T) gate_grad_load<BF16, EC, K, DISPATCH, ST>(a, t0, col_byte, lane, n);

  // W_g as operands of dx, in the order in which the lanes read them
  const float* const wg = a.Wg + static_cast<int64_t>(c0) * a.E;
  if constexpr (BF16) {
    Bf16Parts<KS>* const wl = reinterpret_cast<Bf16Parts<KS>*>(lds);   // [column tile][part][k block][lane]
    constexpr int N = NV * KB * 64 / 256;
    float v[N][KS];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = tid + n * 256, l = i % 64, kb = i / 64 % KB, j = i / (64 * KB);
      const int c = NV * (l & 15) + j, e = S * (l >> 4) + KS * kb;
      const float* const row = wg + min(c, cols - 1) * a.E;
      if (a.Wg16) {
#pragma unroll
        for (int s = 0; s < KS; s += 4) {
          const float4 t = *reinterpret_cast<const float4*>(row + min(e + s, a.E - 4));
          v[n][s] = t.x;
          v[n][s + 1] = t.y;
          v[n][s + 2] = t.z;
          v[n][s + 3] = t.w;
        }
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) v[n][s] = row[min(e + s, a.E - 1)];
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = tid + n * 256, l = i % 64, kb = i / 64 % KB, j = i / (64 * KB);
      const int c = NV * (l & 15) + j, e = S * (l >> 4) + KS * kb;
#pragma unroll
      for (int s = 0; s < KS; ++s) v[n][s] = c < cols && e + s < a.E ? v[n][s] : 0.0f;
      split2<KS>(v[n], wl[(j * 2 * KB + kb) * 64 + l], wl[((j * 2 + 1) * KB + kb) * 64 + l]);
    }
  } else {
    float* const wl = reinterpret_cast<float*>(lds);                 // [expert][column]
    constexpr int N = EP * COLS / 256;
    float v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = tid + n * 256, c = i / EP, e = i % EP;
      v[n] = wg[min(c, cols - 1) * a.E + min(e, a.E - 1)];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = tid + n * 256, c = i / EP, e = i % EP;
      wl[e * COLS + c] = c < cols && e < a.E ? v[n] : 0.0f;
    }
  }
  if (DISPATCH && t0 < a.T) have = gate_grad_rows<K, ST>(a, t0, col_byte, lane, n.dst, 0, dp);
  float slope[S];
#pragma unroll
  for (int s = 0; s < S; ++s) slope[s] = a.slope != nullptr && S * q + s < a.E ? a.slope[S * q + s] * (a.dloss != nullptr ? a.dloss[0] : 1.0f) : 0.0f;
  __syncthreads();

  f32x4_t acc[EC][NV];
  float db[EC];
#pragma unroll
  for (int c = 0; c < EC; ++c) {
    db[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) acc[c][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  for (; t0 < a.T; t0 += step) {
    // (the lane's places in shuffles and rows are worked out anew in every step: kept, they would take tens of registers)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int m = lane & 15, q = lane >> 4;
    // tokens that count, one bit each; items that are there
    const int left = gate_grad_left(a, t0);
    const uint32_t use = static_cast<uint32_t>(__ballot(m < left && n.mask != 0)) & 0xffffu;
    n.idx = lane < left * K && n.idx < a.E ? n.idx : -1;
    // rows of the second choice where there are registers for them, then everything the next step reads
    typename C::Piece second[4];
    uint32_t have_second = 0;
    if (SECOND) have_second = gate_grad_rows<K, ST>(a, t0, col_byte, lane, n.dst, 1, second);
    const bool last = t0 + step >= a.T;
    GateGradStep<BF16, EC> ahead = n;
    if (!last) gate_grad_load<BF16, EC, K, DISPATCH, ST>(a, t0 + step, col_byte, lane, ahead);
    // dl of token m, experts S q + s
    float dl[S];
    {
      const bool on = (use >> m & 1u) != 0;
      if (a.normalize) {
        // in the lanes of the items: dot over their token's items
        const int first = lane / K * K;
        const float mine = n.idx >= 0 ? n.w * n.add : 0.0f;
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j) dot += __shfl(mine, first + j, 64);
        n.add = n.w * (n.add - dot);
      }
      float g[S], own[S];
#pragma unroll
      for (int s = 0; s < S; ++s) own[s] = 0.0f;
#pragma unroll ITEMS
      for (int j = 0; j < K; ++j) {
        const int e = __shfl(n.idx, m * K + j, 64);
        const float v = __shfl(n.add, m * K + j, 64);
#pragma unroll
        for (int s = 0; s < S; ++s) own[s] += e >= 0 && e == S * q + s ? v : 0.0f;
      }
#pragma unroll
      for (int s = 0; s < S; ++s) {
        g[s] = a.normalize ? slope[s] : slope[s] + own[s];
        own[s] = a.normalize ? own[s] : 0.0f;
      }
      float total = 0.0f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        n.p[s] = on && S * q + s < a.E ? n.p[s] : 0.0f;
        total = fmaf(n.p[s], g[s], total);
      }
      total += __shfl_xor(total, 16, 64);
      total += __shfl_xor(total, 32, 64);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        dl[s] = on ? fmaf(n.p[s], g[s] - total, own[s]) : 0.0f;
        dls[(S * q + s) * LD + m] = dl[s];
      }
    }
    // dW_g
    if (use != 0xffffu) {
#pragma unroll
      for (int i = 0; i < 4; ++i) n.x[i] = zero_unless((use >> (4 * q + i) & 1u) != 0, n.x[i]);
    }
    wave_lds_order();
    // (products that add to the same tile are kept apart: each would wait for the one before)
    Bf16Parts<4> xa[NV];
    if constexpr (BF16) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = word(n.x[i], j / 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) xa[j].w[i] = j & 1 ? high_halves(w[2 * i], w[2 * i + 1]) : low_halves(w[2 * i], w[2 * i + 1]);
      }
    }
#pragma unroll
    for (int c = 0; c < EC; ++c) {
      const float4 t = *reinterpret_cast<const float4*>(&dls[(c * 16 + m) * LD + 4 * q]);
      const float v[4] = {t.x, t.y, t.z, t.w};
      db[c] += (v[0] + v[1]) + (v[2] + v[3]);
      if constexpr (BF16) {
        Bf16Parts<4> part[3];
        split3(v, part);
#pragma unroll
        for (int p = 2; p >= 0; --p)
#pragma unroll
          for (int j = 0; j < NV; ++j) acc[c][j] = mfma_bf16(xa[j], part[p], acc[c][j]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float xv[NV];
          unpack<BF16>(n.x[i], xv);
#pragma unroll
          for (int j = 0; j < NV; ++j) acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(xv[j], v[i], acc[c][j], 0, 0, 0);
        }
      }
    }
    wave_lds_order();
    // dx
    f32x4_t o[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) o[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (BF16) {
      const Bf16Parts<KS>* const wl = reinterpret_cast<const Bf16Parts<KS>*>(lds) + lane;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        Bf16Parts<KS> hi, lo;
        split2<KS>(dl + KS * kb, hi, lo);
#pragma unroll
        for (int j0 = 0; j0 < NV; j0 += 4) {
          Bf16Parts<KS> wh[4], wo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            wh[j] = wl[((j0 + j) * 2 * KB + kb) * 64];
            wo[j] = wl[(((j0 + j) * 2 + 1) * KB + kb) * 64];
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j0 + j] = mfma_bf16(hi, wo[j], o[j0 + j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j0 + j] = mfma_bf16(lo, wh[j], o[j0 + j]);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j0 + j] = mfma_bf16(hi, wh[j], o[j0 + j]);
        }
      }
    } else {
      const float4* const wl = reinterpret_cast<const float4*>(lds);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const float4 t = wl[(S * q + s) * 16 + m];
        const float w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int j = 0; j < NV; ++j) o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(dl[s], w[j], o[j], 0, 0, 0);
      }
    }
    if (DISPATCH) {
      gate_grad_add<BF16>(dp, have, o);
      if (SECOND) gate_grad_add<BF16>(second, have_second, o);
#pragma unroll
      for (int j = SECOND ? 2 : 1; j < K; ++j) {
        int dst = n.dst;
        asm volatile("" : "+v"(dst)::"memory");       // (no earlier: their addresses would take registers from here to the top)
        have = gate_grad_rows<K, ST>(a, t0, col_byte, lane, dst, j, dp);
        gate_grad_add<BF16>(dp, have, o);
      }
    }
    loads_have_arrived();
    n = ahead;
    if (DISPATCH && !last) have = gate_grad_rows<K, ST>(a, t0 + step, col_byte, lane, n.dst, 0, dp);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = t0 + 4 * q + i;
      if (t >= a.T || !in) continue;
      float v[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = o[j][i];
      unsigned char* const to = a.dx + t * a.lddx + col_byte;
      typename C::Piece out;
      pack<BF16>(v, out);
      store_piece<ST>(to, out);
    }
  }

  // Sums of the four waves, 16 experts at a time: column NV (4 q + i) + j lies in the order (j, i, q), which 64 lanes write without a
  // bank conflict.
#pragma unroll
  for (int c = 0; c < EC; ++c) {
    float v = db[c];
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    if (q == 0) dbs[wave][16 * c + m] = v;
  }
  float* const dw = (a.splits == 1 ? a.dWg : a.parts + split * a.stride) + static_cast<int64_t>(c0) * a.E;
  __syncthreads();
#pragma unroll
  for (int c = 0; c < EC; ++c) {
    if (16 * c >= a.E) break;
    float* const sums = reinterpret_cast<float*>(lds) + (c & 1) * 4 * COLS * 16;   // (read two turns ago: a barrier lies between)
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[wave * COLS * 16 + ((j * 4 + i) * 4 + q) * 16 + m] = acc[c][j][i];
    __syncthreads();
    const int e = 16 * c + (tid & 15);
    float v[COLS / 16];
#pragma unroll
    for (int n = 0; n < COLS / 16; ++n) {
      const int cc = (tid >> 4) + 16 * n, r = cc / NV;
      const float* s = sums + ((cc % NV) * 16 + (r & 3) * 4 + (r >> 2)) * 16 + (tid & 15);
      v[n] = (s[0] + s[COLS * 16]) + (s[2 * COLS * 16] + s[3 * COLS * 16]);
    }
#pragma unroll
    for (int n = 0; n < COLS / 16; ++n) {
      const int cc = (tid >> 4) + 16 * n;
      if (e < a.E && cc < cols) {
        if (a.marks != nullptr) leave(dw + cc * a.E + e, v[n]);
        else dw[cc * a.E + e] = v[n];
      }
    }
  }
  if (c0 == 0 && tid < a.E) {
    float* const to = a.splits == 1 ? a.dbias : a.parts + split * a.stride + static_cast<int64_t>(a.d) * a.E;
    const float v = (dbs[0][tid] + dbs[1][tid]) + (dbs[2][tid] + dbs[3][tid]);
    if (a.marks != nullptr) leave(to + tid, v);
    else if (to != nullptr) to[tid] = v;
  }
  if (a.marks == nullptr || !last_to_arrive(a.marks + static_cast<int64_t>(c0 / COLS) * a.splits, a.call, split, a.splits, &last_one)) return;
  const int64_t first = static_cast<int64_t>(c0) * a.E;
  for (int i = 2 * tid; i < cols * a.E; i += 512) {       // (an even number: columns come in eights)
    const float2 v = sum_left<GATE_GRAD_FEW_PARTS>(a.parts + first + i, a.splits, a.stride);
    a.dWg[first + i] = v.x;
    a.dWg[first + i + 1] = v.y;
  }
  if (c0 == 0 && a.dbias != nullptr && tid < a.E) {
    float v = 0.0f;
    for (int i = 0; i < a.splits; ++i) v += left_there(a.parts + i * a.stride + static_cast<int64_t>(a.d) * a.E + tid);
    a.dbias[tid] = v;
  }
}

static int gate_grad_cols(int E, int dtype) {
  return dtype != SCMOE_BF16 ? GateGradCfg<false, 1>::COLS : E > 32 ? GateGradCfg<true, 4>::COLS : GateGradCfg<true, 1>::COLS;
}

// Workgroups that share a column block, each with a part of dW_g to leave: as many as are resident together (two per compute unit),
// and no more than it takes for the same number of turns.
static int gate_grad_splits(int T, int d, int E, int dtype) {
  const int blocks = (d + gate_grad_cols(E, dtype) - 1) / gate_grad_cols(E, dtype);
  const int64_t groups = (static_cast<int64_t>(T) + 4 * GG_TOK - 1) / (4 * GG_TOK);
  const int resident = 2 * num_cus();
  const int64_t most = resident > blocks ? resident / blocks : 1;
  const int64_t turns = (groups + most - 1) / most;
  return turns < 1 ? 1 : static_cast<int>((groups + turns - 1) / turns);
}

static int64_t gate_grad_stride(int d, int E) { return (static_cast<int64_t>(d) * E + E + 3) / 4 * 4; }

static size_t gate_grad_bytes(int T, int d, int E) {        // (for either type)
  const int b = gate_grad_splits(T, d, E, SCMOE_BF16), f = gate_grad_splits(T, d, E, SCMOE_F32), s = b > f ? b : f;
  const size_t blocks = (d + gate_grad_cols(E, SCMOE_F32) - 1) / gate_grad_cols(E, SCMOE_F32);
  return s == 1 ? 0 : static_cast<size_t>(s) * (gate_grad_stride(d, E) * 4 + 8 * blocks);   // parts and marks
}

// A column block's last workgroup adds up its parts in the same launch where they are at most eight, of up to 4 KB each and 16 KB in all.
// us a call in a replayed graph / called back to back from Python / waited for one by one, against two launches:
//   bf16, 4 experts (2 KB a part), 4 parts 10.1 / 9.7 / 26.0 (8.5 / 11.3 / 24.7), 8 parts 10.6 / 10.3 / 26.4 (8.6 / 11.3 / 24.7)
//         8 (4 KB), 2 parts 10.3 / 10.0 / 26.2 (8.7 / 11.2 / 24.7), 4 parts 10.7 / 10.4 / 26.6 (8.7 / 11.2 / 24.8),
//         8 parts 11.7 / 11.5 / 27.7 (8.8 / 11.4 / 25.1)
//         16 (8 KB), 2 parts 11.5 / 11.2 / 27.4 (8.7 / 11.2 / 24.8)
//   fp32, 4 experts (1 KB), 8 parts 9.2 / 8.9 / 25.1 (7.3 / 11.3 / 23.5); 8 (2 KB), 8 parts 9.6 / 9.4 / 25.5 (7.6 / 11.3 / 23.8)
//         16 (4 KB), 4 parts 9.7 / 9.3 / 25.7 (7.5 / 11.2 / 23.6), 8 parts 10.7 / 10.5 / 26.7 (7.6 / 11.3 / 23.7)
//         32 (8 KB), 2 parts 13.3 / 12.9 / 29.1 (10.4 / 11.2 / 26.4)
// Up to there the arrival costs the device no more (1.1 to 2.2 us) than the second launch costs the host (2.6 to 2.8); beyond it does.
constexpr int64_t GATE_GRAD_SMALL_PART = 4 << 10;
constexpr int64_t GATE_GRAD_ONE_LAUNCH = 16 << 10;

static int gate_backward(const GateGradArgs& a, int dtype, hipStream_t stream) {
  const int cols = gate_grad_cols(a.E, dtype);
  dim3 grid(((a.d + cols - 1) / cols * a.splits + 7) / 8 * 8), block(256);
  const bool dispatch = a.dst_row != nullptr;
  // (every item counts as kept: the host does not know how many were)
  const bool st = streams_past_caches(static_cast<int64_t>(a.T) * a.d * elem_bytes(dtype) * (dispatch ? 2 + a.k : 2));
#define SCMOE_GATE_GRAD_ST(EC, K, ST)                                                                                                      \
  do {                                                                                                                                     \
    if (dtype == SCMOE_BF16 && dispatch) hipLaunchKernelGGL((gate_backward_kernel<true, EC, K, true, ST>), grid, block, 0, stream, a);     \
    else if (dtype == SCMOE_BF16) hipLaunchKernelGGL((gate_backward_kernel<true, EC, K, false, ST>), grid, block, 0, stream, a);           \
    else if (dispatch) hipLaunchKernelGGL((gate_backward_kernel<false, EC, K, true, ST>), grid, block, 0, stream, a);                      \
    else hipLaunchKernelGGL((gate_backward_kernel<false, EC, K, false, ST>), grid, block, 0, stream, a);                                   \
  } while (0)
#define SCMOE_GATE_GRAD_K(EC, K)                    \
  do {                                              \
    if (st) SCMOE_GATE_GRAD_ST(EC, K, true);        \
    else SCMOE_GATE_GRAD_ST(EC, K, false);          \
  } while (0)
#define SCMOE_GATE_GRAD(EC)                      \
  switch (a.k) {                                 \
    case 1: SCMOE_GATE_GRAD_K(EC, 1); break;     \
    case 2: SCMOE_GATE_GRAD_K(EC, 2); break;     \
    case 3: SCMOE_GATE_GRAD_K(EC, 3); break;     \
    default: SCMOE_GATE_GRAD_K(EC, 4); break;    \
  }
  static_assert(SCMOE_MAX_TOPK == 4, "one instantiation per k above");
  if (a.E <= 16) { SCMOE_GATE_GRAD(1) }
  else if (a.E <= 32) { SCMOE_GATE_GRAD(2) }
  else { SCMOE_GATE_GRAD(4) }
#undef SCMOE_GATE_GRAD
#undef SCMOE_GATE_GRAD_K
#undef SCMOE_GATE_GRAD_ST
  if (const int st = launch_status()) return st;
  if (a.splits == 1 || a.marks != nullptr) return SCMOE_OK;
  return sum_parts(a.parts, a.splits, a.stride, a.dWg, static_cast<int64_t>(a.d) * a.E, a.dbias, a.E, stream);
}

}  // namespace scmoe

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
  a.splits = gate_grad_splits(T, d, E, dtype);
  a.probs16 = E % 4 == 0 && aligned16(probs);
  a.Wg16 = E % 4 == 0 && aligned16(W_g);
  a.parts = static_cast<float*>(workspace); a.stride = gate_grad_stride(d, E);
  a.dWg = dW_g; a.dbias = dbias;
  const int64_t part = static_cast<int64_t>(gate_grad_cols(E, dtype)) * E * 4;
  if (a.splits > 1 && a.splits <= GATE_GRAD_FEW_PARTS && part <= GATE_GRAD_SMALL_PART && a.splits * part <= GATE_GRAD_ONE_LAUNCH) {
    a.marks = reinterpret_cast<unsigned long long*>(a.parts + a.splits * a.stride);
    a.call = next_call();
  }
  return gate_backward(a, dtype, hs);
}
