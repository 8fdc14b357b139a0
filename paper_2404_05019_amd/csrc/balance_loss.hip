// The balance loss of a gate, its counts and its slope.
//
//   loss       = coef E sum_e f_e P_e,  f_e = items of expert e / (k N),  P_e = mean of p[t,e] over the N counted tokens
//   slope[e]   = dloss / dp[t,e] = coef E f_e / N        (the counts have no gradient)
//
// One pass over the probabilities.  One launch: the last workgroup to finish adds up what all have left, in the order of the workgroups,
// so the result has the same bits in every run.  Bound by the chain of load, part, mark and the last one's loads, 8 us, more than by the
// bytes: 32768 tokens of 64 experts (8.7 MB) 10.4 us, 8192 of 8 7.7 (a second launch for the parts: 35 and 10.5 with the loads of that
// stage).
#include "arrival.hpp"
#include "rows.hpp"

namespace scmoe {

constexpr int LOSS_THREADS = 512, LOSS_WAVES = LOSS_THREADS / 64;
constexpr int LOSS_PASSES = 4;         // loads of a thread that are in flight together
constexpr int LOSS_MAX_GROUPS = 256;   // the last one reads what all have left: 128 of them still in one round of loads

struct LossArgs {
  const float* probs; const int32_t* idx; const uint8_t* mask;
  int T, E, k;
  float coef;
  unsigned long long* marks; unsigned long long call;   // [groups] (all_arrived); one group: neither
  float* part_p; int32_t* part_n;                       // [groups][64], [groups][64 + 1]: sums of p; items, counted tokens
  int32_t* load; float* mean_prob; float* slope; float* loss;
};

// The first wave; lane e has the sums of expert e.
__device__ __forceinline__ void loss_finish(const LossArgs& a, float sum, int items, int n) {
  const int e = threadIdx.x;
  const bool in = e < a.E;
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

// L threads share a token, each with V consecutive experts (V = 4: one 16-byte load).
template <int V, int L>
__global__ __launch_bounds__(LOSS_THREADS) void balance_loss_kernel(LossArgs a) {
  constexpr int TOK = LOSS_THREADS / L;                  // tokens of a pass
  constexpr int OWN = L < LOSS_PASSES ? LOSS_PASSES / L : 1;   // tokens whose items a thread counts
  __shared__ float sp[LOSS_WAVES][64];
  __shared__ int sn[64], st, last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid < 64) sn[tid] = 0;
  if (tid == 0) st = 0;
  __syncthreads();
  const int e0 = V * (tid % L);
  float sum[V];
#pragma unroll
  for (int v = 0; v < V; ++v) sum[v] = 0.0f;
  int tokens = 0;
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * (TOK * LOSS_PASSES); b < a.T; b += static_cast<int64_t>(gridDim.x) * (TOK * LOSS_PASSES)) {
    float p[LOSS_PASSES][V];
    bool on[LOSS_PASSES];
#pragma unroll
    for (int i = 0; i < LOSS_PASSES; ++i) {
      const int64_t t = b + i * TOK + tid / L, tc = t < a.T ? t : a.T - 1;
      const float* row = a.probs + tc * a.E;
      if (V == 4) {
        const float4 q = *reinterpret_cast<const float4*>(row + min(e0, a.E - 4));
        p[i][0] = q.x;
        p[i][1 % V] = q.y;
        p[i][2 % V] = q.z;
        p[i][3 % V] = q.w;
      } else {
        p[i][0] = row[min(e0, a.E - 1)];
      }
      on[i] = t < a.T && (a.mask == nullptr || a.mask[tc] != 0);
    }
    // items: a thread has whole tokens; the counts are whole numbers, whose order does not matter
    int e[OWN][SCMOE_MAX_TOPK];
    bool mine[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const int at = tid + i * LOSS_THREADS;
      const int64_t t = b + at;
      mine[i] = at < TOK * LOSS_PASSES && t < a.T;
      const int64_t tc = mine[i] ? t : a.T - 1;
#pragma unroll
      for (int j = 0; j < SCMOE_MAX_TOPK; ++j) e[i][j] = j < a.k ? a.idx[tc * a.k + j] : -1;
      if (a.mask != nullptr) mine[i] = mine[i] && a.mask[tc] != 0;
    }
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      if (!mine[i]) continue;
      ++tokens;
#pragma unroll
      for (int j = 0; j < SCMOE_MAX_TOPK; ++j)
        if (e[i][j] >= 0 && e[i][j] < a.E) atomicAdd(&sn[e[i][j]], 1);
    }
#pragma unroll
    for (int i = 0; i < LOSS_PASSES; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) sum[v] += on[i] && e0 < a.E ? p[i][v] : 0.0f;
  }
#pragma unroll
  for (int off = L; off < 64; off <<= 1)
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] += __shfl_xor(sum[v], off, 64);
  if (lane < L)
#pragma unroll
    for (int v = 0; v < V; ++v) sp[wave][e0 + v] = sum[v];
  if (tokens > 0) atomicAdd(&st, tokens);
  __syncthreads();
  if (wave == 0) {
    float s = 0.0f;
    if (lane < V * L)
#pragma unroll
      for (int w = 0; w < LOSS_WAVES; ++w) s += sp[w][lane];
    if (gridDim.x == 1) {
      loss_finish(a, s, sn[lane], st);
    } else {
      leave(a.part_p + blockIdx.x * 64 + lane, s);
      leave(a.part_n + blockIdx.x * 65 + lane, sn[lane]);
      if (lane == 0) leave(a.part_n + blockIdx.x * 65 + 64, st);
    }
  }
  if (gridDim.x == 1 || !last_to_arrive(a.marks, a.call, blockIdx.x, gridDim.x, &last)) return;
  float s = 0.0f;
  int n = 0, t = 0;
#pragma unroll 16
  for (int i = wave; i < static_cast<int>(gridDim.x); i += LOSS_WAVES) {
    s += left_there(a.part_p + i * 64 + lane);
    n += left_there(a.part_n + i * 65 + lane);
    t += left_there(a.part_n + i * 65 + 64);
  }
  // (sn and st hold this workgroup's own counts, which are among those just read)
  __syncthreads();
  if (tid < 64) sn[tid] = 0;
  if (tid == 0) st = 0;
  sp[wave][lane] = s;
  __syncthreads();
  atomicAdd(&sn[lane], n);
  if (lane == 0) atomicAdd(&st, t);
  __syncthreads();
  if (wave != 0) return;
  s = 0.0f;
#pragma unroll
  for (int w = 0; w < LOSS_WAVES; ++w) s += sp[w][lane];
  loss_finish(a, s, sn[lane], st);
}

// Threads per token where each has four experts and where each has one: a power of two, so that they are neighbours in a wave.
static int loss_lanes(int E, int V) {
  int l = 1;
  while (l * V < E) l *= 2;
  return l;
}

static int loss_groups(int T, int lanes) {
  const int tokens = LOSS_THREADS / lanes * LOSS_PASSES;
  const int64_t g = (static_cast<int64_t>(T) + tokens - 1) / tokens;
  return static_cast<int>(g < 1 ? 1 : g < LOSS_MAX_GROUPS ? g : LOSS_MAX_GROUPS);
}

static size_t loss_bytes(int groups) { return static_cast<size_t>(groups) * (8 + 64 * 4 + 65 * 4); }

}  // namespace scmoe

extern "C" int scmoe_balance_loss_workspace_bytes(int32_t T, int32_t E, size_t* out) {
  using namespace scmoe;
  if (!out) return SCMOE_ERR_NULL;
  if (T < 0 || E < 1 || E > SCMOE_MAX_EXPERTS) return SCMOE_ERR_SHAPE;
  *out = loss_bytes(loss_groups(T, loss_lanes(E, 1)));
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
  if (T > 0 && ws_bytes < loss_bytes(loss_groups(T, loss_lanes(E, 1)))) return SCMOE_ERR_WORKSPACE;
  LossArgs a = {};
  a.probs = probs; a.idx = expert_idx; a.mask = mask;
  a.T = T; a.E = E; a.k = k;
  a.coef = coef;
  const bool wide = E % 4 == 0 && aligned16(probs);
  const int lanes = loss_lanes(E, wide ? 4 : 1), groups = loss_groups(T, lanes);
  a.marks = static_cast<unsigned long long*>(workspace);
  a.call = groups > 1 ? next_call() : 0;
  a.part_p = reinterpret_cast<float*>(a.marks + groups);
  a.part_n = reinterpret_cast<int32_t*>(a.part_p + groups * 64);
  a.load = load; a.mean_prob = mean_prob; a.slope = slope; a.loss = loss;
  hipStream_t hs = static_cast<hipStream_t>(stream);
#define SCMOE_LOSS(V, L)                                                                                    \
  case L: hipLaunchKernelGGL((balance_loss_kernel<V, L>), dim3(groups), dim3(LOSS_THREADS), 0, hs, a); break
  if (wide) {
    switch (lanes) {
      SCMOE_LOSS(4, 1);
      SCMOE_LOSS(4, 2);
      SCMOE_LOSS(4, 4);
      SCMOE_LOSS(4, 8);
      SCMOE_LOSS(4, 16);
    }
  } else {
    switch (lanes) {
      SCMOE_LOSS(1, 1);
      SCMOE_LOSS(1, 2);
      SCMOE_LOSS(1, 4);
      SCMOE_LOSS(1, 8);
      SCMOE_LOSS(1, 16);
      SCMOE_LOSS(1, 32);
      SCMOE_LOSS(1, 64);
    }
  }
#undef SCMOE_LOSS
  return launch_status();
}
