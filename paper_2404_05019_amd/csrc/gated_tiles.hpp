// The products of the gated feed-forward block and of its gradient, on the matrix cores (bf16 and fp32): one kernel, whose operands may
// lie along k or across it, over the packed segments of the experts.
//
//   GATE  [g; u] = W1[e] x       both operands along k; act(g) u on store, g and u beside it where they are kept
//   DOWN  y = W2[e] h            both along k
//   DH    dh = W2[e]^T dy        W2 across k; on store the gradients of g and u, and h again, from the kept g and u
//   DX    dx = W1[e]^T [dg; du]  W1 across k
//   DW    dW1[e] = [dg; du]^T x, dW2[e] = dy^T h     both across k, which is the rows of the segment
//
// A tile of BM x BN is one workgroup's; its operands come through NS stages in LDS, copied there directly (16 bytes a lane).
//  * Along k, a stage holds rows of 128 bytes of k (64 bf16 or 32 fp32), 16-byte chunks swizzled (swz); a fragment is 16 rows, lane
//    (l16, lq) holding chunk 4 s + lq of row l16 for step s: 32 k of bf16 for one instruction, 16 of fp32 for four, which take element c
//    of every chunk (the order of k inside a step is the same for both operands).
//  * Across k, it holds the 64 (32) rows of k as they lie in memory, all columns of the tile, and the fragments are transposed on the way
//    out of LDS: bf16 by ds_read_b64_tr_b16, in which 16 lanes read four rows of 16 columns and lane i gets column i of them; fp32 by four
//    reads of 4 bytes.  Units of 16 columns are swizzled by the row, so that the rows a read touches lie in different banks.
//    Nothing is transposed in memory.
//  * Rows past a segment, columns past a matrix and k past its end read zeros (offsets outside the buffer), in both operands, so that what
//    lies there (another expert's rows, NaN) reaches nothing.
//  * Persistent workgroups, as in ffn_mfma.hip, whose schedule, barrier and two-group refill of a stage these kernels share.
// Bound by the matrix rate at the power limit where the segments are long (32768 rows, d = 2048, F = 8192, E = 16: DW 1378 TFLOP/s, DX 1402, DH
// 976, whose epilogue has 26 vector operations an element), by streaming the weights where they are short (64 rows: GATE 4.9 TB/s).
#pragma once
#include "checkpoint.hpp"
#include "gated_act.hpp"
#include "pair_share.hpp"
#include "rows.hpp"
#include <atomic>
#include <math.h>

namespace scmoe {

enum { G_GATE = 0, G_DOWN = 1, G_DH = 2, G_DX = 3, G_DW = 4 };
enum { KEEP_NONE = 0, KEEP_FULL = 1, KEEP_8BIT = 2 };

// One product; strides in elements.  A: [rows, Kd] (DW: [rows, M]).  B: [E, N, Kd], GATE [E, 2 N, Kd]; DH, DX [E, Kd, N]; DW [rows, N].
struct GatedJob {
  const unsigned char* A; int64_t lda;
  const unsigned char* B; int64_t ldb;
  unsigned char* C; int64_t ldc;       // [rows, N]: hidden, y, h again, dx;  DW: [E, M, N]
  int M, N, Kd;
  int mt, nt;                          // tiles of a DW matrix down and across; of the others across
  int tiles;                           // DW: E mt nt
};
struct GatedArgs {
  GatedJob j[2];                       // DW: two products in a launch (the second may have no tiles)
  const int32_t* offsets;
  int E, act;
  unsigned char* pre; int64_t ldpre;   // GATE: written, DH: read: [rows, 2 F], or checkpoint rows 2 r, 2 r + 1 (strides in bytes)
  unsigned char* dpre; int64_t lddpre; // DH: gradients of g and u, [rows, 2 F]
  int* zero; int zeros;                // GATE: ints to clear for the launch that follows (nullptr: none)
};

template <bool F32_, int BM_, int BN_, int WM_, int WN_, int NS_, int PATCH_ = F32_ ? 0 : 4096>
struct GatedCfg {                      // NS_: stages; PATCH_: bytes of LDS that a wave has for the epilogue (2048: of DOWN, DX and DW alone)
  static constexpr bool F32 = F32_;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_;
  static constexpr int EB = F32 ? 4 : 2, VE = 16 / EB, BK = 128 / EB, KS = 2;      // KS: k steps of 64 bytes in a stage
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NJ = TN / 16;
  static constexpr int NH = MI > 1 ? 2 : 1;                                          // halves of a wave's rows that a stage is refilled by
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
  static constexpr int APW = A_BYTES / 1024 / WAVES, BPW = B_BYTES / 1024 / WAVES;  // copies of a wave and k-tile
  static constexpr int PATCH = PATCH_;
  static constexpr int LDS = NS * STAGE + WAVES * PATCH;
  static_assert(LDS <= 160 * 1024, "LDS budget");
  static constexpr int MOST_WG = (MI > 1 ? 8 : 16) / WAVES;                          // by registers: two waves a SIMD, small tiles four
  static constexpr int WG_PER_CU = (160 * 1024 / LDS) < MOST_WG ? (160 * 1024 / LDS) : MOST_WG;
  static_assert(TM % (16 * NH) == 0 && TN == 64 && APW % NH == 0 && WG_PER_CU >= 1 && NS >= 2, "tile shape");
};

// Swizzle of an operand across k: a read takes rows k of 8 consecutive ones at a time of two (bf16: lanes' groups of 16 on rows
// 8 lq + 0..3) or of four (fp32: rows 4 lq + c) groups.  ROWB: bytes of a row in LDS; the result is added (xor) to the unit of 16 columns.
template <bool F32, int ROWB>
__host__ __device__ constexpr int across_swz(int k) {
  static_assert(ROWB >= (F32 ? 256 : 128), "four units of 16 columns");
  if (F32) return (k >> 2) & 3;
  return ROWB >= 256 ? (k & 3) | (((k >> 3) & 1) << 2) : ((k >> 1) & 1) | (((k >> 3) & 1) << 1);
}

typedef unsigned int g_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int g_u32x2 __attribute__((ext_vector_type(2)));
typedef short g_i16x4 __attribute__((ext_vector_type(4)));

// Sixteen columns of four rows each of k, transposed (see above).  The second pointer is for the compiler alone: two that are said not to
// overlap give the read a scope of its own, without which it would wait for every copy in flight to LDS (vmcnt(0)) ahead of it, once a
// k-tile; the kernel waits for the copies that it needs (gradient of both weights, 32768 rows, d = 2048, F = 8192, E = 16: 3836 us with
// that wait, 2544 without).
__device__ __forceinline__ g_u32x2 lds_read_transposed(__attribute__((address_space(3))) g_i16x4* __restrict at,
                                                       __attribute__((address_space(3))) g_i16x4* __restrict /*elsewhere*/) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_bit_cast(g_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at));
#else
  return g_u32x2{0, 0};
#endif
}
__device__ __forceinline__ g_u32x2 lds_read_transposed(uint32_t at) {
  typedef __attribute__((address_space(3))) g_i16x4* lds8_ptr;
  return lds_read_transposed(reinterpret_cast<lds8_ptr>(static_cast<uintptr_t>(at)), reinterpret_cast<lds8_ptr>(static_cast<uintptr_t>(at + 64)));
}

// Stores of 16, 8 and 1 bytes to base + off; loads from base + off + step.  base and step are the same for the wave; an offset of
// BUFFER_NOWHERE stores nothing and reads zeros.  No branch: behind stores under a condition, which it cannot count, the compiler would
// make every later load's wait one for these stores as well.  (BUFFER_NOWHERE + step does not wrap: GATED_MOST_LD.)
// The stores take no step in a scalar register: a store of more than 8 bytes a lane still reads its data when the next instruction
// issues, and the compiler keeps that instruction from writing the data's registers only where the scalar offset is a constant (with a
// register, now and then the first four bytes of a lane's sixteen were others).
template <class V>
__device__ __forceinline__ void buffer_put(unsigned char* base, uint32_t off, V v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_make_buffer_rsrc(base, 0, static_cast<uint32_t>(BUFFER_SPAN), 0x00020000);
  if constexpr (sizeof(V) == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(g_u32x4, v), r, off, 0, 0);
  else if constexpr (sizeof(V) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(g_u32x2, v), r, off, 0, 0);
  else __builtin_amdgcn_raw_buffer_store_b8(v, r, off, 0, 0);
#endif
}
template <class V>
__device__ __forceinline__ V buffer_get(const unsigned char* base, uint32_t off, uint32_t step) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, static_cast<uint32_t>(BUFFER_SPAN), 0x00020000);
  if constexpr (sizeof(V) == 16) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(r, off, step, 0));
  else if constexpr (sizeof(V) == 8) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(r, off, step, 0));
  else return __builtin_amdgcn_raw_buffer_load_b8(r, off, step, 0);
#else
  return V{};
#endif
}

// The largest value over the four lanes that hold 16 columns each of a row's 32 (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ uint32_t max_over_lq(uint32_t v) {
  const g_u32x2 a = __builtin_bit_cast(g_u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
  v = max(a[0], a[1]);
  const g_u32x2 b = __builtin_bit_cast(g_u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));
  return max(b[0], b[1]);
}

__device__ __forceinline__ void store4(unsigned char* p, const float* v) { *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void load4(const unsigned char* p, float* v) {
  const f32x4_t t = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = t[q];
}

// The schedule's constructor, and its search for a tile's segment, read the segments' bounds one after the other; here a wave reads 64 at
// a time (2000 rows of 64 experts, forward 139.7 us / 131.5, gradient 322.9 / 314.6); the search so from 17 experts on: with 8 it is 1 % slower.
struct SegmentTiles {
  int tiles, incl, all;                            // row tiles of segment e0 + lane, of those up to it, of the 64
  template <int BM>
  __device__ __forceinline__ static SegmentTiles of(const int32_t* offsets, int E, int e0, int lane) {
    SegmentTiles m;
    const int q = e0 + lane;
    const int s = offsets[q < E ? q : E], t = offsets[q + 1 < E ? q + 1 : E];
    m.tiles = (t - s + BM - 1) / BM;               // (0 past the last segment)
    m.incl = m.tiles;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int up = __shfl_up(m.incl, off, 64);
      if (lane >= off) m.incl += up;
    }
    m.all = __builtin_amdgcn_readlane(m.incl, 63);
    return m;
  }
};
// The segment of the XCD's tile `item`, from which the schedule's search then starts.
template <int BM, class S>
__device__ __forceinline__ void gated_find(S& sched, int item, int lane) {
  const int tile = item < sched.rr ? ((item / S::RR) * 8 + sched.xcd) * S::RR + item % S::RR : sched.b0 + item - sched.rr;
  int before = 0;                                  // row tiles of the segments ahead of e0
  for (int e0 = 0; e0 < sched.E; e0 += 64) {
    const SegmentTiles m = SegmentTiles::of<BM>(sched.offsets, sched.E, e0, lane);
    const unsigned long long hit = __ballot((before + m.incl) * sched.nt > tile);
    if (hit != 0) {
      const int at = __builtin_ctzll(hit);
      sched.cur_e = e0 + at;
      sched.cur_base = (before + __builtin_amdgcn_readlane(m.incl, at) - __builtin_amdgcn_readlane(m.tiles, at)) * sched.nt;
      return;
    }
    before += m.all;
  }
}
// The share of an XCD of the row tiles of E segments.
template <int BM, class S>
__device__ __forceinline__ void gated_share(S& sched, int E, int lane) {
  int all = 0;
  for (int e0 = 0; e0 < E; e0 += 64) all += SegmentTiles::of<BM>(sched.offsets, E, e0, lane).all;
  const int routed = all * sched.nt;
  sched.E = E;
  sched.rr = routed / (8 * S::RR) * S::RR;
  const int rest = routed - 8 * sched.rr, chunk = (rest + 7) >> 3, mine = rest - sched.xcd * chunk;
  sched.b0 = 8 * sched.rr + sched.xcd * chunk;
  sched.ngemm = sched.rr + (mine < 0 ? 0 : mine > chunk ? chunk : mine);
}

// What workgroup `block` of `blocks` does of a product.
template <class CFG, int MODE, int KEEP, int ACT>
__device__ __forceinline__ void gated_product(const GatedArgs& p, const int block, const int blocks) {
  constexpr bool F32 = CFG::F32;
  constexpr int BM = CFG::BM, BN = CFG::BN, EB = CFG::EB, VE = CFG::VE, BK = CFG::BK, KS = CFG::KS, NS = CFG::NS;
  constexpr int MI = CFG::MI, NJ = CFG::NJ, TM = CFG::TM, TN = CFG::TN, STAGE = CFG::STAGE, A_BYTES = CFG::A_BYTES;
  constexpr int APW = CFG::APW, BPW = CFG::BPW, LPW = APW + BPW, NH = CFG::NH, H = MI / NH, APH = APW / NH;
  constexpr bool A_ACROSS = MODE == G_DW, B_ACROSS = MODE >= G_DH;
  constexpr int BNF = MODE == G_GATE ? BN / 2 : BN;             // columns of the output that a tile has
  constexpr int A_ROWB = BM / NH * EB, B_ROWB = BN * EB;        // across k: bytes of an LDS row (A: of a half of the tile's columns, see issue_a)
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, lq = lane >> 4;
  const int wave_m = wave / CFG::WN, wave_n = wave % CFG::WN;

  // ---- what this workgroup does: tiles slot, slot + nslots, ... of its XCD's share ---------------------------
  const int xcd = block & 7, nslots = blocks >> 3;
  int it = block >> 3;
  constexpr int GM = MODE == G_GATE || MODE == G_DH ? 6 : 4;
  using Schedule = TileSchedule<BM, BNF, GM>;
  constexpr int RR = Schedule::RR;
  // (constructed without segments: gated_share counts them)
  Schedule sched(MODE == G_DW ? 0 : p.j[0].nt, 0, p.offsets, 0, 1, false, 1, xcd, nslots);
  if constexpr (MODE != G_DW) gated_share<BM>(sched, p.E, lane);
  // DW: as many tiles for every expert; dealt like the schedule's
  const int dw_all = p.j[0].tiles + p.j[1].tiles;
  const int dw_dealt = dw_all / (8 * RR) * RR, dw_rest = dw_all - 8 * dw_dealt, dw_share = (dw_rest + 7) >> 3;
  int items = sched.ngemm;
  if (MODE == G_DW) {
    int more = dw_rest - xcd * dw_share;
    more = more < 0 ? 0 : more > dw_share ? dw_share : more;
    items = dw_dealt + more;
  }

  // ---- the tile in hand -----------------------------------------------------------------------------------
  int e = 0, row0 = 0, row_end = 0, n0 = 0, nk = 0, k_all = 0, which = 0;   // DW: row0, row_end are rows of the output
  const unsigned char* abase = nullptr;
  const unsigned char* bbase = nullptr;
  int64_t lda = 0, ldb = 0;
  uint32_t aoff[APW], boff[BPW];
  // A copy of the lane that what is worked out from it does not outlive its use: nothing of a tile's start or end takes registers of the
  // k loop.
  auto lane_here = [&]() {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };
  // Place of this lane's 16 bytes of copy i: row and first column (along k: of the k-tile's row; across: of the tile).
  auto a_row = [&](int i) {                      // along k: LDS row = tile row that copy i begins with
    constexpr int HALF = TM / NH;
    const int q = (wave * APH + i % APH) * 8;
    return (q / HALF) * TM + (i / APH) * HALF + q % HALF;
  };
  auto a_k = [&](int i, int ln) { return ((wave * APH + i % APH) * 1024) / A_ROWB + ln / (A_ROWB / 16); };   // across
  auto b_k = [&](int i, int ln) { return ((wave * BPW + i) * 1024) / B_ROWB + ln / (B_ROWB / 16); };
  auto setup = [&](int item) {
    const GatedJob* jb = &p.j[0];
    if constexpr (MODE == G_DW) {
      int t = item < dw_dealt ? ((item / RR) * 8 + xcd) * RR + item % RR : 8 * dw_dealt + xcd * dw_share + item - dw_dealt;
      which = t >= p.j[0].tiles ? 1 : 0;
      if (which) { t -= p.j[0].tiles; jb = &p.j[1]; }
      const int per = jb->mt * jb->nt;
      e = t / per;
      int m;
      sched.nt = jb->nt;
      sched.raster(t - e * per, jb->mt, m, n0);
      row0 = m * BM;
      row_end = jb->M;
      const int s = p.offsets[e];
      k_all = p.offsets[e + 1] - s;
      abase = jb->A + static_cast<int64_t>(s) * jb->lda * EB;
      bbase = jb->B + static_cast<int64_t>(s) * jb->ldb * EB;
    } else {
      if (p.E > 16) gated_find<BM>(sched, item, lane_here());
      sched.locate(item, e, row0, row_end, n0);
      k_all = jb->Kd;
      abase = jb->A + static_cast<int64_t>(row0) * jb->lda * EB;
      bbase = jb->B + static_cast<int64_t>(e) * (MODE == G_GATE ? 2 * jb->N : MODE == G_DOWN ? jb->N : jb->Kd) * jb->ldb * EB;
    }
    nk = (k_all + BK - 1) / BK;
    lda = jb->lda;
    ldb = jb->ldb;
    const int ln = lane_here();
#pragma unroll
    for (int i = 0; i < APW; ++i) {
      if constexpr (A_ACROSS) {
        const int k = a_k(i, ln), c = (ln % (A_ROWB / 16)) ^ (across_swz<F32, A_ROWB>(k) * (16 / VE));
        const int lc = c * VE, col = row0 + (lc / (TM / NH)) * TM + (i / APH) * (TM / NH) + lc % (TM / NH);
        aoff[i] = col < row_end ? static_cast<uint32_t>((static_cast<int64_t>(k) * lda + col) * EB) : BUFFER_NOWHERE;
      } else {
        const int r = a_row(i) + ln / 8, kc = (ln % 8) ^ swz<8>(r);
        aoff[i] = row0 + r < row_end ? static_cast<uint32_t>(static_cast<int64_t>(r) * lda * EB + kc * 16) : BUFFER_NOWHERE;
      }
    }
#pragma unroll
    for (int i = 0; i < BPW; ++i) {
      if constexpr (B_ACROSS) {
        const int k = b_k(i, ln), c = (ln % (B_ROWB / 16)) ^ (across_swz<F32, B_ROWB>(k) * (16 / VE));
        const int col = n0 + c * VE;
        boff[i] = col < jb->N ? static_cast<uint32_t>((static_cast<int64_t>(k) * ldb + col) * EB) : BUFFER_NOWHERE;
      } else {
        const int r = (wave * BPW + i) * 8 + ln / 8, kc = (ln % 8) ^ swz<8>(r);
        int n = n0 + r, row = n;
        if constexpr (MODE == G_GATE) {            // 64 columns of a wave: 32 of g, and the same 32 of u
          const int in = r % TN;
          n = n0 + (r / TN) * (TN / 2) + in % (TN / 2);
          row = n + (in / (TN / 2)) * jb->N;
        }
        boff[i] = n < jb->N ? static_cast<uint32_t>(static_cast<int64_t>(row - n0) * ldb * EB + kc * 16) : BUFFER_NOWHERE;
      }
    }
    if constexpr (!B_ACROSS) bbase += static_cast<int64_t>(n0) * ldb * EB;
  };
  // The last k-tile may be cut short: what lies past the end is not read (zeros).
  auto a_off = [&](int i, int kt, int ln) {
    const int k = A_ACROSS ? a_k(i, ln) : ((ln % 8) ^ swz<8>(a_row(i) + ln / 8)) * VE;
    return kt * BK + k < k_all ? aoff[i] : BUFFER_NOWHERE;
  };
  auto b_off = [&](int i, int kt, int ln) {
    const int k = B_ACROSS ? b_k(i, ln) : ((ln % 8) ^ swz<8>((wave * BPW + i) * 8 + ln / 8)) * VE;
    return kt * BK + k < k_all ? boff[i] : BUFFER_NOWHERE;
  };
  // whole_c: the k-tile is known to be whole
  auto issue_a = [&](int kt, int stage, auto half_c, auto whole_c) {
    constexpr int h = decltype(half_c)::value;
    const unsigned char* const base = A_ACROSS ? abase + static_cast<int64_t>(kt) * (BK * EB) * lda : abase;
    const uint32_t soff = A_ACROSS ? 0u : static_cast<uint32_t>(kt) * 128;
    // (across: the columns of the waves' first halves, then of their second halves, BK rows of A_ROWB bytes each)
    auto to = [&](int i) { return smem + stage * STAGE + (A_ACROSS ? h * (A_BYTES / NH) + (wave * APH + i % APH) * 1024 : a_row(i) * 128); };
    if (decltype(whole_c)::value || (kt + 1) * BK <= k_all) {
#pragma unroll
      for (int i = h * APH; i < (h + 1) * APH; ++i) buffer_to_lds16(base, to(i), aoff[i], soff);
    } else {
      const int ln = lane_here();
#pragma unroll
      for (int i = h * APH; i < (h + 1) * APH; ++i) buffer_to_lds16(base, to(i), a_off(i, kt, ln), soff);
    }
  };
  auto issue_b = [&](int kt, int stage, auto whole_c) {
    const unsigned char* const base = B_ACROSS ? bbase + static_cast<int64_t>(kt) * (BK * EB) * ldb : bbase;
    const uint32_t soff = B_ACROSS ? 0u : static_cast<uint32_t>(kt) * 128;
    unsigned char* const to = smem + stage * STAGE + A_BYTES + wave * BPW * 1024;
    if (decltype(whole_c)::value || (kt + 1) * BK <= k_all) {
#pragma unroll
      for (int i = 0; i < BPW; ++i) buffer_to_lds16(base, to + i * 1024, boff[i], soff);
    } else {
      const int ln = lane_here();
#pragma unroll
      for (int i = 0; i < BPW; ++i) buffer_to_lds16(base, to + i * 1024, b_off(i, kt, ln), soff);
    }
  };
  auto issue_ba0 = [&](int kt, int stage, auto whole_c) {
    issue_b(kt, stage, whole_c);
    issue_a(kt, stage, std::integral_constant<int, 0>{}, whole_c);
  };
  auto issue_a1 = [&](int kt, int stage, auto whole_c) {
    if constexpr (NH > 1) issue_a(kt, stage, std::integral_constant<int, 1>{}, whole_c);
  };
  auto issue_prologue = [&]() {
#pragma unroll
    for (int t = 0; t < NS; ++t)
      if (t < nk) {
        issue_ba0(t, t, std::false_type{});
        issue_a1(t, t, std::false_type{});
      }
  };
  auto wait_vm = [&](auto n_c) {
    constexpr int n = decltype(n_c)::value;
    static_assert(n < 64, "vmcnt field");
    __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | 0x0F70);
  };
  auto wait_tiles = [&](int tiles, auto extra_c) {      // at most so many k-tiles, and `extra` copies, still in flight
    constexpr int x = decltype(extra_c)::value;
    if (NS > 3 && tiles >= 3) wait_vm(std::integral_constant<int, 3 * LPW + x < 63 ? 3 * LPW + x : 63>{});
    else if (NS > 2 && tiles >= 2) wait_vm(std::integral_constant<int, 2 * LPW + x < 63 ? 2 * LPW + x : 63>{});
    else if (tiles >= 1) wait_vm(std::integral_constant<int, LPW + x>{});
    else wait_vm(std::integral_constant<int, x>{});
  };

  // ---- fragments -----------------------------------------------------------------------------------------
  unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(SCMOE_LDS_PTR(smem)));
  asm volatile("" : "+s"(lds0));
  constexpr int UNITB = 16 * EB;                          // bytes of 16 columns
  // Along k: address of (row l16, chunk of step s), the row block an immediate.  Across k: of this lane's first row of the step, the unit
  // (16 columns) swizzled per subtile: the swizzle of a lane's rows is the same throughout.
  const int kin = F32 ? lq * 4 : lq * 8 + (l16 >> 2);
  const unsigned in_unit = F32 ? l16 * 4 : (l16 & 3) * 8;
  unsigned xa[A_ACROSS ? H : KS], wb[B_ACROSS ? NJ : KS];
  if constexpr (A_ACROSS) {
#pragma unroll
    for (int i = 0; i < H; ++i) xa[i] = lds0 + kin * A_ROWB + (((wave_m * H + i) ^ across_swz<F32, A_ROWB>(kin)) * UNITB) + in_unit;
  } else {
#pragma unroll
    for (int s = 0; s < KS; ++s) xa[s] = lds0 + (wave_m * TM + l16) * 128 + (((s * 4 + lq) ^ swz<8>(l16)) << 4);
  }
  if constexpr (B_ACROSS) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) wb[j] = lds0 + A_BYTES + kin * B_ROWB + (((wave_n * TN / 16 + j) ^ across_swz<F32, B_ROWB>(kin)) * UNITB) + in_unit;
  } else {
#pragma unroll
    for (int s = 0; s < KS; ++s) wb[s] = lds0 + A_BYTES + (wave_n * TN + l16) * 128 + (((s * 4 + lq) ^ swz<8>(l16)) << 4);
  }
  typedef const __attribute__((address_space(3))) g_u32x4* lds16_ptr;
  typedef const __attribute__((address_space(3))) uint32_t* lds4_ptr;
  auto read_along = [&](unsigned at) { return *reinterpret_cast<lds16_ptr>(static_cast<uintptr_t>(at)); };
  auto read_across = [&](unsigned at, auto rowb_c) {
    constexpr int rowb = decltype(rowb_c)::value;
    g_u32x4 v;
    if constexpr (F32) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = *reinterpret_cast<lds4_ptr>(static_cast<uintptr_t>(at + c * rowb));
    } else {
      const g_u32x2 lo = lds_read_transposed(at), hi = lds_read_transposed(at + 4 * rowb);
      v = g_u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    return v;
  };
  constexpr int KROWS = BK / KS;                          // rows of k in a step
  f32x4_t acc[MI][NJ];
  g_u32x4 wf[2][NJ], xf[2][H];
  static_assert((NS * KS) % 2 == 0, "the weight-fragment buffers alternate over the unrolled k loop");
  // halves_c: how many halves of its rows the wave has (those past the segment are not read or multiplied)
  auto load_frags = [&](int R, int hs, auto halves_c) {   // half-step hs: step hs % KS, row-subtile half hs / KS
    if (hs / KS >= decltype(halves_c)::value) return;
    const int s = hs % KS, half = hs / KS, st = R * STAGE, wbuf = (R * KS + s) & 1, xbuf = hs & 1;
#pragma unroll
    for (int t = 0; t < (H > NJ ? H : NJ); ++t) {
      if (half == 0 && t < NJ) {
        if constexpr (B_ACROSS) wf[wbuf][t] = read_across(wb[t] + st + s * KROWS * B_ROWB, std::integral_constant<int, B_ROWB>{});
        else wf[wbuf][t] = read_along(wb[s] + st + t * 16 * 128);
      }
      if (t < H) {
        if constexpr (A_ACROSS) xf[xbuf][t] = read_across(xa[t] + st + half * (A_BYTES / NH) + s * KROWS * A_ROWB, std::integral_constant<int, A_ROWB>{});
        else xf[xbuf][t] = read_along(xa[s] + st + (half * H + t) * 16 * 128);
      }
    }
  };
  auto mfma_step = [&](int R, int hs, auto halves_c) {
    if (hs / KS >= decltype(halves_c)::value) return;
    const int s = hs % KS, half = hs / KS, wbuf = (R * KS + s) & 1, xbuf = hs & 1;
#pragma unroll
    for (int c = 0; c < (F32 ? 4 : 1); ++c)
#pragma unroll
      for (int i = 0; i < H; ++i)
#pragma unroll
        for (int jj = 0; jj < NJ; ++jj) {
          const int j = (i & 1) ? NJ - 1 - jj : jj;       // there and back: one operand changes at a time
          f32x4_t& a = acc[half * H + i][j];
          if constexpr (F32) a = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(wf[wbuf][j][c]), __uint_as_float(xf[xbuf][i][c]), a, 0, 0, 0);
          else a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, wf[wbuf][j]), __builtin_bit_cast(bf16x8_t, xf[xbuf][i]), a, 0, 0, 0);
        }
  };
  // issue order of a half-step: a matrix instruction, then reads for the next half-step
  auto interleave = [&](auto hs_c, auto next_hs_c, auto halves_c) {
    constexpr int halves = decltype(halves_c)::value, next = decltype(next_hs_c)::value / KS;
    if constexpr (decltype(hs_c)::value / KS >= halves) return;
    constexpr int RA = A_ACROSS ? (F32 ? 4 : 2) : 1, RB = B_ACROSS ? (F32 ? 4 : 2) : 1;
    constexpr int reads = next >= halves ? 0 : H * RA + (next ? 0 : NJ * RB);
    constexpr int mfmas = H * NJ * (F32 ? 4 : 1), per = reads > mfmas ? (reads + mfmas - 1) / mfmas : 1, groups = reads / per;
#pragma unroll
    for (int q = 0; q < groups; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, per, 0);
    }
    if constexpr (reads % per != 0) __builtin_amdgcn_sched_group_barrier(0x100, reads % per, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, mfmas - groups, 0);
  };

  if (it >= items) return;
  setup(it);
  issue_prologue();
  if (MODE == G_GATE && p.zero != nullptr && block == 0)
    for (int i = threadIdx.x; i < p.zeros; i += CFG::THREADS) p.zero[i] = 0;
  for (;;) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    wait_vm(std::integral_constant<int, 0>{});
    lds_barrier();
    constexpr int HS = NH * KS;
    using X0 = std::integral_constant<int, 0>;
    using XA1 = std::integral_constant<int, (NH - 1) * APH>;
    // One k-tile (the order of its half-steps, copies and barriers is gemm_bf16_kernel's): B and the first halves of the rows are
    // refilled with k-tile kt + NS while the second halves are multiplied, these behind a second barrier.  Without halves the whole stage
    // is refilled ahead of the last step, when its fragments are in registers.
    auto k_tile = [&](auto stage_c, auto steady_c, auto halves_c, int kt) {
      constexpr int stage = decltype(stage_c)::value;
      constexpr bool steady = decltype(steady_c)::value;      // k-tiles kt + 1 .. kt + NS all exist, and are whole
      constexpr int next = stage + 1 == NS ? 0 : stage + 1;
      static_for<0, HS>([&](auto hs_c) {
        constexpr int hs = decltype(hs_c)::value;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (NH > 1 && hs == KS - 1) {
          if constexpr (steady) wait_tiles(NS - 1, X0{});
          else wait_tiles(nk - 1 - kt < NS - 1 ? nk - 1 - kt : NS - 1, X0{});
          lds_barrier();
          if (steady || kt + NS < nk) issue_ba0(kt + NS, stage, steady_c);
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (hs == HS - 1) {
          if (steady || kt + 1 < nk) {
            if constexpr (NH > 1) {
              if (steady || kt + NS < nk) wait_tiles(NS - 1, X0{});
              else wait_tiles(nk - 2 - kt, XA1{});
            } else {
              // k-tile kt + 1 must have landed; in flight may be those after it, up to kt + NS - 1
              if constexpr (steady) wait_tiles(NS - 2, X0{});
              else wait_tiles(nk - 2 - kt < NS - 2 ? nk - 2 - kt : NS - 2, X0{});
            }
            lds_barrier();
            if (steady || kt + NS < nk) {
              if constexpr (NH > 1) issue_a1(kt + NS, stage, steady_c);
              else issue_ba0(kt + NS, stage, steady_c);
            }
            __builtin_amdgcn_sched_barrier(0);
            load_frags(next, 0, halves_c);
          }
          mfma_step(stage, hs, halves_c);
          if constexpr (steady) interleave(hs_c, std::integral_constant<int, 0>{}, halves_c);
        } else {
          load_frags(stage, hs + 1, halves_c);
          mfma_step(stage, hs, halves_c);
          interleave(hs_c, std::integral_constant<int, hs + 1>{}, halves_c);
        }
      });
    };
    using std::bool_constant;
    using std::integral_constant;
    // fp32: a sum is made of parts of some 16 k-tiles (512 products), whose chains are short: dx of 200 rows, d = 2048, F = 8192
    // (16384 products) is 6.0e-7 off so, in the 2-norm, 2.4e-6 in one chain; the time is 1 % more.
    constexpr int PART = 16;
    f32x4_t sum[F32 ? MI : 1][F32 ? NJ : 1];
    auto next_part = [&](auto first_c) {
#pragma unroll
      for (int i = 0; i < (F32 ? MI : 0); ++i)
#pragma unroll
        for (int j = 0; j < (F32 ? NJ : 0); ++j) {
          sum[i][j] = decltype(first_c)::value ? f32x4_t{0.0f, 0.0f, 0.0f, 0.0f} : sum[i][j] + acc[i][j];
          acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
    };
    next_part(std::true_type{});
    auto multiply = [&](auto halves_c) {
      load_frags(0, 0, halves_c);
      int kt = 0;
      const int whole = k_all / BK;
      auto turn = [&]() { static_for<0, NS>([&](auto s) { k_tile(s, bool_constant<true>{}, halves_c, kt + decltype(s)::value); }); };
      if constexpr (F32) {
        while (kt + 2 * NS <= whole) {
          const int end = kt + PART < whole ? kt + PART : whole;
          for (; kt < end && kt + 2 * NS <= whole; kt += NS) turn();
          next_part(std::false_type{});
        }
      } else {
        for (; kt + 2 * NS <= whole; kt += NS) turn();
      }
      for (; kt < nk; kt += NS)
        static_for<0, NS>([&](auto s) {
          if (kt + decltype(s)::value < nk) k_tile(s, bool_constant<false>{}, halves_c, kt + decltype(s)::value);
        });
    };
    if (nk > 0) {
      // DX, whose tiles stay with few rows for a long k where it shares a launch with DW: a wave without rows, or with a half of them, leaves
      // out the products of the others (gradient of 2000 rows, d = 768, F = 2048, E = 64 283 us, so 270; 4000, 1024, 1024, 64 216, so 199).  The
      // other products gain nothing (their time is the weights').
      const int rows_here = row_end - row0 - wave_m * TM;
      if (MODE == G_DX && NH > 1 && rows_here <= 0) multiply(integral_constant<int, 0>{});
      else if (MODE == G_DX && NH > 1 && rows_here <= H * 16) multiply(integral_constant<int, 1>{});
      else multiply(integral_constant<int, NH>{});
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] += sum[i][j];
      }
    }
    lds_barrier();                                  // every wave holds its last fragments: LDS is free

    const GatedJob& jc = p.j[MODE == G_DW ? which : 0];
    const int ce = e, crow0 = row0, crow_end = row_end, cn0 = n0;
    unsigned char* const cC = jc.C;
    const int64_t cldc = jc.ldc;
    const int cN = jc.N;
    const int itn = MODE == G_DW ? it + nslots : sched.next(it);
    const bool more = itn < items;
    // bf16: an output row's 16-byte pieces as a wave stores them, 8 rows at a time: lane l has piece l % 8 of row l / 8, and of row
    // 8 + l / 8, of a subtile of 16 rows.  Offsets are from the wave tile's first row.
    const int le = lane_here(), pr = le >> 3, pc = le & 7;
    const int l16 = le & 15, lq = le >> 4;
    const int pn = cn0 + wave_n * TN + pc * 8;                 // its first column
    const int wrow0 = crow0 + wave_m * TM, left = crow_end - wrow0;           // rows that the wave tile has
    unsigned char* const obase = cC + (MODE == G_DW ? static_cast<int64_t>(ce) * jc.M + wrow0 : static_cast<int64_t>(wrow0)) * cldc * EB;
    unsigned char* const kbase = p.pre + static_cast<int64_t>(wrow0) * (KEEP == KEEP_8BIT ? 2 * p.ldpre : p.ldpre * EB);
    unsigned char* const dbase = p.dpre + static_cast<int64_t>(wrow0) * p.lddpre * EB;
    const uint32_t ostep = static_cast<uint32_t>(cldc) * EB, dstep = static_cast<uint32_t>(p.lddpre) * EB;
    const uint32_t kstep = KEEP == KEEP_8BIT ? static_cast<uint32_t>(p.ldpre) * 2 : static_cast<uint32_t>(p.ldpre) * EB;   // of a row: two checkpoint rows
    const uint32_t ubytes = KEEP == KEEP_8BIT ? static_cast<uint32_t>(p.ldpre) : static_cast<uint32_t>(cN) * EB;         // from g to u
    const uint32_t dubytes = static_cast<uint32_t>(cN) * EB;
    auto if_in = [&](bool in, uint32_t off) { return in ? off : BUFFER_NOWHERE; };
    // DH: g and u of a subtile's pieces (8 bits: codes, and the blocks' scales), a subtile ahead of their use
    g_u32x4 kg[2][2], ku[2][2];
    auto load_kept = [&](int i) {
      if constexpr (MODE == G_DH && !F32) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int rr = i * 16 + t * 8;
          const bool in = rr + pr < left && pn < cN;
          if constexpr (KEEP == KEEP_8BIT) {
            const uint32_t row = static_cast<uint32_t>(pr) * kstep, step = static_cast<uint32_t>(rr) * kstep;
            const uint32_t codes = if_in(in, row + pn), scale = if_in(in, row + cN + pn / CKPT_BLOCK);
            const g_u32x2 a = buffer_get<g_u32x2>(kbase, codes, step), b = buffer_get<g_u32x2>(kbase + ubytes, codes, step);
            kg[i & 1][t] = g_u32x4{a[0], a[1], buffer_get<unsigned char>(kbase, scale, step), buffer_get<unsigned char>(kbase + ubytes, scale, step)};
            ku[i & 1][t] = g_u32x4{b[0], b[1], 0, 0};
          } else {
            const uint32_t off = if_in(in, static_cast<uint32_t>(pr) * kstep + pn * EB), step = static_cast<uint32_t>(rr) * kstep;
            kg[i & 1][t] = buffer_get<g_u32x4>(kbase, off, step);
            ku[i & 1][t] = buffer_get<g_u32x4>(kbase + ubytes, off, step);
          }
        }
      }
    };
    load_kept(0);
    if (more) {
      setup(itn);
      issue_prologue();
    }

    // ---- store: acc[i][j][q] is row l16 of subtile i, column 4 lq + q of subtile j -----------------------------
    // bf16: rows are put together in the wave's patch of LDS, a subtile of 16 rows at a time, and leave it as whole lines.
    unsigned char* const patch = smem + NS * STAGE + wave * CFG::PATCH;
    if constexpr (!F32) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (i * 16 >= left) break;                             // (wave-uniform)
        wave_lds_order();                                      // (the patch has been read)
        __builtin_amdgcn_sched_barrier(0);                     // (a subtile at a time: several take registers that are not there)
        if constexpr (MODE == G_DH) {
          if (i + 1 < MI) load_kept(i + 1);
          // dh in fp32: 16 rows of 256 bytes, chunks swizzled by the row
#pragma unroll
          for (int j = 0; j < NJ; ++j) *reinterpret_cast<f32x4_t*>(patch + l16 * 256 + (((j * 4 + lq) ^ l16) << 4)) = acc[i][j];
          wave_lds_order();
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int rr = t * 8 + pr;
            float dh[8], g[8], u[8], h[8];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const f32x4_t v = *reinterpret_cast<const f32x4_t*>(patch + rr * 256 + (((pc * 2 + c) ^ rr) << 4));
#pragma unroll
              for (int q = 0; q < 4; ++q) dh[c * 4 + q] = v[q];
            }
            const g_u32x4 wg = kg[i & 1][t], wu = ku[i & 1][t];
            if constexpr (KEEP == KEEP_8BIT) {
              const float sg = ckpt_scale(wg[2]), su = ckpt_scale(wg[3]);
              ckpt_decode4(wg[0], sg, g);
              ckpt_decode4(wg[1], sg, g + 4);
              ckpt_decode4(wu[0], su, u);
              ckpt_decode4(wu[1], su, u + 4);
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                g[2 * q] = __uint_as_float(wg[q] << 16);
                g[2 * q + 1] = __uint_as_float(wg[q] & 0xffff0000u);
                u[2 * q] = __uint_as_float(wu[q] << 16);
                u[2 * q + 1] = __uint_as_float(wu[q] & 0xffff0000u);
              }
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              float a, s;
              gated_act_slope<F32, ACT>(g[q], a, s);
              h[q] = a * u[q];
              g[q] = dh[q] * u[q] * s;
              u[q] = dh[q] * a;
            }
            auto pack8 = [&](const float* v) { return g_u32x4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])}; };
            const g_u32x4 oh = pack8(h), og = pack8(g), ou = pack8(u);
            const bool in = i * 16 + rr < left && pn < cN;
            buffer_put(obase + static_cast<int64_t>(i * 16 + t * 8) * ostep, if_in(in, static_cast<uint32_t>(pr) * ostep + pn * 2), oh);
            const uint32_t to = if_in(in, static_cast<uint32_t>(pr) * dstep + pn * 2);
            buffer_put(dbase + static_cast<int64_t>(i * 16 + t * 8) * dstep, to, og);
            buffer_put(dbase + dubytes + static_cast<int64_t>(i * 16 + t * 8) * dstep, to, ou);
          }
        } else if constexpr (MODE == G_GATE) {
          // 32 columns a wave: hidden, g, u in 16 rows of 64 bytes each (in 8 bits: of 32), one behind the other
          constexpr int J2 = NJ / 2;
          static_assert(J2 * 16 == CKPT_BLOCK, "a wave has one block of g and of u");
          const int f0 = cn0 + wave_n * (TN / 2);
          uint32_t byte[2] = {0, 0};
          float inv[2] = {0.0f, 0.0f};
          if constexpr (KEEP == KEEP_8BIT) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              uint32_t most = 0;
#pragma unroll
              for (int j = 0; j < J2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) most = max(most, magnitude(acc[i][t * J2 + j][q]));
              byte[t] = ckpt_scale_byte(max_over_lq(most));
              inv[t] = ckpt_inverse(byte[t]);
            }
          }
          const int sw = (l16 >> 1) & 3;                       // 64-byte rows: chunks of 16 bytes, swizzled
#pragma unroll
          for (int j = 0; j < J2; ++j) {
            float h[4];
            const f32x4_t g = acc[i][j], u = acc[i][J2 + j];
#pragma unroll
            for (int q = 0; q < 4; ++q) h[q] = gated_act<F32, ACT>(g[q]) * u[q];
            const int at = l16 * 64 + (((j * 2 + (lq >> 1)) ^ sw) << 4) + (lq & 1) * 8;
            *reinterpret_cast<uint2*>(patch + at) = make_uint2(cvt_pk_bf16(h[0], h[1]), cvt_pk_bf16(h[2], h[3]));
            if constexpr (KEEP == KEEP_FULL) {
              *reinterpret_cast<uint2*>(patch + 1024 + at) = make_uint2(cvt_pk_bf16(g[0], g[1]), cvt_pk_bf16(g[2], g[3]));
              *reinterpret_cast<uint2*>(patch + 2048 + at) = make_uint2(cvt_pk_bf16(u[0], u[1]), cvt_pk_bf16(u[2], u[3]));
            } else if constexpr (KEEP == KEEP_8BIT) {
              *reinterpret_cast<uint32_t*>(patch + 1024 + l16 * 32 + j * 16 + lq * 4) = ckpt_encode4(g[0], g[1], g[2], g[3], inv[0]);
              *reinterpret_cast<uint32_t*>(patch + 1536 + l16 * 32 + j * 16 + lq * 4) = ckpt_encode4(u[0], u[1], u[2], u[3], inv[1]);
            }
          }
          wave_lds_order();
          {
            const int rr = le >> 2, c = le & 3, f = f0 + c * 8;
            const int at = rr * 64 + ((c ^ ((rr >> 1) & 3)) << 4);
            const bool in = i * 16 + rr < left && f < cN;
            buffer_put(obase + static_cast<int64_t>(i * 16) * ostep, if_in(in, static_cast<uint32_t>(rr) * ostep + f * 2), *reinterpret_cast<const g_u32x4*>(patch + at));
            if constexpr (KEEP == KEEP_FULL) {
              const uint32_t to = if_in(in, static_cast<uint32_t>(rr) * kstep + f * 2);
              buffer_put(kbase + static_cast<int64_t>(i * 16) * kstep, to, *reinterpret_cast<const g_u32x4*>(patch + 1024 + at));
              buffer_put(kbase + ubytes + static_cast<int64_t>(i * 16) * kstep, to, *reinterpret_cast<const g_u32x4*>(patch + 2048 + at));
            }
          }
          if constexpr (KEEP == KEEP_8BIT) {
            // lane l: 16 codes, half l % 2 of row l / 2 % 16 of g (lanes 0 .. 31) or u; the width is a multiple of 8
            const int t = le >> 5, rr = (le >> 1) & 15, c = le & 1, f = f0 + c * 16;
            const g_u32x4 codes = *reinterpret_cast<const g_u32x4*>(patch + 1024 + t * 512 + rr * 32 + c * 16);
            const uint32_t to = static_cast<uint32_t>(rr) * kstep + t * ubytes + f;
            const bool row = i * 16 + rr < left;
            buffer_put(kbase + static_cast<int64_t>(i * 16) * kstep, if_in(row && f + 16 <= cN, to), codes);
            buffer_put(kbase + static_cast<int64_t>(i * 16) * kstep, if_in(row && f + 8 == cN, to), g_u32x2{codes[0], codes[1]});
            const uint32_t ts = static_cast<uint32_t>(l16) * kstep + lq * ubytes + cN + f0 / CKPT_BLOCK;
            buffer_put(kbase + static_cast<int64_t>(i * 16) * kstep, if_in(lq < 2 && i * 16 + l16 < left && f0 < cN, ts), static_cast<unsigned char>(lq == 0 ? byte[0] : byte[1]));
          }
        } else {
          unsigned char* const half = patch + (CFG::PATCH > 2048 ? (i & 1) * 2048 : 0);   // 16 rows of 128 bytes
#pragma unroll
          for (int j = 0; j < NJ; ++j)
            *reinterpret_cast<uint2*>(half + l16 * 128 + (((2 * j + (lq >> 1)) ^ swz<8>(l16)) << 4) + (lq & 1) * 8) =
                make_uint2(cvt_pk_bf16(acc[i][j][0], acc[i][j][1]), cvt_pk_bf16(acc[i][j][2], acc[i][j][3]));
          wave_lds_order();
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int rr = t * 8 + pr;
            const g_u32x4 v = *reinterpret_cast<const g_u32x4*>(half + rr * 128 + ((pc ^ swz<8>(rr)) << 4));
            buffer_put(obase + static_cast<int64_t>(i * 16 + t * 8) * ostep, if_in(i * 16 + rr < left && pn < cN, static_cast<uint32_t>(pr) * ostep + pn * 2), v);
          }
        }
      }
    } else {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int r = crow0 + wave_m * TM + i * 16 + l16;
      const bool in = r < crow_end;
      if constexpr (MODE == G_GATE) {
        constexpr int J2 = NJ / 2;
        static_assert(J2 * 16 == CKPT_BLOCK, "a wave has one block of g and of u");
        const int f0 = cn0 + wave_n * (TN / 2);
#pragma unroll
        for (int j = 0; j < J2; ++j) {
          const int f = f0 + j * 16 + 4 * lq;
          float h[4], g[4], u[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            g[q] = acc[i][j][q];
            u[q] = acc[i][J2 + j][q];
            h[q] = gated_act<F32, ACT>(g[q]) * u[q];
          }
          if (in && f < cN) {
            store4(cC + (static_cast<int64_t>(r) * cldc + f) * EB, h);
            if constexpr (KEEP == KEEP_FULL) {
              store4(p.pre + (static_cast<int64_t>(r) * p.ldpre + f) * EB, g);
              store4(p.pre + (static_cast<int64_t>(r) * p.ldpre + cN + f) * EB, u);
            }
          }
        }
        if constexpr (KEEP == KEEP_8BIT) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t most = 0;
#pragma unroll
            for (int j = 0; j < J2; ++j)
#pragma unroll
              for (int q = 0; q < 4; ++q) most = max(most, magnitude(acc[i][t * J2 + j][q]));
            most = max_over_lq(most);
            const uint32_t byte = ckpt_scale_byte(most);
            const float inv = ckpt_inverse(byte);
            unsigned char* const row = p.pre + (2 * static_cast<int64_t>(r) + t) * p.ldpre;
#pragma unroll
            for (int j = 0; j < J2; ++j) {
              const int f = f0 + j * 16 + 4 * lq;
              const f32x4_t& a = acc[i][t * J2 + j];
              if (in && f < cN) *reinterpret_cast<uint32_t*>(row + f) = ckpt_encode4(a[0], a[1], a[2], a[3], inv);
            }
            if (in && lq == 0 && f0 < cN) row[cN + f0 / CKPT_BLOCK] = static_cast<unsigned char>(byte);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int n = cn0 + wave_n * TN + j * 16 + 4 * lq;
          float v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q];
          if (!in || n >= cN) continue;
          if constexpr (MODE == G_DH) {
            float g[4], u[4], h[4], dg[4], du[4];
            if constexpr (KEEP == KEEP_8BIT) {
              const unsigned char* row = p.pre + 2 * static_cast<int64_t>(r) * p.ldpre;
              ckpt_decode4(*reinterpret_cast<const uint32_t*>(row + n), ckpt_scale(row[cN + n / CKPT_BLOCK]), g);
              row += p.ldpre;
              ckpt_decode4(*reinterpret_cast<const uint32_t*>(row + n), ckpt_scale(row[cN + n / CKPT_BLOCK]), u);
            } else {
              load4(p.pre + (static_cast<int64_t>(r) * p.ldpre + n) * EB, g);
              load4(p.pre + (static_cast<int64_t>(r) * p.ldpre + cN + n) * EB, u);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float a, s;
              gated_act_slope<F32, ACT>(g[q], a, s);
              h[q] = a * u[q];
              du[q] = v[q] * a;
              dg[q] = v[q] * u[q] * s;
            }
            store4(cC + (static_cast<int64_t>(r) * cldc + n) * EB, h);
            store4(p.dpre + (static_cast<int64_t>(r) * p.lddpre + n) * EB, dg);
            store4(p.dpre + (static_cast<int64_t>(r) * p.lddpre + cN + n) * EB, du);
          } else {
            const int64_t at = MODE == G_DW ? (static_cast<int64_t>(ce) * jc.M + r) * cldc + n : static_cast<int64_t>(r) * cldc + n;
            store4(cC + at * EB, v);
          }
        }
      }
    }
    }
    it = itn;
    if (!more) break;
  }
}

template <class CFG, int MODE, int KEEP, int ACT>
__global__ __launch_bounds__(CFG::THREADS, CFG::WG_PER_CU * CFG::WAVES / 4) void gated_kernel(const GatedArgs p) {
  gated_product<CFG, MODE, KEEP, ACT>(p, blockIdx.x, gridDim.x);
}

// DX and DW, which both wait for DH alone, in one launch: the first xblocks workgroups have DX, the others DW.  By itself DX, one to two rounds
// of long tiles, often leaves a good part of the compute units without work, and both have a start and an end.
template <class X_, class W_>
struct GatedPair {
  using X = X_;
  using W = W_;
  static constexpr int LDS = X::LDS > W::LDS ? X::LDS : W::LDS;
  static constexpr int WG_PER_CU = X::WG_PER_CU < W::WG_PER_CU ? X::WG_PER_CU : W::WG_PER_CU;
  static_assert(X::THREADS == W::THREADS, "one launch");
};
template <class P>
__global__ __launch_bounds__(P::X::THREADS, P::WG_PER_CU * P::X::WAVES / 4) void gated_pair_kernel(const GatedArgs x, const GatedArgs w, const int xblocks) {
  const int block = blockIdx.x;
  if (block < xblocks) gated_product<typename P::X, G_DX, KEEP_NONE, 0>(x, block, xblocks);
  else gated_product<typename P::W, G_DW, KEEP_NONE, 0>(w, block - xblocks, gridDim.x - xblocks);
}

// ---- host side ----------------------------------------------------------------------------------------------

// LDS of a kernel's launches, said once a device.
template <class KERNEL>
static int allow_lds(KERNEL* kernel, int bytes, std::atomic<bool>* said) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = -1;
  if (dev < 0 || !said[dev].load(std::memory_order_acquire)) {
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err != hipSuccess) return hip_fail(err);
    if (dev >= 0) said[dev].store(true, std::memory_order_release);
  }
  return SCMOE_OK;
}

// Tiles of a launch's products as the host expects them: an expert's last row tile half full, unless the average leaves room in one.
inline double likely_tiles(const GatedArgs& a, int mode, int64_t max_rows, int rows, int cols) {
  const double segs = static_cast<double>(a.E < max_rows ? a.E : max_rows), mean = max_rows > 0 ? static_cast<double>(max_rows) / segs : 0.0;
  double n = 0;
  for (const GatedJob& j : a.j) {
    if (j.C == nullptr) continue;
    const double across = (j.N + cols - 1) / cols;
    n += across * (mode == G_DW ? static_cast<double>((j.M + rows - 1) / rows) * a.E : segs * (mean <= 0.75 * rows ? 1.0 : mean / rows + 0.5));
  }
  return n;
}

// Fills in the tiles of a launch's products; returns how many there are at most.
template <class CFG, int MODE>
static int64_t count_tiles(GatedArgs& a, int64_t max_rows) {
  constexpr int BNF = MODE == G_GATE ? CFG::BN / 2 : CFG::BN;
  int64_t tiles = 0;
  for (GatedJob& j : a.j) {
    if (j.C == nullptr) continue;                       // (no second product)
    j.nt = (j.N + BNF - 1) / BNF;
    if (MODE == G_DW) {
      j.mt = (j.M + CFG::BM - 1) / CFG::BM;
      j.tiles = a.E * j.mt * j.nt;                       // (check_gated: they fit)
      tiles += j.tiles;
    } else {
      // sum_e ceil(c_e / BM) is at most rows / BM and one more for every segment that can hold a row
      tiles += (max_rows / CFG::BM + (a.E < max_rows ? a.E : max_rows)) * j.nt;
    }
  }
  return tiles;
}

template <class CFG, int MODE, int KEEP, int ACT>
static int launch_gated_cfg(GatedArgs a, int64_t max_rows, hipStream_t stream) {
  static std::atomic<bool> said[64];
  const int st = allow_lds(&gated_kernel<CFG, MODE, KEEP, ACT>, CFG::LDS, said);
  if (st != SCMOE_OK) return st;
  int64_t slots = (count_tiles<CFG, MODE>(a, max_rows) + 7) / 8;
  const int resident = (num_cus() / 8) * CFG::WG_PER_CU;
  if (slots > resident) slots = resident;
  if (slots < 1) slots = 1;
  hipLaunchKernelGGL((gated_kernel<CFG, MODE, KEEP, ACT>), dim3(static_cast<unsigned>(8 * slots)), dim3(CFG::THREADS), CFG::LDS, stream, a);
  return launch_status();
}

// A tile's time, in products of a k-tile's width: its k-tiles, and three for its start and end.
template <class CFG, int MODE>
static double tile_cost(const GatedArgs& a, int64_t max_rows) {
  const double k = MODE == G_DW ? static_cast<double>(max_rows) / a.E / CFG::BK + 0.5 : a.j[0].Kd / CFG::BK;
  return (k + 3.0) * CFG::BM * CFG::BN;
}

// (DX's tiles as expected, not as many as there may be: 4000 rows, d = 512, F = 2048, E = 64, gradient 226 us, the other way 264.)
template <class X, class W>
static int pair_resident() {
  const int each = (num_cus() / 8) * GatedPair<X, W>::WG_PER_CU;
  return each < 2 ? 2 : each;
}
template <class X, class W>
static PairShare share_gated_pair(const GatedArgs& x, const GatedArgs& w, int64_t max_rows) {
  return share_pair(likely_tiles(x, G_DX, max_rows, X::BM, X::BN), tile_cost<X, G_DX>(x, max_rows), likely_tiles(w, G_DW, max_rows, W::BM, W::BN),
                    tile_cost<W, G_DW>(w, max_rows), pair_resident<X, W>(), num_cus());
}

template <class X, class W>
static int launch_gated_pair(GatedArgs x, GatedArgs w, int64_t max_rows, hipStream_t stream) {
  using P = GatedPair<X, W>;
  static std::atomic<bool> said[64];
  const int st = allow_lds(&gated_pair_kernel<P>, P::LDS, said);
  if (st != SCMOE_OK) return st;
  count_tiles<X, G_DX>(x, max_rows);
  count_tiles<W, G_DW>(w, max_rows);
  hipLaunchKernelGGL((gated_pair_kernel<P>), dim3(static_cast<unsigned>(8 * pair_resident<X, W>())), dim3(X::THREADS), P::LDS, stream, x, w,
                     8 * share_gated_pair<X, W>(x, w, max_rows).first);
  return launch_status();
}

// One launch of a product (DW: of one or two), of either type.
int launch_gated_bf16(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream);
int launch_gated_f32(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream);
// DX and DW, in one launch where that is better.
int launch_gated_gradients_bf16(const GatedArgs& x, const GatedArgs& w, int64_t max_rows, hipStream_t stream);
int launch_gated_gradients_f32(const GatedArgs& x, const GatedArgs& w, int64_t max_rows, hipStream_t stream);

// GATE (kept in full or not at all) and DOWN of a few rows.
int launch_gated_few(const GatedArgs& a, int mode, int keep, int64_t max_rows, int dtype, hipStream_t stream);

template <class CFG, int MODE, int KEEP>
static int launch_gated_act(const GatedArgs& a, int64_t max_rows, hipStream_t stream) {
  switch (a.act) {
    case SCMOE_SILU: return launch_gated_cfg<CFG, MODE, KEEP, SCMOE_SILU>(a, max_rows, stream);
    case SCMOE_GELU_TANH: return launch_gated_cfg<CFG, MODE, KEEP, SCMOE_GELU_TANH>(a, max_rows, stream);
    default: return launch_gated_cfg<CFG, MODE, KEEP, SCMOE_GELU_ERF>(a, max_rows, stream);
  }
}

template <class CFG>
static int launch_gated_rows(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  switch (mode) {
    case G_GATE:
      return keep == KEEP_NONE ? launch_gated_act<CFG, G_GATE, KEEP_NONE>(a, max_rows, stream)
             : keep == KEEP_FULL ? launch_gated_act<CFG, G_GATE, KEEP_FULL>(a, max_rows, stream)
                                 : launch_gated_act<CFG, G_GATE, KEEP_8BIT>(a, max_rows, stream);
    case G_DH:
      return keep == KEEP_FULL ? launch_gated_act<CFG, G_DH, KEEP_FULL>(a, max_rows, stream) : launch_gated_act<CFG, G_DH, KEEP_8BIT>(a, max_rows, stream);
    case G_DOWN: return launch_gated_cfg<CFG, G_DOWN, KEEP_NONE, 0>(a, max_rows, stream);
    default: return launch_gated_cfg<CFG, G_DX, KEEP_NONE, 0>(a, max_rows, stream);
  }
}
template <class CFG>
static int launch_gated_mode(const GatedArgs& a, int mode, int keep, int64_t max_rows, hipStream_t stream) {
  if (mode == G_DW) return launch_gated_cfg<CFG, G_DW, KEEP_NONE, 0>(a, max_rows, stream);
  return launch_gated_rows<CFG>(a, mode, keep, max_rows, stream);
}

}  // namespace scmoe
