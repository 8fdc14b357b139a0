// Activation checkpoints in 8 bits (checkpoint.hpp): rows packed and restored.
//
// Bound by HBM: a value is read and a little over a byte written, or the other way round.  A lane has pieces of 16 bytes of x (four
// lanes a block in bf16, eight in fp32), so that every load and store of a wave is of whole lines (pieces of 32 bytes, stored in halves:
// unpack 144 us -> 318); the block's largest magnitude comes by lane moves.  A workgroup walks over the pieces of as many rows as there are, four a turn, whose loads are in flight together;
// where a piece lies is counted on, not divided out.  32768 x 8192 in bf16, pack and unpack: 289 us,
// 5.6 TB/s.
#include "checkpoint.hpp"
#include "rows.hpp"

namespace scmoe {

struct CkptArgs {
  unsigned char* x; int64_t ldx;          // strides in bytes
  unsigned char* q; int64_t ldq;
  const int32_t* n_rows; int64_t max_rows;
  int width, pieces;                      // pieces of a row, of whole blocks
  int64_t row_step; int col_step;         // from a lane's piece to its next one
};

constexpr int CKPT_THREADS = 256, CKPT_TURN = 4;

template <bool ST>
__device__ __forceinline__ void store8(unsigned char* p, uint2 q) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  if (ST) __builtin_nontemporal_store(u32x2_t{q.x, q.y}, reinterpret_cast<u32x2_t*>(p));
  else *reinterpret_cast<u32x2_t*>(p) = u32x2_t{q.x, q.y};
}

template <bool BF16, bool PACK, bool ST>
__global__ __launch_bounds__(CKPT_THREADS) void checkpoint_kernel(const CkptArgs a) {
  int64_t rows = a.max_rows;
  if (a.n_rows != nullptr) {
    const int64_t n = *a.n_rows;
    rows = n < rows ? n : rows;
  }
  constexpr int COLS = BF16 ? 8 : 4, WORDS = COLS / 4;               // columns of a piece, words of its codes
  const int64_t first = static_cast<int64_t>(blockIdx.x) * CKPT_THREADS + threadIdx.x;
  int64_t r = first / a.pieces;
  int col = static_cast<int>(first - r * a.pieces);
  while (r < rows) {
    // (the lanes of a block are at the same place: pieces and steps are whole blocks)
    unsigned char* xp[CKPT_TURN];
    unsigned char* qp[CKPT_TURN];
    int cc[CKPT_TURN];
    bool in[CKPT_TURN];
#pragma unroll
    for (int u = 0; u < CKPT_TURN; ++u) {
      cc[u] = col * COLS;
      in[u] = r < rows && cc[u] < a.width;
      xp[u] = a.x + r * a.ldx + col * 16;
      qp[u] = a.q + r * a.ldq;
      r += a.row_step;
      col += a.col_step;
      if (col >= a.pieces) {
        col -= a.pieces;
        ++r;
      }
    }
    if constexpr (PACK) {
      uint4 w[CKPT_TURN];
#pragma unroll
      for (int u = 0; u < CKPT_TURN; ++u) {
        w[u] = make_uint4(0, 0, 0, 0);
        if (in[u]) w[u] = load16<ST>(xp[u]);
      }
#pragma unroll
      for (int u = 0; u < CKPT_TURN; ++u) {
        float v[COLS];
        unpack16<BF16>(w[u], v);
        uint32_t most = 0;
#pragma unroll
        for (int t = 0; t < COLS; ++t) most = max(most, magnitude(v[t]));
        most = max(most, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(most), 0xB1, 0xf, 0xf, true)));   // neighbour
        most = max(most, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(most), 0x4E, 0xf, 0xf, true)));   // pair
        if (!BF16) most = max(most, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(most), 0x141, 0xf, 0xf, true)));   // mirrored 8
        const uint32_t byte = ckpt_scale_byte(most);
        const float inv = ckpt_inverse(byte);
        if (in[u]) {
          const uint32_t codes = ckpt_encode4(v[0], v[1], v[2], v[3], inv);
          if constexpr (BF16) store8<ST>(qp[u] + cc[u], make_uint2(codes, ckpt_encode4(v[COLS - 4], v[COLS - 3], v[COLS - 2], v[COLS - 1], inv)));
          else *reinterpret_cast<uint32_t*>(qp[u] + cc[u]) = codes;
          if ((cc[u] & (CKPT_BLOCK - 1)) == 0) qp[u][a.width + cc[u] / CKPT_BLOCK] = static_cast<unsigned char>(byte);
        }
      }
    } else {
      uint32_t codes[CKPT_TURN][WORDS], byte[CKPT_TURN];
#pragma unroll
      for (int u = 0; u < CKPT_TURN; ++u) {
        byte[u] = 0;
#pragma unroll
        for (int t = 0; t < WORDS; ++t) codes[u][t] = 0;
        if (in[u]) {
          byte[u] = qp[u][a.width + cc[u] / CKPT_BLOCK];
#pragma unroll
          for (int t = 0; t < WORDS; ++t) codes[u][t] = reinterpret_cast<const uint32_t*>(qp[u] + cc[u])[t];
        }
      }
#pragma unroll
      for (int u = 0; u < CKPT_TURN; ++u) {
        float v[COLS];
#pragma unroll
        for (int t = 0; t < WORDS; ++t) ckpt_decode4(codes[u][t], ckpt_scale(byte[u]), v + 4 * t);
        if (in[u]) store16<ST>(xp[u], pack16<BF16>(v));
      }
    }
  }
}

template <bool PACK>
static int launch_checkpoint(CkptArgs a, int dtype, hipStream_t stream) {
  const int cols = 16 / elem_bytes(dtype);
  a.pieces = (a.width + CKPT_BLOCK - 1) / CKPT_BLOCK * (CKPT_BLOCK / cols);
  // Workgroups of one turn each, and where that leaves compute units less than eight of them, of fewer pieces a lane (16384 x 1024: 11.7 us
  // so, 15.7 with a piece a lane; 32768 x 8192, pack: 143 us with two turns, 158 with sixteen).
  const int64_t blocks = (a.max_rows * a.pieces + CKPT_THREADS - 1) / CKPT_THREADS, turns = (blocks + CKPT_TURN - 1) / CKPT_TURN, few = int64_t(num_cus()) * 8;
  int64_t n = turns > few ? turns : blocks < few ? blocks : few;
  if (n > (1 << 23)) n = 1 << 23;                                     // (under 2^32 threads)
  const int64_t step = n * CKPT_THREADS;
  a.row_step = step / a.pieces;
  a.col_step = static_cast<int>(step - a.row_step * a.pieces);
  const dim3 grid(static_cast<unsigned>(n)), block(CKPT_THREADS);
  const bool st = streams_past_caches(a.max_rows * a.width * (elem_bytes(dtype) + 1));
#define SCMOE_CHECKPOINT(BF16, ST) hipLaunchKernelGGL((checkpoint_kernel<BF16, PACK, ST>), grid, block, 0, stream, a)
  if (dtype == SCMOE_BF16) {
    if (st) SCMOE_CHECKPOINT(true, true);
    else SCMOE_CHECKPOINT(true, false);
  } else {
    if (st) SCMOE_CHECKPOINT(false, true);
    else SCMOE_CHECKPOINT(false, false);
  }
#undef SCMOE_CHECKPOINT
  return launch_status();
}

int checkpoint_pack(const void* x, int64_t ldx, int dtype, const int32_t* n_rows, int64_t max_rows, int width, void* q, int64_t ldq, hipStream_t stream) {
  CkptArgs a{};
  a.x = static_cast<unsigned char*>(const_cast<void*>(x)); a.ldx = ldx * elem_bytes(dtype);
  a.q = static_cast<unsigned char*>(q); a.ldq = ldq;
  a.n_rows = n_rows; a.max_rows = max_rows; a.width = width;
  return launch_checkpoint<true>(a, dtype, stream);
}

int checkpoint_unpack(const void* q, int64_t ldq, const int32_t* n_rows, int64_t max_rows, int width, void* x, int64_t ldx, int dtype, hipStream_t stream) {
  CkptArgs a{};
  a.x = static_cast<unsigned char*>(x); a.ldx = ldx * elem_bytes(dtype);
  a.q = static_cast<unsigned char*>(const_cast<void*>(q)); a.ldq = ldq;
  a.n_rows = n_rows; a.max_rows = max_rows; a.width = width;
  return launch_checkpoint<false>(a, dtype, stream);
}

static int check_checkpoint(const void* x, int64_t ldx, int dtype, int32_t max_rows, int32_t width, const void* q, int64_t ldq) {
  if (!dtype_ok(dtype)) return SCMOE_ERR_DTYPE;
  if (max_rows < 0 || width <= 0 || width % 8 != 0 || width > SCMOE_MAX_CHECKPOINT_WIDTH) return SCMOE_ERR_SHAPE;   // (columns and their bytes: 32 bits)
  if (max_rows == 0) return SCMOE_OK;
  if (!x || !q) return SCMOE_ERR_NULL;
  return view_ok(x, ldx, width, dtype) && ckpt_view_ok(q, ldq, width) ? SCMOE_OK : SCMOE_ERR_SHAPE;
}

}  // namespace scmoe

extern "C" int scmoe_checkpoint_ld(int32_t width, int64_t* ld) {
  using namespace scmoe;
  if (!ld) return SCMOE_ERR_NULL;
  if (width <= 0 || width % 8 != 0 || width > SCMOE_MAX_CHECKPOINT_WIDTH) return SCMOE_ERR_SHAPE;
  *ld = (ckpt_bytes(width) + 15) / 16 * 16;
  return SCMOE_OK;
}

extern "C" int scmoe_checkpoint_pack(const void* x, int64_t ldx, int32_t dtype, const int32_t* n_rows, int32_t max_rows, int32_t width,
                                     void* q, int64_t ldq, void* stream) {
  using namespace scmoe;
  const int st = check_checkpoint(x, ldx, dtype, max_rows, width, q, ldq);
  if (st != SCMOE_OK || max_rows == 0) return st;
  return checkpoint_pack(x, ldx, dtype, n_rows, max_rows, width, q, ldq, static_cast<hipStream_t>(stream));
}

extern "C" int scmoe_checkpoint_unpack(const void* q, int64_t ldq, const int32_t* n_rows, int32_t max_rows, int32_t width, void* x,
                                       int64_t ldx, int32_t dtype, void* stream) {
  using namespace scmoe;
  const int st = check_checkpoint(x, ldx, dtype, max_rows, width, q, ldq);
  if (st != SCMOE_OK || max_rows == 0) return st;
  return checkpoint_unpack(q, ldq, n_rows, max_rows, width, x, ldx, dtype, static_cast<hipStream_t>(stream));
}
