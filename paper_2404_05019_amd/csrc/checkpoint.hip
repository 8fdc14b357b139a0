// Activation checkpoints in 8 bits (checkpoint.hpp): rows packed and restored.
//
// Bound by HBM: a value is read and a little over a byte written, or the other way round.  A lane has 8 columns, four lanes a block,
// whose largest magnitude they find by two permutes inside the quad; a workgroup walks over the pieces of as many rows as there are.
#include "checkpoint.hpp"
#include "rows.hpp"

namespace scmoe {

struct CkptArgs {
  unsigned char* x; int64_t ldx;          // strides in bytes
  unsigned char* q; int64_t ldq;
  const int32_t* n_rows; int64_t max_rows;
  int width, pieces;                      // pieces of 8 columns, a whole number of blocks
};

constexpr int CKPT_THREADS = 256;

template <bool BF16, bool PACK>
__global__ __launch_bounds__(CKPT_THREADS) void checkpoint_kernel(const CkptArgs a) {
  int64_t rows = a.max_rows;
  if (a.n_rows != nullptr) {
    const int64_t n = *a.n_rows;
    rows = n < rows ? n : rows;
  }
  constexpr int EB = BF16 ? 2 : 4, NV = BF16 ? 1 : 2;                // 16-byte vectors of a piece
  const int64_t total = rows * a.pieces, step = static_cast<int64_t>(gridDim.x) * CKPT_THREADS;
  // (whole quads: total and step are multiples of four)
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * CKPT_THREADS + threadIdx.x; i < total; i += step) {
    const int64_t r = i / a.pieces;
    const int c = static_cast<int>(i - r * a.pieces) * 8;
    const bool in = c < a.width;
    unsigned char* const xp = a.x + r * a.ldx + static_cast<int64_t>(c) * EB;
    unsigned char* const qp = a.q + r * a.ldq;
    float v[8];
    if constexpr (PACK) {
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (in) w = *reinterpret_cast<const uint4*>(xp + t * 16);
        unpack16<BF16>(w, v + t * (8 / NV));
      }
      uint32_t most = 0;
#pragma unroll
      for (int t = 0; t < 8; ++t) most = max(most, magnitude(v[t]));
      most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 1)));
      most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 2)));
      const uint32_t byte = ckpt_scale_byte(most);
      const float inv = ckpt_inverse(byte);
      if (in) {
        *reinterpret_cast<uint2*>(qp + c) = make_uint2(ckpt_encode4(v[0], v[1], v[2], v[3], inv), ckpt_encode4(v[4], v[5], v[6], v[7], inv));
        if ((c & (CKPT_BLOCK - 1)) == 0) qp[a.width + c / CKPT_BLOCK] = static_cast<unsigned char>(byte);
      }
    } else if (in) {
      const uint2 w = *reinterpret_cast<const uint2*>(qp + c);
      const float s = ckpt_scale(qp[a.width + c / CKPT_BLOCK]);
      ckpt_decode4(w.x, s, v);
      ckpt_decode4(w.y, s, v + 4);
#pragma unroll
      for (int t = 0; t < NV; ++t) *reinterpret_cast<uint4*>(xp + t * 16) = pack16<BF16>(v + t * (8 / NV));
    }
  }
}

template <bool PACK>
static int launch_checkpoint(CkptArgs a, int dtype, hipStream_t stream) {
  a.pieces = (a.width + CKPT_BLOCK - 1) / CKPT_BLOCK * (CKPT_BLOCK / 8);
  const int64_t blocks = (a.max_rows * a.pieces + CKPT_THREADS - 1) / CKPT_THREADS, most = int64_t(num_cus()) * 32;
  const dim3 grid(static_cast<unsigned>(blocks < most ? blocks : most)), block(CKPT_THREADS);
  if (dtype == SCMOE_BF16) hipLaunchKernelGGL((checkpoint_kernel<true, PACK>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((checkpoint_kernel<false, PACK>), grid, block, 0, stream, a);
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
  if (max_rows < 0 || width <= 0 || width % 8 != 0) return SCMOE_ERR_SHAPE;
  if (max_rows == 0) return SCMOE_OK;
  if (!x || !q) return SCMOE_ERR_NULL;
  return view_ok(x, ldx, width, dtype) && ckpt_view_ok(q, ldq, width) ? SCMOE_OK : SCMOE_ERR_SHAPE;
}

}  // namespace scmoe

extern "C" int scmoe_checkpoint_ld(int32_t width, int64_t* ld) {
  using namespace scmoe;
  if (!ld) return SCMOE_ERR_NULL;
  if (width <= 0 || width % 8 != 0) return SCMOE_ERR_SHAPE;
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
