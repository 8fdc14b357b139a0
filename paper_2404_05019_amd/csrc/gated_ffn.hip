// The gated feed-forward block over packed expert segments and its gradient: which launches a call makes, and the checks of its arguments.
//
//   forward    GATE (hidden rows, and g and u where they are kept), DOWN
//   backward   DH (gradients of g and u, h again), DW (both weights' gradients in one launch), DX
#include "gated_tiles.hpp"
#include <math.h>

namespace scmoe {

// A row stride with which 32-bit offsets inside a tile (at most 256 rows) stay inside the buffer, and BUFFER_NOWHERE and the offset of a
// wave tile's row (at most 127 rows, of two checkpoint rows each) below 2^32.
constexpr int64_t GATED_MOST_LD = 1 << 18;
static_assert(BUFFER_NOWHERE + 127ull * 2 * GATED_MOST_LD < (1ull << 32) && 256ll * 4 * GATED_MOST_LD < BUFFER_SPAN);
static_assert(BUFFER_NOWHERE + 127ull * 2 * (2 * SCMOE_MAX_GATED_WIDTH + 64) < (1ull << 32));   // (the workspace's padded rows)
static bool gated_view_ok(const void* p, int64_t ld, int64_t cols, int dtype) { return view_ok(p, ld, cols, dtype) && ld <= GATED_MOST_LD; }

// Which calls take the kernel for few rows (gated_few.hip).  A wave of it has one column of a segment's tile.  It streams the column's weights well where
// they are long (4 KB and more), and costs some 0.6 ns of its own, all waves together: more than a row of 512 values.  So it is taken
//  * up to an average of so many rows an expert (bf16: two, in DOWN one, above which the experts' second product does better; fp32, whose matrix instructions
//    have less to gain: five and two), where the columns are long enough for the number of waves;
//  * up to five rows an expert, where the waves are so few that the others' launch takes longer anyhow;
//  * for no more rows than a tile has.
// us of a forward call, random loads, other kernels / few rows in GATE alone / in DOWN alone / in both:
//   bf16  1 row, d = 2048, F = 8192, E = 16 36 / 29 / - / 23;  8 rows 147 / 126 / 143 / 121;  16, E = 32 263 / 237 / 256 / 218;  but 40, E = 8 161 / 191 / 199 / 228
//         5, 512, 2048, 4 17 / 16 / 16 / 16;  but 40, 512, 2048, 8 17 / 30 / 21 / 34;  64, 256, 1024, 64 21 / 36 / 25 / 40;  96, 512, 512, 64 22 / 28 / 37 / 44;
//         64, 1024, 4096, 64 170 / 206 / 170 / 208;  200, 256, 1024, 200 46 / 130 / 67 / 151
//   fp32  5, 1024, 4096, 1 89 / 79 / 31 / 18;  16, 1024, 4096, 8 129 / 111 / 90 / 72;  40, 1024, 4096, 8 138 / 133 / 114 / 110;  20, 256, 1024, 4 31 / 30 / 17 / 17;
//         64, 2048, 2048, 32 323 / 273 / 304 / 252;  but 80, 2048, 8192, 16 733 / 820 / 831 / 924;  320, 256, 1024, 64 64 / 100 / 74 / 110
// Of 770 such calls the choice is 0.8 % above the best of the four in the mean, 25 % at most (by the average alone 11 %, and up to three and a half times as
// long).  Where a load is skewed, a segment has many tiles of four rows, each of which reads its weights, if from the caches: all rows at one expert of 16,
// bf16, d = 2048, F = 8192, 16 rows 79 us where the others take 35, 32 rows 104 where they take 35.  A random load of as many takes 160 to 260.
// Beyond 256 experts, four times what the gate has, the average alone decides, as tests/test_gated_abi.py has it for 600 (1100 rows, d = 64, F = 2048 1430 us, by
// the other kernels 304).
static bool few_rows(int mode, int dtype, int64_t rows, int E, int N, int Kd) {
  if (rows > 4096) return false;                         // (tiles of rows are the grid's y)
  const bool f32 = dtype == SCMOE_F32, gate = mode == G_GATE;
  if (rows <= 4) return true;
  if (E > 256) return rows <= (f32 ? 5 : gate ? 2 : 1) * static_cast<int64_t>(E);
  // segments that have rows, of rows that are spread at random
  const double bytes = static_cast<double>(Kd) * elem_bytes(dtype), occupied = E * (1.0 - pow(1.0 - 1.0 / E, static_cast<double>(rows)));
  const double waves = (occupied > rows / 3.0 ? occupied : rows / 3.0) * N;
  if (!f32 && gate) return (rows <= 2 * E && (bytes >= 4000.0 || waves <= 12.0 * bytes)) || (rows <= 5 * E && waves <= 8000.0);
  if (!f32) return (rows <= E && waves <= 2.0 * bytes) || (rows <= 5 * E && waves <= 4000.0);
  if (gate) return rows <= 5 * E && (bytes >= 4000.0 || waves <= 24.0 * bytes);
  return (rows <= 2 * E && (bytes >= 8000.0 || waves <= 12.0 * bytes)) || (rows <= 5 * E && waves <= 16000.0);
}

static bool takes_few(const GatedArgs& a, int mode, int keep, int dtype, int64_t rows) {
  return ((mode == G_GATE && keep != KEEP_8BIT) || mode == G_DOWN) && few_rows(mode, dtype, rows, a.E, a.j[0].N, a.j[0].Kd);
}

static int launch_gated(const GatedArgs& a, int mode, int keep, int64_t max_rows, int dtype, hipStream_t stream) {
  if (takes_few(a, mode, keep, dtype, max_rows)) return launch_gated_few(a, mode, keep, max_rows, dtype, stream);
  return dtype == SCMOE_BF16 ? launch_gated_bf16(a, mode, keep, max_rows, stream) : launch_gated_f32(a, mode, keep, max_rows, stream);
}

static GatedJob gated_job(const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, int M, int N, int Kd) {
  GatedJob j{};
  j.A = static_cast<const unsigned char*>(A); j.lda = lda;
  j.B = static_cast<const unsigned char*>(B); j.ldb = ldb;
  j.C = static_cast<unsigned char*>(C); j.ldc = ldc;
  j.M = M; j.N = N; j.Kd = Kd;
  return j;
}

// Sizes, options and weights that both calls take.
static int check_gated(int dtype, int32_t max_rows, int32_t E, int32_t d, int32_t F, int32_t act) {
  if (!dtype_ok(dtype)) return SCMOE_ERR_DTYPE;
  if (max_rows < 0 || E < 1 || d <= 0 || F <= 0 || d % 8 != 0 || F % 8 != 0 || d > SCMOE_MAX_GATED_WIDTH || F > SCMOE_MAX_GATED_WIDTH) return SCMOE_ERR_SHAPE;
  // rows and tiles are counted in 32 bits (tiles of 128 x 64 at the least: the products' outputs have 2 F, F and d columns)
  const int64_t wide = (2 * static_cast<int64_t>(F) > d ? 2 * static_cast<int64_t>(F) : d) / 64 + 1;
  if (max_rows > SCMOE_MAX_GATED_ROWS || (max_rows / 128 + static_cast<int64_t>(E)) * wide > (1 << 30)) return SCMOE_ERR_SHAPE;
  if (static_cast<int64_t>(E) * (2 * static_cast<int64_t>(F) / 128 + 1) * (d / 64 + 1) + static_cast<int64_t>(E) * (d / 128 + 1) * (F / 64 + 1) > (1 << 30)) return SCMOE_ERR_SHAPE;
  if (act != SCMOE_GELU_ERF && act != SCMOE_GELU_TANH && act != SCMOE_SILU) return SCMOE_ERR_ARG;
  return SCMOE_OK;
}
// An expert's rows of a weight matrix lie inside one buffer.
static bool gated_weights_ok(const void* W, int64_t ld, int64_t rows, int64_t cols, int dtype) {
  return gated_view_ok(W, ld, cols, dtype) && rows * ld * elem_bytes(dtype) < BUFFER_SPAN;
}
static bool kept_ok(const void* p, int64_t ld, int64_t width, int keep, int dtype) {
  return keep == SCMOE_KEEP_8BIT ? ckpt_view_ok(p, ld, width) && ld <= GATED_MOST_LD : gated_view_ok(p, ld, width, dtype);
}

// Where y = W2 h is the second product of the experts without a gate (ffn_mfma.hip, ffn_direct.hip): in bf16, where its tiled kernel takes
// the widths, and for up to 16 rows an expert, when its other kernel streams the weights; else this block's own.  us of a forward call,
// so / with DOWN: 16384 rows, d = 1024, F = 4096, E = 8 372 / 394; 30 rows, d = 1000, F = 2728 45 / 52; but 500 rows 73 / 64, 5003 rows, E = 32
// 272 / 208.  In fp32 DOWN does better from 40 rows on (d = 1024, F = 4096, E = 8 148 / 161; 4096 rows, F = 2048 381 / 417).
static bool second_is_the_experts(int dtype, int64_t rows, int E, int d, int F) {
  if (dtype == SCMOE_F32 || few_rows(G_DOWN, dtype, rows, E, d, F)) return false;
  return ffn_mfma_supported(d, F) || rows <= 64 || (rows <= 16 * static_cast<int64_t>(E) && rows <= 1024);
}

struct GatedWs { int64_t ldp, ldh; size_t dpre, hidden, x, total; };
static GatedWs gated_ws(int dtype, int64_t rows, int d, int F) {
  GatedWs w;
  const int64_t eb = elem_bytes(dtype);
  auto up = [](int64_t n) { return static_cast<size_t>((n + 255) / 256 * 256); };
  w.ldp = padded_ld(2 * static_cast<int64_t>(F), dtype);
  w.ldh = padded_ld(F, dtype);
  w.dpre = 0;
  w.hidden = w.dpre + up(rows * w.ldp * eb);
  w.x = w.hidden + up(rows * w.ldh * eb);
  w.total = w.x + up(rows * d * eb);
  return w;
}

}  // namespace scmoe

extern "C" int scmoe_gated_ffn_workspace_bytes(int32_t dtype, int32_t d, int32_t F, size_t* out) {
  using namespace scmoe;
  if (!out) return SCMOE_ERR_NULL;
  const int st = check_gated(dtype, 0, 1, d, F, SCMOE_SILU);
  if (st == SCMOE_OK) *out = dtype == SCMOE_BF16 && ffn_mfma_supported(d, F) ? ffn_mfma_scratch_bytes() : 0;
  return st;
}

extern "C" int scmoe_gated_ffn(const void* x_perm, int64_t ld_perm, int32_t dtype, const int32_t* offsets, int32_t max_rows, int32_t E,
                               int32_t d, int32_t F, const void* W1, int64_t ldw1, const void* W2, int64_t ldw2, int32_t act, void* hidden,
                               int64_t ldh, void* pre, int64_t ldpre, int32_t pre_keep, void* y_perm, int64_t ldy, void* workspace,
                               size_t ws_bytes, void* stream) {
  using namespace scmoe;
  int st = check_gated(dtype, max_rows, E, d, F, act);
  if (st != SCMOE_OK) return st;
  if (pre_keep != SCMOE_KEEP_NOTHING && pre_keep != SCMOE_KEEP_FULL && pre_keep != SCMOE_KEEP_8BIT) return SCMOE_ERR_ARG;
  if (max_rows == 0) return SCMOE_OK;
  if (!x_perm || !offsets || !W1 || !W2 || !hidden || !y_perm || (pre_keep != SCMOE_KEEP_NOTHING && !pre)) return SCMOE_ERR_NULL;
  if (!gated_view_ok(x_perm, ld_perm, d, dtype) || !gated_view_ok(y_perm, ldy, d, dtype) || !gated_view_ok(hidden, ldh, F, dtype) ||
      !gated_weights_ok(W1, ldw1, 2 * static_cast<int64_t>(F), d, dtype) || !gated_weights_ok(W2, ldw2, d, F, dtype) || !aligned16(workspace))
    return SCMOE_ERR_SHAPE;
  if (pre_keep != SCMOE_KEEP_NOTHING && !kept_ok(pre, ldpre, pre_keep == SCMOE_KEEP_8BIT ? F : 2 * static_cast<int64_t>(F), pre_keep, dtype)) return SCMOE_ERR_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  GatedArgs a{};
  a.offsets = offsets; a.E = E; a.act = act;
  a.pre = static_cast<unsigned char*>(pre); a.ldpre = ldpre;
  a.j[0] = gated_job(x_perm, ld_perm, W1, ldw1, hidden, ldh, 0, F, d);
  const bool experts = second_is_the_experts(dtype, max_rows, E, d, F);
  if (experts && workspace != nullptr && ws_bytes >= ffn_mfma_scratch_bytes() && !takes_few(a, G_GATE, pre_keep, dtype, max_rows)) {
    a.zero = static_cast<int*>(workspace);                  // (the counters of tiles that the second product cuts along K; the kernel for few rows clears none)
    a.zeros = ffn_mfma_counter_ints();
  }
  st = launch_gated(a, G_GATE, pre_keep, max_rows, dtype, s);
  if (st != SCMOE_OK) return st;
  if (experts) {
    FfnArgs f{};
    f.offsets = offsets; f.max_rows = max_rows; f.E = E; f.d = d; f.F = F;
    f.W2 = W2; f.ldw2 = ldw2; f.hidden = hidden; f.ldh = ldh; f.y = y_perm; f.ldy = ldy;
    f.scratch = workspace; f.scratch_bytes = ws_bytes; f.scratch_zeroed = a.zero != nullptr;
    return ffn_second(f, dtype, s);
  }
  a.j[0] = gated_job(hidden, ldh, W2, ldw2, y_perm, ldy, 0, d, F);
  return launch_gated(a, G_DOWN, KEEP_NONE, max_rows, dtype, s);
}

extern "C" int scmoe_gated_ffn_backward_workspace_bytes(int32_t dtype, int32_t max_rows, int32_t E, int32_t d, int32_t F, size_t* out) {
  using namespace scmoe;
  if (!out) return SCMOE_ERR_NULL;
  const int st = check_gated(dtype, max_rows, E, d, F, SCMOE_SILU);
  if (st == SCMOE_OK) *out = gated_ws(dtype, max_rows, d, F).total;
  return st;
}

extern "C" int scmoe_gated_ffn_backward(const void* dy_perm, int64_t lddy, int32_t dtype, const void* x, int64_t ldx, int32_t x_keep,
                                        const void* pre, int64_t ldpre, int32_t pre_keep, const int32_t* offsets, int32_t max_rows, int32_t E,
                                        int32_t d, int32_t F, const void* W1, int64_t ldw1, const void* W2, int64_t ldw2, int32_t act,
                                        void* dx_perm, int64_t lddx, void* dW1, void* dW2, void* workspace, size_t ws_bytes, void* stream) {
  using namespace scmoe;
  int st = check_gated(dtype, max_rows, E, d, F, act);
  if (st != SCMOE_OK) return st;
  const auto kind = [](int keep) { return keep == SCMOE_KEEP_FULL || keep == SCMOE_KEEP_8BIT; };
  if (!kind(pre_keep) || (dW1 && !kind(x_keep))) return SCMOE_ERR_ARG;
  if (!dx_perm && !dW1 && !dW2) return SCMOE_ERR_NULL;
  if (max_rows == 0 && !dW1 && !dW2) return SCMOE_OK;
  if (!offsets || (dW1 && !aligned16(dW1)) || (dW2 && !aligned16(dW2))) return offsets ? SCMOE_ERR_SHAPE : SCMOE_ERR_NULL;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  GatedArgs a{};
  a.offsets = offsets; a.E = E; a.act = act;
  const GatedWs w = gated_ws(dtype, max_rows, d, F);
  if (max_rows > 0) {
    if (!dy_perm || !pre || !W2 || !workspace || (dW1 && !x) || (dx_perm && !W1)) return SCMOE_ERR_NULL;
    if (!gated_view_ok(dy_perm, lddy, d, dtype) || !kept_ok(pre, ldpre, pre_keep == SCMOE_KEEP_8BIT ? F : 2 * static_cast<int64_t>(F), pre_keep, dtype) ||
        (dW1 && !kept_ok(x, ldx, d, x_keep, dtype)) || !gated_weights_ok(W2, ldw2, d, F, dtype) ||
        (dx_perm && (!gated_weights_ok(W1, ldw1, 2 * static_cast<int64_t>(F), d, dtype) || !gated_view_ok(dx_perm, lddx, d, dtype))) || !aligned16(workspace))
      return SCMOE_ERR_SHAPE;
    if (ws_bytes < w.total) return SCMOE_ERR_WORKSPACE;
  }
  unsigned char* const ws = static_cast<unsigned char*>(workspace);
  unsigned char* const dpre = ws + w.dpre;
  unsigned char* const hid = ws + w.hidden;
  if (max_rows > 0) {
    a.pre = static_cast<unsigned char*>(const_cast<void*>(pre)); a.ldpre = ldpre;
    a.dpre = dpre; a.lddpre = w.ldp;
    a.j[0] = gated_job(dy_perm, lddy, W2, ldw2, hid, w.ldh, 0, F, d);
    st = launch_gated(a, G_DH, pre_keep, max_rows, dtype, s);
    if (st != SCMOE_OK) return st;
    if (dW1 && x_keep == SCMOE_KEEP_8BIT) {
      st = checkpoint_unpack(x, ldx, offsets + E, max_rows, d, ws + w.x, d, dtype, s);
      if (st != SCMOE_OK) return st;
      x = ws + w.x;
      ldx = d;
    }
  }
  GatedArgs b = a;
  if (dW1 || dW2) {
    int n = 0;
    if (dW1) a.j[n++] = gated_job(dpre, w.ldp, x, ldx, dW1, d, 2 * F, d, 0);
    if (dW2) a.j[n++] = gated_job(dy_perm, lddy, hid, w.ldh, dW2, F, d, F, 0);
    if (!dx_perm || max_rows == 0) return launch_gated(a, G_DW, KEEP_NONE, max_rows, dtype, s);
  }
  b.j[0] = gated_job(dpre, w.ldp, W1, ldw1, dx_perm, lddx, 0, d, 2 * F);
  if (!dW1 && !dW2) return launch_gated(b, G_DX, KEEP_NONE, max_rows, dtype, s);
  // dx may take the place of dy or of x, which dW1 and dW2 are made of: then it is made after them.
  if (dx_perm == dy_perm || dx_perm == x) {
    st = launch_gated(a, G_DW, KEEP_NONE, max_rows, dtype, s);
    return st == SCMOE_OK ? launch_gated(b, G_DX, KEEP_NONE, max_rows, dtype, s) : st;
  }
  return dtype == SCMOE_BF16 ? launch_gated_gradients_bf16(b, a, max_rows, s) : launch_gated_gradients_f32(b, a, max_rows, s);
}
