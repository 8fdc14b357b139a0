// The gated feed-forward block over packed expert segments and its gradient: which launches a call makes, and the checks of its arguments.
//
//   forward    GATE (hidden rows, and g and u where they are kept), DOWN
//   backward   DH (gradients of g and u, h again), DW (both weights' gradients in one launch), DX
#include "gated_tiles.hpp"

namespace scmoe {

// A row stride with which 32-bit offsets inside a tile (at most 256 rows) stay inside the buffer, and BUFFER_NOWHERE and the offset of a
// wave tile's row (at most 127 rows, of two checkpoint rows each) below 2^32.
constexpr int64_t GATED_MOST_LD = 1 << 18;
static_assert(BUFFER_NOWHERE + 127ull * 2 * GATED_MOST_LD < (1ull << 32) && 256ll * 4 * GATED_MOST_LD < BUFFER_SPAN);
static_assert(BUFFER_NOWHERE + 127ull * 2 * (2 * SCMOE_MAX_GATED_WIDTH + 64) < (1ull << 32));   // (the workspace's padded rows)
static bool gated_view_ok(const void* p, int64_t ld, int64_t cols, int dtype) { return view_ok(p, ld, cols, dtype) && ld <= GATED_MOST_LD; }

// Which calls take the kernel for few rows (gated_few.hip): where experts average at most two rows (DOWN: one, above which the experts'
// second product does better), or there are no more than it takes at a time; in fp32, whose matrix instructions have less to gain, five.
// us of a forward call, other kernels / few rows in GATE alone / in both:
//   bf16, d = 2048, F = 8192, E = 16    1 row 36.1 / 28.8 / 22.7, 8 rows 160 / 139 / 138, 16 rows 202 / 182 / 178, 32 rows 298 / 259 / 267, 64 rows 312 / 330 / 385
//   bf16, 4 rows of one expert 34.4 / 30.9 / 25.9, 16 rows 36.5 / 60.7 / 68.5;   30 rows, d = 1000, F = 2728, E = 8 39.8 / 44.4 / 48.1
//   fp32, d = 1024, F = 4096, E = 8     1 row 35.0 / 21.6 / 16.8, 16 rows 123 / 107 / 64, 40 rows 138 / 130 / 106;   64 rows, d = 64, F = 256, E = 4 17.5 / 17.9 / 16.8
static bool few_rows(int mode, int dtype, int64_t rows, int E) {
  if (rows > 4096) return false;                         // (tiles of rows are the grid's y)
  const int64_t per = dtype == SCMOE_F32 ? 5 : mode == G_GATE ? 2 : 1;
  return rows <= 4 || rows <= per * E;
}

static bool takes_few(int mode, int keep, int dtype, int64_t rows, int E) {
  return ((mode == G_GATE && keep != KEEP_8BIT) || mode == G_DOWN) && few_rows(mode, dtype, rows, E);
}

static int launch_gated(const GatedArgs& a, int mode, int keep, int64_t max_rows, int dtype, hipStream_t stream) {
  if (takes_few(mode, keep, dtype, max_rows, a.E)) return launch_gated_few(a, mode, keep, max_rows, dtype, stream);
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
  if (dtype == SCMOE_F32 || few_rows(G_DOWN, dtype, rows, E)) return false;
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
  if (experts && workspace != nullptr && ws_bytes >= ffn_mfma_scratch_bytes() && !takes_few(G_GATE, pre_keep, dtype, max_rows, E)) {
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
