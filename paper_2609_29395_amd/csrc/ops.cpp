// C entries of the operators on caller-owned tensors: argument checks, then
// one launcher call each.
#include <cmath>
#include <new>

#include "ops.h"
#include "runtime.h"

namespace {

// gcpsl_fail for entries that must not throw: the message is dropped if there
// is no memory for it.
int fail(int code, const char *msg) noexcept {
  try {
    return gcpsl_fail(code, msg);
  } catch (const std::bad_alloc &) {
    return code;
  }
}

int launched(hipError_t e) noexcept {
  if (e == hipSuccess) return GCPSL_OK;
  if (e == hipErrorInvalidConfiguration) return fail(GCPSL_EUNSUPPORTED, "too many tiles for one launch");
  try {
    return gcpsl_fail(GCPSL_EHIP, std::string("launch failed: ") + hipGetErrorString(e));
  } catch (const std::bad_alloc &) {
    return GCPSL_EHIP;
  }
}

constexpr int64_t kMaxRows = INT32_MAX, kMaxLd = INT32_MAX, kMaxStride = (int64_t)1 << 40;
// Grouped rows: a row of the last tile (256 rows at most), or a group's rows and
// the pieces that they are cut into (513 at most), stay below 2^31 in sum.
constexpr int64_t kMaxGroupRows = ((int64_t)1 << 31) - 1024;
constexpr int kMaxGroups = 1024, kMaxCols = 1 << 28;  // column counters and their tile sums stay below 2^31

bool is_type(int dtype) { return dtype == GCPSL_F32 || dtype == GCPSL_BF16; }
size_t elem_bytes(int dtype) { return dtype == GCPSL_F32 ? 4 : 2; }
bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A [rows][cols] tensor of row stride ld; an input's rows may overlap.
const char *bad_tensor(const void *p, size_t elem, int64_t rows, int64_t cols, int64_t ld, bool out) {
  if (rows > 0 && !p) return "null tensor";
  if (!aligned(p, elem)) return "tensor not aligned to its elements";
  if (ld < 0 || ld > kMaxLd) return "row stride out of range";
  if (out && rows > 1 && ld < cols) return "rows of an output overlap";
  return nullptr;
}

bool drop_of(double p, uint64_t seed, Drop &d) {
  const double t = std::nearbyint(65536.0 * p);
  if (!(p >= 0.0) || !(t <= 65535.0)) return false;
  d.key = gc_mix64(seed + GCPSL_TAG_DROP);
  d.thr = (uint32_t)t;
  d.scale = (float)(65536.0 / (65536.0 - t));
  return true;
}

const char *bad_groups(int dtype, int G, int64_t rows, int n, int k, const int32_t *offsets) {
  if (!is_type(dtype)) return "unknown dtype";
  if (G < 1 || G > kMaxGroups) return "groups must lie in [1, 1024]";
  if (rows < 0 || rows > kMaxRows) return "rows must lie in [0, 2^31)";
  if (n < 1 || k < 1 || n > kMaxCols || k > kMaxCols) return "n and k must lie in [1, 2^28]";
  if (!offsets || !aligned(offsets, 4)) return "offsets null or misaligned";
  return nullptr;
}

const char *bad_stride(int64_t s) { return s < 0 || s > kMaxStride ? "group stride out of range" : nullptr; }

#define CHECK(expr)                                          \
  do {                                                       \
    if (const char *why_ = (expr)) return fail(GCPSL_EINVAL, why_); \
  } while (0)

#define CHECK_GROUPS(...)                                                                            \
  do {                                                                                               \
    CHECK(bad_groups(__VA_ARGS__));                                                                  \
    if (rows > kMaxGroupRows) return fail(GCPSL_EUNSUPPORTED, "more than 2^31 - 1024 grouped rows"); \
  } while (0)

}  // namespace

extern "C" int gcpsl_group_forward(int32_t dtype, int32_t G, int64_t rows, int32_t n, int32_t k,
                                   const int32_t *offsets, const void *x, int64_t ldx, const void *w, int64_t w_gs,
                                   const float *bias, int64_t bias_gs, int32_t relu, double p, uint64_t seed, void *y,
                                   int64_t ldy, void *stream) {
  gcpsl_clear_error();
  CHECK_GROUPS(dtype, G, rows, n, k, offsets);
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(x, e, rows, k, ldx, false));
  CHECK(bad_tensor(w, e, G, k, k, false));
  CHECK(bad_stride(w_gs));
  CHECK(bad_stride(bias_gs));
  if (!aligned(bias, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  CHECK(bad_tensor(y, e, rows, n, ldy, true));
  GroupArgs a{};
  if (!drop_of(p, seed, a.drop)) return fail(GCPSL_EINVAL, "p must lie in [0, 65535/65536]");
  if (rows == 0) return GCPSL_OK;
  a.off = offsets;
  a.G = G; a.M = (int)rows; a.N = n; a.Q = k;
  a.a = x; a.lda = ldx;
  a.b = w; a.ldb = k; a.b_gs = w_gs;
  a.out = y; a.ldo = ldy;
  a.bias = bias; a.bias_gs = bias_gs;
  a.relu = relu != 0;
  return launched(launch_group(dtype, GROUP_FWD, a, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" int gcpsl_group_input_grad(int32_t dtype, int32_t G, int64_t rows, int32_t n, int32_t k,
                                      const int32_t *offsets, const void *dy, int64_t lddy, const void *w,
                                      int64_t w_gs, const void *gate, int64_t ldgate, double p, void *dx, int64_t lddx,
                                      void *stream) {
  gcpsl_clear_error();
  CHECK_GROUPS(dtype, G, rows, n, k, offsets);
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(dy, e, rows, n, lddy, false));
  CHECK(bad_tensor(w, e, G, k, k, false));
  CHECK(bad_stride(w_gs));
  CHECK(bad_tensor(dx, e, rows, k, lddx, true));
  GroupArgs a{};
  if (!drop_of(p, 0, a.drop)) return fail(GCPSL_EINVAL, "p must lie in [0, 65535/65536]");
  if (gate) CHECK(bad_tensor(gate, e, rows, k, ldgate, false));
  else if (a.drop.thr) return fail(GCPSL_EINVAL, "p without a gate");
  if (rows == 0) return GCPSL_OK;
  a.off = offsets;
  a.G = G; a.M = (int)rows; a.N = k; a.Q = n;
  a.a = dy; a.lda = lddy;
  a.b = w; a.ldb = k; a.b_gs = w_gs;
  a.out = dx; a.ldo = lddx;
  a.gate = gate; a.ldg = ldgate;
  return launched(launch_group(dtype, GROUP_DX, a, reinterpret_cast<hipStream_t>(stream)));
}

namespace {
const char *bad_act(int act) { return act < GCPSL_SILU || act > GCPSL_RELU ? "unknown activation" : nullptr; }
// Pairs have twice the columns.
const char *bad_pairs(int n) { return n > kMaxCols / 2 ? "n must lie in [1, 2^27]" : nullptr; }
}  // namespace

extern "C" int gcpsl_group_gated_forward(int32_t dtype, int32_t G, int64_t rows, int32_t n, int32_t k,
                                         const int32_t *offsets, const void *x, int64_t ldx, const void *w,
                                         int64_t w_gs, const float *bias, int64_t bias_gs, int32_t act, void *y,
                                         int64_t ldy, void *pre, int64_t ldpre, void *stream) {
  gcpsl_clear_error();
  CHECK_GROUPS(dtype, G, rows, n, k, offsets);
  CHECK(bad_pairs(n));
  CHECK(bad_act(act));
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(x, e, rows, k, ldx, false));
  CHECK(bad_tensor(w, e, G, k, k, false));
  CHECK(bad_stride(w_gs));
  CHECK(bad_stride(bias_gs));
  if (!aligned(bias, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  CHECK(bad_tensor(y, e, rows, n, ldy, true));
  if (pre) CHECK(bad_tensor(pre, e, rows, 2 * (int64_t)n, ldpre, true));
  if (rows == 0) return GCPSL_OK;
  GroupArgs a{};
  a.off = offsets;
  a.G = G; a.M = (int)rows; a.N = n; a.Q = k;
  a.a = x; a.lda = ldx;
  a.b = w; a.ldb = k; a.b_gs = w_gs;
  a.out = y; a.ldo = ldy;
  a.bias = bias; a.bias_gs = bias_gs;
  a.act = act;
  a.pre = pre; a.ldp = ldpre;
  return launched(launch_group(dtype, GROUP_GATED, a, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" int gcpsl_group_gated_grad(int32_t dtype, int32_t G, int64_t rows, int32_t m, int32_t n,
                                      const int32_t *offsets, const void *dz, int64_t lddz, const void *v,
                                      int64_t v_gs, int32_t act, const void *pre, int64_t ldpre, void *dpre,
                                      int64_t lddpre, void *stream) {
  gcpsl_clear_error();
  CHECK_GROUPS(dtype, G, rows, m, n, offsets);
  CHECK(bad_pairs(n));
  CHECK(bad_act(act));
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(dz, e, rows, m, lddz, false));
  CHECK(bad_tensor(v, e, G, n, n, false));
  CHECK(bad_stride(v_gs));
  CHECK(bad_tensor(pre, e, rows, 2 * (int64_t)n, ldpre, false));
  CHECK(bad_tensor(dpre, e, rows, 2 * (int64_t)n, lddpre, true));
  if (rows == 0) return GCPSL_OK;
  GroupArgs a{};
  a.off = offsets;
  a.G = G; a.M = (int)rows; a.N = n; a.Q = m;
  a.a = dz; a.lda = lddz;
  a.b = v; a.ldb = n; a.b_gs = v_gs;
  a.out = dpre; a.ldo = lddpre;
  a.act = act;
  a.pre = const_cast<void *>(pre); a.ldp = ldpre;
  return launched(launch_group(dtype, GROUP_GATED_GRAD, a, reinterpret_cast<hipStream_t>(stream)));
}

namespace {
// Partials of a weight gradient: the weights' and then the biases'.
size_t partial_bytes(const GroupPieces &p, int n, int k) { return sizeof(float) * (size_t)p.slots * n * ((size_t)k + 1); }
}  // namespace

extern "C" int gcpsl_group_workspace_bytes(int32_t dtype, int32_t G, int64_t rows, int32_t n, int32_t k,
                                           size_t *bytes) {
  gcpsl_clear_error();
  if (!bytes) return fail(GCPSL_EINVAL, "null output");
  alignas(4) static const int32_t none = 0;
  CHECK_GROUPS(dtype, G, rows, n, k, &none);
  *bytes = partial_bytes(group_pieces(dtype, G, rows, n, k), n, k);
  return GCPSL_OK;
}

extern "C" int gcpsl_group_weight_grad(int32_t dtype, int32_t G, int64_t rows, int32_t n, int32_t k,
                                       const int32_t *offsets, const void *dy, int64_t lddy, const void *x,
                                       int64_t ldx, float *dw, int64_t dw_gs, float *db, int64_t db_gs,
                                       void *workspace, size_t workspace_bytes, void *stream) {
  gcpsl_clear_error();
  CHECK_GROUPS(dtype, G, rows, n, k, offsets);
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(dy, e, rows, n, lddy, false));
  CHECK(bad_tensor(x, e, rows, k, ldx, false));
  if (!dw || !aligned(dw, 4) || !aligned(db, 4)) return fail(GCPSL_EINVAL, "null or misaligned gradient");
  CHECK(bad_stride(dw_gs));
  CHECK(bad_stride(db_gs));
  if (G > 1 && (dw_gs < (int64_t)n * k || (db && db_gs < n))) return fail(GCPSL_EINVAL, "groups of an output overlap");
  GroupArgs a{};
  const GroupPieces pieces = group_pieces(dtype, G, rows, n, k);
  if (partial_bytes(pieces, n, k) > workspace_bytes) return fail(GCPSL_EINVAL, "workspace too small");
  if (pieces.slots && (!workspace || !aligned(workspace, 16)))
    return fail(GCPSL_EINVAL, "workspace null or not 16-byte aligned");
  a.piece = pieces.piece;
  a.slots = pieces.slots;
  a.off = offsets;
  a.G = G; a.M = n; a.N = k; a.Q = (int)rows;
  a.a = dy; a.lda = lddy;
  a.b = x; a.ldb = ldx;
  a.out = dw; a.ldo = k; a.out_gs = dw_gs;
  a.db = db; a.db_gs = db_gs;
  a.part = (float *)workspace;
  a.part_db = a.part ? a.part + (size_t)a.slots * n * k : nullptr;
  return launched(launch_group(dtype, GROUP_DW, a, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" int gcpsl_dropout(int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, double p,
                             uint64_t seed, void *y, int64_t ldy, void *stream) {
  gcpsl_clear_error();
  if (!is_type(dtype)) return fail(GCPSL_EINVAL, "unknown dtype");
  if (rows < 0 || rows > kMaxRows || cols < 0 || cols > kMaxCols) return fail(GCPSL_EINVAL, "rows or cols out of range");
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(x, e, cols ? rows : 0, cols, ldx, false));
  CHECK(bad_tensor(y, e, cols ? rows : 0, cols, ldy, true));
  if (x && x == y && rows > 1 && ldx != ldy) return fail(GCPSL_EINVAL, "in place needs equal row strides");
  Drop d;
  if (!drop_of(p, seed, d)) return fail(GCPSL_EINVAL, "p must lie in [0, 65535/65536]");
  if (rows == 0 || cols == 0) return GCPSL_OK;
  return launched(launch_dropout(dtype, rows, cols, x, ldx, y, ldy, d, reinterpret_cast<hipStream_t>(stream)));
}

namespace {
const char *bad_rows(int dtype, int64_t rows, int L) {
  if (!is_type(dtype)) return "unknown dtype";
  if (rows < 0 || rows > kMaxRows) return "rows must lie in [0, 2^31)";
  return L < 1 || L > kMaxCols ? "L must lie in [1, 2^28]" : nullptr;
}
const char *bad_top(int top, int L) {
  return top < 0 || top > kMaxTop || top > L ? "top must lie in [0, min(L, 32)]" : nullptr;
}
}  // namespace

extern "C" int gcpsl_score_workspace_bytes(int32_t dtype, int64_t rows, int32_t L, int32_t top, size_t *bytes) {
  gcpsl_clear_error();
  if (!bytes) return fail(GCPSL_EINVAL, "null output");
  CHECK(bad_rows(dtype, rows, L));
  CHECK(bad_top(top, L));
  *bytes = score_work_bytes(dtype, rows, L, top);
  return GCPSL_OK;
}

extern "C" int gcpsl_score(int32_t dtype, int64_t rows, int32_t L, const void *z, int64_t ldz, const int32_t *labels,
                           int32_t top, float *logp, float *entropy, float *lse, float *top_logp, int32_t *top_class,
                           void *workspace, size_t workspace_bytes, void *stream) {
  gcpsl_clear_error();
  CHECK(bad_rows(dtype, rows, L));
  CHECK(bad_top(top, L));
  CHECK(bad_tensor(z, elem_bytes(dtype), rows, L, ldz, false));
  if (rows > 0 && logp && !labels) return fail(GCPSL_EINVAL, "log probabilities need labels");
  if (rows > 0 && top > 0 && (!top_logp || !top_class)) return fail(GCPSL_EINVAL, "null output");
  for (const void *p : {(const void *)labels, (const void *)logp, (const void *)entropy, (const void *)lse,
                        (const void *)top_logp, (const void *)top_class})
    if (!aligned(p, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  const size_t need = score_work_bytes(dtype, rows, L, top);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 16))))
    return fail(GCPSL_EINVAL, "workspace null, too small or not 16-byte aligned");
  if (rows == 0) return GCPSL_OK;
  const ScoreArgs a{z, ldz, rows, L, top, labels, logp, entropy, lse, top_logp, top_class, workspace};
  return launched(launch_score(dtype, a, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" int gcpsl_score_grad(int32_t dtype, int64_t rows, int32_t L, const void *z, int64_t ldz,
                                const int32_t *labels, const float *lse, const float *entropy, const float *g_logp,
                                const float *g_entropy, void *dz, int64_t lddz, void *stream) {
  gcpsl_clear_error();
  CHECK(bad_rows(dtype, rows, L));
  CHECK(bad_tensor(z, elem_bytes(dtype), rows, L, ldz, false));
  CHECK(bad_tensor(dz, elem_bytes(dtype), rows, L, lddz, true));
  if (z && z == dz && rows > 1 && ldz != lddz) return fail(GCPSL_EINVAL, "in place needs equal row strides");
  if (rows > 0 && !lse) return fail(GCPSL_EINVAL, "null lse");
  if (rows > 0 && !g_logp && !g_entropy) return fail(GCPSL_EINVAL, "no gradient given");
  if (rows > 0 && g_logp && !labels) return fail(GCPSL_EINVAL, "log probabilities need labels");
  if (rows > 0 && g_entropy && !entropy) return fail(GCPSL_EINVAL, "null entropy");
  for (const void *p : {(const void *)labels, (const void *)lse, (const void *)entropy, (const void *)g_logp,
                        (const void *)g_entropy})
    if (!aligned(p, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  if (rows == 0) return GCPSL_OK;
  const ScoreGradArgs a{z, ldz, rows, L, labels, lse, entropy, g_logp, g_entropy, dz, lddz};
  return launched(launch_score_grad(dtype, a, reinterpret_cast<hipStream_t>(stream)));
}

namespace {
const char *bad_residual(int dtype, int G, int64_t rows, int n, const int32_t *offsets) {
  return bad_groups(dtype, G, rows, n, 1, offsets);
}
// Vectors [n] fp32 of every group; `out` ones must not overlap.
const char *bad_vectors(const float *p, int64_t gs, int G, int n, bool out) {
  if (!aligned(p, 4)) return "tensor not aligned to its elements";
  if (const char *why = bad_stride(gs)) return why;
  return p && out && G > 1 && gs < n ? "groups of an output overlap" : nullptr;
}
bool finite_f32(double v) { return std::fabs(v) <= 3.0e38; }  // (false for a NaN)
size_t residual_bytes(const GroupPieces &p, int n) { return sizeof(float) * 2 * (size_t)p.slots * (size_t)n; }
}  // namespace

extern "C" int gcpsl_group_residual_norm(int32_t dtype, int32_t G, int64_t rows, int32_t n, const int32_t *offsets,
                                         const void *x, int64_t ldx, const void *y, int64_t ldy, const void *gate,
                                         int64_t ldgate, const float *w_block, int64_t w_block_gs, const float *w_next,
                                         int64_t w_next_gs, double alpha, double beta, double eps, void *out,
                                         int64_t ldo, void *h, int64_t ldh, float *r_block, float *r_next,
                                         void *stream) {
  gcpsl_clear_error();
  CHECK(bad_residual(dtype, G, rows, n, offsets));
  if (rows > kMaxGroupRows) return fail(GCPSL_EUNSUPPORTED, "more than 2^31 - 1024 grouped rows");
  const size_t e = elem_bytes(dtype);
  CHECK(bad_tensor(x, e, rows, n, ldx, false));
  if (rows > 0 && !y && (gate || w_block || out || alpha != 1.0))
    return fail(GCPSL_EINVAL, "no block output: gate, w_block and out must be null and alpha 1");
  if (y) {
    CHECK(bad_tensor(y, e, rows, n, ldy, false));
    CHECK(bad_tensor(out, e, rows, n, ldo, true));
    if (out && out == x && rows > 1 && ldo != ldx) return fail(GCPSL_EINVAL, "in place needs equal row strides");
  }
  if (gate) CHECK(bad_tensor(gate, e, rows, n, ldgate, false));
  CHECK(bad_vectors(w_block, w_block_gs, G, n, false));
  CHECK(bad_vectors(w_next, w_next_gs, G, n, false));
  if (rows > 0 && !w_next != !h) return fail(GCPSL_EINVAL, "w_next and h come together");
  if (rows > 0 && !y && !w_next) return fail(GCPSL_EINVAL, "nothing to compute");
  if (h) CHECK(bad_tensor(h, e, rows, n, ldh, true));
  if (!aligned(r_block, 4) || !aligned(r_next, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  if (!finite_f32(alpha) || !finite_f32(beta)) return fail(GCPSL_EINVAL, "alpha and beta must be finite");
  if (!(eps >= std::ldexp(1.0, -100) && eps <= std::ldexp(1.0, 100)))
    return fail(GCPSL_EINVAL, "eps must lie in [2^-100, 2^100]");
  if (rows == 0) return GCPSL_OK;
  ResidualArgs a{};
  a.off = offsets;
  a.G = G; a.n = n; a.rows = rows;
  a.x = x; a.ldx = ldx;
  a.y = y; a.ldy = ldy;
  a.gate = gate; a.ldg = ldgate;
  a.w_block = w_block; a.wb_gs = w_block_gs;
  a.w_next = w_next; a.wn_gs = w_next_gs;
  a.alpha = (float)alpha; a.beta = (float)beta; a.eps = (float)eps;
  a.out = out; a.ldo = ldo;
  a.h = h; a.ldh = ldh;
  a.r_block = w_block ? r_block : nullptr;
  a.r_next = w_next ? r_next : nullptr;
  return launched(launch_residual(dtype, a, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" int gcpsl_group_residual_workspace_bytes(int32_t dtype, int32_t G, int64_t rows, int32_t n, size_t *bytes) {
  gcpsl_clear_error();
  if (!bytes) return fail(GCPSL_EINVAL, "null output");
  alignas(4) static const int32_t none = 0;
  CHECK(bad_residual(dtype, G, rows, n, &none));
  if (rows > kMaxGroupRows) return fail(GCPSL_EUNSUPPORTED, "more than 2^31 - 1024 grouped rows");
  *bytes = residual_bytes(residual_pieces(dtype, G, rows, n), n);
  return GCPSL_OK;
}

extern "C" int gcpsl_group_residual_norm_grad(
    int32_t dtype, int32_t G, int64_t rows, int32_t n, const int32_t *offsets, const void *out, int64_t ldo,
    const void *g_out, int64_t ldgo, const void *g_h, int64_t ldgh, const void *y, int64_t ldy, const void *gate,
    int64_t ldgate, const float *w_block, int64_t w_block_gs, const float *w_next, int64_t w_next_gs,
    const float *r_block, const float *r_next, double alpha, double beta, void *dx, int64_t lddx, void *dy,
    int64_t lddy, void *dgate, int64_t lddgate, float *dw_block, int64_t dw_block_gs, float *dw_next,
    int64_t dw_next_gs, void *workspace, size_t workspace_bytes, void *stream) {
  gcpsl_clear_error();
  CHECK(bad_residual(dtype, G, rows, n, offsets));
  if (rows > kMaxGroupRows) return fail(GCPSL_EUNSUPPORTED, "more than 2^31 - 1024 grouped rows");
  const size_t e = elem_bytes(dtype);
  if (g_h && !w_next) return fail(GCPSL_EINVAL, "g_h without w_next");  // (the weights' gradients without rows, too)
  if (rows > 0) {
    if (!g_out && !g_h) return fail(GCPSL_EINVAL, "no gradient given");
    if (!g_h != !w_next || (g_h && (!r_next || !out))) return fail(GCPSL_EINVAL, "g_h, w_next, r_next and out come together");
    if (!y && (gate || w_block || dy || alpha != 1.0))
      return fail(GCPSL_EINVAL, "no block output: gate, w_block and dy must be null and alpha 1");
    if (w_block && !r_block) return fail(GCPSL_EINVAL, "null r_block");
  }
  if ((dgate && !gate) || (dw_block && !w_block) || (dw_next && !w_next))
    return fail(GCPSL_EINVAL, "a gradient of what is not given");
  if (g_h) CHECK(bad_tensor(out, e, rows, n, ldo, false));
  if (g_out) CHECK(bad_tensor(g_out, e, rows, n, ldgo, false));
  if (g_h) CHECK(bad_tensor(g_h, e, rows, n, ldgh, false));
  if (y) {
    CHECK(bad_tensor(y, e, rows, n, ldy, false));
    CHECK(bad_tensor(dy, e, rows, n, lddy, true));
  }
  if (gate) CHECK(bad_tensor(gate, e, rows, n, ldgate, false));
  CHECK(bad_vectors(w_block, w_block_gs, G, n, false));
  CHECK(bad_vectors(w_next, w_next_gs, G, n, false));
  CHECK(bad_tensor(dx, e, rows, n, lddx, true));
  if (dgate) CHECK(bad_tensor(dgate, e, rows, n, lddgate, true));
  CHECK(bad_vectors(dw_block, dw_block_gs, G, n, true));
  CHECK(bad_vectors(dw_next, dw_next_gs, G, n, true));
  if (!aligned(r_block, 4) || !aligned(r_next, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  if (!finite_f32(alpha) || !finite_f32(beta)) return fail(GCPSL_EINVAL, "alpha and beta must be finite");
  const GroupPieces pieces = residual_pieces(dtype, G, rows, n);
  if (dw_block || dw_next) {
    if (residual_bytes(pieces, n) > workspace_bytes) return fail(GCPSL_EINVAL, "workspace too small");
    if (pieces.slots && (!workspace || !aligned(workspace, 16)))
      return fail(GCPSL_EINVAL, "workspace null or not 16-byte aligned");
  }
  if (rows == 0 && !dw_block && !dw_next) return GCPSL_OK;
  ResidualGradArgs a{};
  a.off = offsets;
  a.G = G; a.n = n; a.rows = rows;
  a.x = out; a.ldx = ldo;
  a.g_out = g_out; a.ldgo = ldgo;
  a.g_h = g_h; a.ldgh = ldgh;
  a.y = y; a.ldy = ldy;
  a.gate = gate; a.ldg = ldgate;
  a.w_block = w_block; a.wb_gs = w_block_gs;
  a.w_next = w_next; a.wn_gs = w_next_gs;
  a.r_block = r_block; a.r_next = r_next;
  a.alpha = (float)alpha; a.beta = (float)beta;
  a.dx = dx; a.lddx = lddx;
  a.dy = dy; a.lddy = lddy;
  a.dgate = dgate; a.lddg = lddgate;
  a.dw_block = dw_block; a.dwb_gs = dw_block_gs;
  a.dw_next = dw_next; a.dwn_gs = dw_next_gs;
  a.piece = pieces.piece;
  a.slots = pieces.slots;
  a.part = (float *)workspace;
  return launched(launch_residual_grad(dtype, a, reinterpret_cast<hipStream_t>(stream)));
}

namespace {
const char *bad_teacher(int64_t rows, int top, const int32_t *t_class, const float *t_value, double temperature) {
  if (top < 1 || top > kMaxTeacher) return "top must lie in [1, 256]";
  if (rows > 0 && (!t_class || !t_value)) return "null teacher";
  if (!aligned(t_class, 4) || !aligned(t_value, 4)) return "tensor not aligned to its elements";
  return !(temperature >= 1.0 / 1024 && temperature <= 1024.0) ? "temperature must lie in [2^-10, 2^10]" : nullptr;
}
}  // namespace

extern "C" int gcpsl_distill_workspace_bytes(int32_t dtype, int64_t rows, int32_t L, size_t *bytes) {
  gcpsl_clear_error();
  if (!bytes) return fail(GCPSL_EINVAL, "null output");
  CHECK(bad_rows(dtype, rows, L));
  *bytes = distill_work_bytes(dtype, rows, L);
  return GCPSL_OK;
}

extern "C" int gcpsl_distill(int32_t dtype, int64_t rows, int32_t L, const void *z, int64_t ldz, int32_t top,
                             const int32_t *t_class, const float *t_value, double temperature, const int32_t *labels,
                             float *kl, float *lse_t, float *logp, float *lse, void *workspace, size_t workspace_bytes,
                             void *stream) {
  gcpsl_clear_error();
  CHECK(bad_rows(dtype, rows, L));
  CHECK(bad_tensor(z, elem_bytes(dtype), rows, L, ldz, false));
  CHECK(bad_teacher(rows, top, t_class, t_value, temperature));
  if (rows > 0 && logp && !labels) return fail(GCPSL_EINVAL, "log probabilities need labels");
  for (const void *p : {(const void *)labels, (const void *)kl, (const void *)lse_t, (const void *)logp,
                        (const void *)lse})
    if (!aligned(p, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  const size_t need = distill_work_bytes(dtype, rows, L);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 16))))
    return fail(GCPSL_EINVAL, "workspace null, too small or not 16-byte aligned");
  if (rows == 0) return GCPSL_OK;
  const DistillArgs a{z,  ldz,   rows, L,   top,      t_class, t_value, (float)temperature,
                      labels, kl, lse_t, logp, lse, workspace};
  return launched(launch_distill(dtype, a, reinterpret_cast<hipStream_t>(stream)));
}

extern "C" int gcpsl_distill_grad(int32_t dtype, int64_t rows, int32_t L, const void *z, int64_t ldz, int32_t top,
                                  const int32_t *t_class, const float *t_value, double temperature,
                                  const int32_t *labels, const float *lse_t, const float *lse, const float *g_kl,
                                  const float *g_logp, void *dz, int64_t lddz, void *stream) {
  gcpsl_clear_error();
  CHECK(bad_rows(dtype, rows, L));
  CHECK(bad_tensor(z, elem_bytes(dtype), rows, L, ldz, false));
  CHECK(bad_tensor(dz, elem_bytes(dtype), rows, L, lddz, true));
  if (z && z == dz && rows > 1 && ldz != lddz) return fail(GCPSL_EINVAL, "in place needs equal row strides");
  if (rows > 0 && !g_kl && !g_logp) return fail(GCPSL_EINVAL, "no gradient given");
  CHECK(bad_teacher(g_kl ? rows : 0, top, t_class, t_value, temperature));
  if (rows > 0 && g_kl && !lse_t) return fail(GCPSL_EINVAL, "null lse_t");
  if (rows > 0 && g_logp && (!labels || !lse)) return fail(GCPSL_EINVAL, "log probabilities need labels and lse");
  for (const void *p : {(const void *)labels, (const void *)lse_t, (const void *)lse, (const void *)g_kl,
                        (const void *)g_logp})
    if (!aligned(p, 4)) return fail(GCPSL_EINVAL, "tensor not aligned to its elements");
  if (rows == 0) return GCPSL_OK;
  const DistillGradArgs a{z,      ldz,   rows, L,    top,    t_class, t_value, (float)temperature,
                          labels, lse_t, lse,  g_kl, g_logp, dz,      lddz};
  return launched(launch_distill_grad(dtype, a, reinterpret_cast<hipStream_t>(stream)));
}
