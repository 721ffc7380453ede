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
