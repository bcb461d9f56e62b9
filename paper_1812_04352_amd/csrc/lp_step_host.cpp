// Host side of the layer steps of any width, the 8-bit checkpoints and the head over a large
// vocabulary (include/lp.h): argument checks, workspace layouts, dispatch by element type.
#include <math.h>

#include <algorithm>

#include "../../include/lp.h"
#include "lp_checkpoint.h"
#include "lp_internal.h"
#include "lp_mm.h"

namespace {

using lp::check_ws;
using lp::fail;
using lp::hip_fail;

constexpr size_t up(size_t x) { return (x + 255) / 256 * 256; }

// Row and feature counts keep 32-bit index arithmetic inside a tile (a stage's rows of an
// operand, the workgroups of a launch) far from its limits.
constexpr int kMaxRows = 1 << 24, kMaxWidth = 1 << 20, kMaxClasses = 1 << 24;
constexpr double kMaxResult = 34359738368.0;  // 2^35 values of a product's result

bool bad_type(int32_t d) { return d != LP_F32 && d != LP_BF16 && d != LP_F16; }
size_t esize(int32_t d) { return d == LP_F32 ? 4 : 2; }

int check_type(int32_t dtype) {
  if (dtype == LP_F64) return fail(LP_EUNSUPPORTED, "no kernel for dtype LP_F64 (LP_F32, LP_BF16, LP_F16)");
  if (bad_type(dtype)) return fail(LP_EINVAL, "bad dtype %d", dtype);
  return LP_OK;
}

int check_rows(int32_t B) {
  if (B < 0) return fail(LP_EINVAL, "B = %d < 0", B);
  if (B > kMaxRows) return fail(LP_EUNSUPPORTED, "B = %d > %d", B, kMaxRows);
  return LP_OK;
}

int check_step(const lp_step* s) {
  if (!s) return fail(LP_EINVAL, "step is NULL");
  if (s->abi_version != LP_ABI_VERSION) return fail(LP_EINVAL, "abi_version %d != %d", s->abi_version, LP_ABI_VERSION);
  int rc = check_type(s->dtype);
  if (rc) return rc;
  if (s->act < LP_TANH || s->act > LP_IDENTITY) return fail(LP_EINVAL, "bad activation %d", s->act);
  if ((rc = check_rows(s->B))) return rc;
  if (s->ni < 1 || s->no < 1) return fail(LP_EINVAL, "bad widths ni = %d, no = %d", s->ni, s->no);
  if (s->ni > kMaxWidth || s->no > kMaxWidth)
    return fail(LP_EUNSUPPORTED, "widths ni = %d, no = %d > %d", s->ni, s->no, kMaxWidth);
  if (std::max({(double)s->B * s->no, (double)s->B * s->ni, (double)s->no * s->ni}) > kMaxResult)
    return fail(LP_EUNSUPPORTED, "more than 2^35 values in an array");
  if (!isfinite(s->h) || !isfinite((float)s->h)) return fail(LP_EINVAL, "h must be finite in fp32");
  return LP_OK;
}

int check_head(const lp_label_head* h) {
  if (!h) return fail(LP_EINVAL, "head is NULL");
  if (h->abi_version != LP_ABI_VERSION) return fail(LP_EINVAL, "abi_version %d != %d", h->abi_version, LP_ABI_VERSION);
  int rc = check_type(h->dtype);
  if (rc) return rc;
  if ((rc = check_rows(h->B))) return rc;
  if (h->q < 1 || h->nc < 1) return fail(LP_EINVAL, "bad sizes q = %d, nc = %d", h->q, h->nc);
  if (h->q > kMaxWidth || h->nc > kMaxClasses)
    return fail(LP_EUNSUPPORTED, "q = %d > %d or nc = %d > %d", h->q, kMaxWidth, h->nc, kMaxClasses);
  if (std::max({(double)h->B * h->nc, (double)h->B * h->q, (double)h->nc * h->q}) > kMaxResult)
    return fail(LP_EUNSUPPORTED, "more than 2^35 values in an array");
  return LP_OK;
}

// the checkpoint calls take shapes directly
int check_ck(int32_t dtype, int32_t B, int32_t q, const void* x, const void* x8, const void* xe) {
  int rc = check_type(dtype);
  if (rc) return rc;
  if ((rc = check_rows(B))) return rc;
  if (q < 1) return fail(LP_EINVAL, "q = %d < 1", q);
  if (q > kMaxWidth) return fail(LP_EUNSUPPORTED, "q = %d > %d", q, kMaxWidth);
  if ((double)B * q > kMaxResult) return fail(LP_EUNSUPPORTED, "more than 2^35 values in an array");
  if (B && (!x || !x8 || !xe)) return fail(LP_EINVAL, "NULL array argument");
  if (B && x == x8) return fail(LP_EINVAL, "x and x8 alias");
  return LP_OK;
}

}  // namespace

namespace lp {

StepLayout step_layout(int dtype, int B, int ni, int no) {
  const size_t e = esize(dtype);
  StepLayout l;
  l.z = mm::plan_rows(e, B, no, ni);
  l.zx = mm::plan_of(e, B, ni, no);
  l.zw = mm::plan_of(e, no, ni, B);
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t r = at;
    at += up(bytes);
    return r;
  };
  l.g = take((size_t)B * mm::padded(e, no) * e);
  l.x = take((size_t)B * mm::padded(e, ni) * e);
  l.W = take((size_t)no * mm::padded(e, ni) * e);
  l.col = take((size_t)l.z.tm * no * 4);
  l.part = take(std::max({l.z.part_bytes(), l.zx.part_bytes(), l.zw.part_bytes()}));
  l.total = std::max<size_t>(at, 256);
  return l;
}

// A piece of the vocabulary holds at most PIECE_BYTES of probabilities, and of weights where those are
// copied (rows that do not start on 16 bytes), in whole tiles of classes (at least one).
constexpr size_t PIECE_BYTES = (size_t)256 << 20;

// The logits are kept in fp32 for the gradients where that takes less time than forming them twice:
// few enough to stay in the last cache (KEEP_CACHED: 520 rows, 50021 classes, 128 features f16 143 us
// against 170; 1024 rows, 32000 classes bf16 142 against 141; 2048 rows 270 against 230), or enough
// features (4096 rows, 65536 classes: bf16 1167 us against 1057 with 256, 1462 against 1480 with 512, 2137
// against 2351 with 1024; f32 1581 against 1533 with 64, 2047 against 2146 with 128, 4947 against 5980 with
// 512), and no more than KEEP_BYTES, a 70th of the card's memory.
constexpr size_t KEEP_BYTES = (size_t)4 << 30, KEEP_CACHED = (size_t)128 << 20;

bool keep_logits(size_t e, size_t bytes, int q) {
  return bytes <= KEEP_CACHED || (bytes <= KEEP_BYTES && q >= (e == 2 ? 512 : 128));
}

LabelLayout label_layout(int dtype, int B, int q, int nc, bool grad) {
  const size_t e = esize(dtype), ldq = mm::padded(e, q);
  LabelLayout l{};
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t r = at;
    at += up(bytes);
    return r;
  };
  const auto classes = [&](size_t row_bytes) {
    const size_t fit = row_bytes ? PIECE_BYTES / row_bytes / 256 * 256 : nc;
    return (int)std::min<size_t>(nc, std::max<size_t>(fit, 256));
  };
  l.piece = classes(grad ? B * e : 0);
  l.copied = std::min(l.piece, classes(ldq * e));
  size_t tiles = 0, split = 0, col = 0;
  for (int piece : {l.piece, l.copied}) {
    // every piece but the last is alike
    const int last = nc % piece ? nc % piece : piece, others = (nc - last) / piece;
    size_t t = 0;
    for (int i = 0; i < 2; ++i) {
      const int n = i ? last : piece;
      const mm::Plan z = mm::plan_rows(e, B, n, q);
      t += (size_t)z.tn * (i ? 1 : others);
      split = std::max(split, z.part_bytes());
      if (grad) {
        split = std::max({split, mm::plan_of(e, B, q, n).part_bytes(), mm::plan_of(e, n, q, B).part_bytes()});
        col = std::max(col, (size_t)std::max(z.tm, mm::ceil_div(B, 32)) * n * 4);  // (of products, or of 32 rows each)
      }
    }
    tiles = std::max(tiles, t);
  }
  l.part = take(tiles * B * 8);
  l.zl = take((size_t)B * 4);
  l.row = take((size_t)B * 4);
  l.u = take((size_t)B * ldq * e);
  l.W = take((size_t)l.copied * ldq * e);
  l.split = take(split);
  if (grad) {
    l.from = take((size_t)B * 4);
    l.to = take((size_t)B * 4);
    l.lab = take((size_t)B * 8);
    l.count = take(4);
    l.scale = take(4);
    l.lse = take((size_t)B * 4);
    const size_t logits = (size_t)B * mm::padded(e, nc) * 4;
    // (of floats the kept logits become P in place: a tile's rows, up to 256, lie within 2 GiB of each other)
    l.keep = keep_logits(e, logits, q) && (size_t)std::min(B, 256) * mm::padded(e, nc) * 4 < (size_t)1 << 31;
    if (l.keep) l.z = take(logits);
    l.P = l.keep && e == 4 ? l.z : take((size_t)B * mm::padded(e, l.piece) * e);
    l.du = take(l.copied < nc ? (size_t)B * q * 4 : 0);
    l.col = take(col);
  }
  l.total = std::max<size_t>(at, 256);
  return l;
}

}  // namespace lp

#define LP_BY_TYPE(dtype, call, ...)                     \
  ((dtype) == LP_F32    ? lp::call##_f32(__VA_ARGS__)    \
   : (dtype) == LP_BF16 ? lp::call##_bf16(__VA_ARGS__)   \
                        : lp::call##_f16(__VA_ARGS__))

extern "C" {

size_t lp_step_workspace_bytes(const lp_step* s) {
  if (check_step(s) != LP_OK) return 0;
  lp::clear_error();
  return lp::step_layout(s->dtype, s->B, s->ni, s->no).total;
}

int32_t lp_step_forward(const lp_step* s, const void* x, const void* W, const void* b, const void* r, void* y,
                        int8_t* y8, uint8_t* ye, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_step(s);
  if (rc) return rc;
  if (!W || (s->B && (!x || !y))) return fail(LP_EINVAL, "NULL array argument");
  if (s->B && (!y8 != !ye)) return fail(LP_EINVAL, "y8 and ye are given together or not at all");
  if (s->B && (y == x || y == W || (b && y == b))) return fail(LP_EINVAL, "y aliases an input other than r");
  if ((rc = check_ws(ws, ws_bytes, lp::step_layout(s->dtype, s->B, s->ni, s->no).total))) return rc;
  if (s->B == 0) return LP_OK;
  lp::StepArgs a{};
  a.dtype = s->dtype, a.act = s->act, a.B = s->B, a.ni = s->ni, a.no = s->no, a.h = s->h;
  a.x = x, a.W = W, a.b = b, a.r = r, a.y = y, a.y8 = y8, a.ye = ye, a.ws = ws;
  const hipError_t e = LP_BY_TYPE(s->dtype, step_forward, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "step forward");
}

int32_t lp_step_backward(const lp_step* s, const void* x, const int8_t* x8, const uint8_t* xe, const void* W,
                         const void* b, const void* dy, int32_t residual, void* dx, void* dW, void* db, void* ws,
                         size_t ws_bytes, void* stream) {
  int rc = check_step(s);
  if (rc) return rc;
  if (residual != 0 && residual != 1) return fail(LP_EINVAL, "residual must be 0 or 1");
  if (residual && s->ni != s->no) return fail(LP_EINVAL, "a residual of x needs ni = no (%d, %d)", s->ni, s->no);
  if (!W || (s->B && !dy)) return fail(LP_EINVAL, "NULL array argument");
  if (s->B && x && (x8 || xe)) return fail(LP_EINVAL, "x and its checkpoint are both given");
  if (s->B && !x && (!x8 || !xe)) return fail(LP_EINVAL, "neither x nor its checkpoint is given");
  for (const void* out : {(const void*)dx, (const void*)dW, (const void*)db})
    if (out && (out == x || out == x8 || out == xe || out == W || out == b || out == dy))
      return fail(LP_EINVAL, "an output aliases an input");
  if ((dx && (dx == dW || dx == db)) || (dW && dW == db)) return fail(LP_EINVAL, "outputs alias each other");
  if ((rc = check_ws(ws, ws_bytes, lp::step_layout(s->dtype, s->B, s->ni, s->no).total))) return rc;
  lp::StepArgs a{};
  a.dtype = s->dtype, a.act = s->act, a.B = s->B, a.ni = s->ni, a.no = s->no, a.h = s->h;
  a.x = x, a.x8 = x8, a.xe = xe, a.W = W, a.b = b, a.dy = dy, a.residual = residual;
  a.dx = dx, a.dW = dW, a.db = db, a.ws = ws;
  const hipError_t e = LP_BY_TYPE(s->dtype, step_backward, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "step backward");
}

int32_t lp_checkpoint_store(int32_t dtype, int32_t B, int32_t q, const void* x, int8_t* x8, uint8_t* xe, void* stream) {
  int rc = check_ck(dtype, B, q, x, x8, xe);
  if (rc || B == 0) return rc;
  const hipError_t e = LP_BY_TYPE(dtype, ck_store, x, x8, xe, B, q, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "checkpoint store");
}

int32_t lp_checkpoint_load(int32_t dtype, int32_t B, int32_t q, const int8_t* x8, const uint8_t* xe, void* x,
                           void* stream) {
  int rc = check_ck(dtype, B, q, x, x8, xe);
  if (rc || B == 0) return rc;
  const hipError_t e = LP_BY_TYPE(dtype, ck_load, x8, xe, x, B, q, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "checkpoint load");
}

size_t lp_loss_labels_workspace_bytes(const lp_label_head* h, int32_t grad) {
  if (check_head(h) != LP_OK) return 0;
  lp::clear_error();
  return lp::label_layout(h->dtype, h->B, h->q, h->nc, grad != 0).total;
}

int32_t lp_loss_labels(const lp_label_head* h, const void* u, const void* W, const void* mu, const int64_t* labels,
                       double gscale, float* J, float* row, void* du, void* dW, void* dmu, void* ws, size_t ws_bytes,
                       void* stream) {
  int rc = check_head(h);
  if (rc) return rc;
  if (!W || !J || (h->B && (!u || !labels))) return fail(LP_EINVAL, "NULL array argument");
  const bool grad = du || dW || dmu;
  if (dmu && !mu) return fail(LP_EINVAL, "dmu is given without mu");
  if (!isfinite(gscale) || !isfinite((float)gscale)) return fail(LP_EINVAL, "gscale must be finite in fp32");
  const void* outs[] = {J, row, du, dW, dmu};
  for (int i = 0; i < 5; ++i) {
    const void* out = outs[i];
    if (!out) continue;
    if (out == u || out == W || out == mu || out == labels) return fail(LP_EINVAL, "an output aliases an input");
    for (int j = 0; j < i; ++j)
      if (out == outs[j]) return fail(LP_EINVAL, "outputs alias each other");
  }
  if ((rc = check_ws(ws, ws_bytes, lp::label_layout(h->dtype, h->B, h->q, h->nc, grad).total))) return rc;
  const lp::LabelArgs a{h->dtype, h->B, h->q, h->nc, u, W, mu, labels, gscale, J, row, du, dW, dmu, ws};
  const hipError_t e = LP_BY_TYPE(h->dtype, loss_labels, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "loss of labels");
}

}  // extern "C"
