// Host side of the layer norm, the gated layers and the orthogonalised updates (include/lp.h): argument checks, workspace layouts, dispatch by
// element type.
#include <math.h>

#include <algorithm>

#include "../../include/lp.h"
#include "lp_internal.h"
#include "lp_mm.h"

namespace {

using lp::check_ws;
using lp::fail;
using lp::hip_fail;

constexpr size_t up(size_t x) { return (x + 255) / 256 * 256; }

// Limits as for the layer steps (lp_step_host.cpp): 32-bit index arithmetic inside a tile stays far from its own.
constexpr int kMaxRows = 1 << 24, kMaxWidth = 1 << 20, kMaxShort = 1 << 15, kMaxSteps = 64;
constexpr double kMaxValues = 34359738368.0;  // 2^35

size_t esize(int32_t d) { return d == LP_F32 ? 4 : 2; }

int check_type(int32_t abi, int32_t dtype) {
  if (abi != LP_ABI_VERSION) return fail(LP_EINVAL, "abi_version %d != %d", abi, LP_ABI_VERSION);
  if (dtype == LP_F64) return fail(LP_EUNSUPPORTED, "no kernel for dtype LP_F64 (LP_F32, LP_BF16, LP_F16)");
  if (dtype != LP_F32 && dtype != LP_BF16 && dtype != LP_F16) return fail(LP_EINVAL, "bad dtype %d", dtype);
  return LP_OK;
}

int check_rows(int32_t B) {
  if (B < 0) return fail(LP_EINVAL, "B = %d < 0", B);
  if (B > kMaxRows) return fail(LP_EUNSUPPORTED, "B = %d > %d", B, kMaxRows);
  return LP_OK;
}

int check_gated(const lp_gated* g) {
  if (!g) return fail(LP_EINVAL, "layer is NULL");
  int rc = check_type(g->abi_version, g->dtype);
  if (rc) return rc;
  if (g->act < LP_TANH || g->act > LP_GELU) return fail(LP_EINVAL, "bad activation %d", g->act);
  if ((rc = check_rows(g->B))) return rc;
  if (g->ni < 1 || g->no < 1) return fail(LP_EINVAL, "bad widths ni = %d, no = %d", g->ni, g->no);
  if (g->ni > kMaxWidth || g->no > kMaxWidth)
    return fail(LP_EUNSUPPORTED, "widths ni = %d, no = %d > %d", g->ni, g->no, kMaxWidth);
  if (std::max({(double)g->B * g->no, (double)g->B * g->ni, (double)g->no * g->ni}) > kMaxValues)
    return fail(LP_EUNSUPPORTED, "more than 2^35 values in an array");
  return LP_OK;
}

int check_norm(const lp_norm* n) {
  if (!n) return fail(LP_EINVAL, "norm is NULL");
  int rc = check_type(n->abi_version, n->dtype);
  if (rc || (rc = check_rows(n->B))) return rc;
  if (n->q < 1) return fail(LP_EINVAL, "q = %d < 1", n->q);
  if (n->q > kMaxWidth) return fail(LP_EUNSUPPORTED, "q = %d > %d", n->q, kMaxWidth);
  if ((double)n->B * n->q > kMaxValues) return fail(LP_EUNSUPPORTED, "more than 2^35 values in an array");
  if (!(n->eps >= 0) || !isfinite((float)n->eps)) return fail(LP_EINVAL, "eps must be >= 0 and finite in fp32");
  return LP_OK;
}

int check_orth(const lp_orth* o) {
  if (!o) return fail(LP_EINVAL, "update is NULL");
  const int rc = check_type(o->abi_version, o->dtype);
  if (rc) return rc;
  if (o->N < 0) return fail(LP_EINVAL, "N = %d < 0", o->N);
  if (o->no < 1 || o->ni < 1) return fail(LP_EINVAL, "bad sizes no = %d, ni = %d", o->no, o->ni);
  if (o->steps < 1 || o->steps > kMaxSteps) return fail(LP_EINVAL, "steps = %d, not in 1..%d", o->steps, kMaxSteps);
  if (o->nesterov != 0 && o->nesterov != 1) return fail(LP_EINVAL, "nesterov must be 0 or 1");
  for (double v : {o->a, o->b, o->c, o->mu})
    if (!isfinite(v) || !isfinite((float)v)) return fail(LP_EINVAL, "a, b, c and mu must be finite in fp32");
  if (!(o->eps >= 0) || !isfinite(o->eps)) return fail(LP_EINVAL, "eps must be >= 0 and finite");
  if (o->N > kMaxRows || o->no > kMaxWidth || o->ni > kMaxWidth || std::min(o->no, o->ni) > kMaxShort)
    return fail(LP_EUNSUPPORTED, "N = %d > %d, no = %d or ni = %d > %d, or both > %d", o->N, kMaxRows, o->no, o->ni, kMaxWidth, kMaxShort);
  if ((double)o->N * o->no * o->ni > kMaxValues) return fail(LP_EUNSUPPORTED, "more than 2^35 values in an array");
  return LP_OK;
}

// whether two of n arrays (nullable) are the same
bool any_same(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    if (!*o) continue;
    for (const void* i : ins)
      if (*o == i) return true;
    for (auto p = outs.begin(); p != o; ++p)
      if (*o == *p) return true;
  }
  return false;
}

// Offsets of a workspace's parts
struct Parts {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t r = at;
    at += up(bytes);
    return r;
  }
  size_t total() const { return std::max<size_t>(at, 256); }
};

}  // namespace

namespace lp {

// dx and dz^T x as one launch where both take the smallest tiles and contract over at most so many stages, unsplit; one side
// alone is then unsplit too, so that its bits do not depend on what else is wanted. The whole way back against a launch
// each, split as the plans are, microseconds by the longer contraction's stages.
//   bf16: 21 (209 x 649 -> 649) 22.9 (25.3), 38 (1500 x 100 -> 1200) 30.1 (36.1), 57 (300 x 200 -> 1800) 24.6 (26.2), 72
//         (4600 x 200 -> 700) 38.5 (43.6), 79 (400 x 300 -> 2500) 42.5 (38.0)
//   f32:  20 (600 x 300 -> 300) 35.1 (41.7), 25 (800 x 100 -> 150) 30.7 (33.3), 26 (700 x 200 -> 400) 36.6 (40.0), 29
//         (900 x 128 -> 200) 33.7 (34.5), 30 (250 x 300 -> 450) 41.5 (37.9), 32 (100 x 100 -> 500) 35.9 (28.2), 38
//         (1000 x 220 -> 587) 47.8 (48.4); dx alone of the last two unsplit 36.1 (22.0) and 46.9 (32.0)
constexpr int both_stages(size_t e) { return e == 2 ? 72 : 28; }

// The pair's plan. Its smallest tile (two waves, 32 features of each array) takes 0.30 us a stage alone on a CU and 0.45 beside
// another (floats 0.75, 1.15), no less than its weights' reading takes; joining a split 5 us: 24 x 2048 -> 5120 f16
// 14.2 us whole, 17.2, 21.8 and 28.1 in two, four and eight; 2 x 4096 -> 4096 bf16 22.9, 23.1, 24.3, 35.3.
static mm::Plan pair_plan(size_t e, int B, int ni, int no) {
  mm::Plan p = mm::plan_of(e, B, 2L * no, ni);
  if (p.tile != 64) return p;
  const int steps = mm::ceil_div(ni * (long)e, mm::STAGE_BYTES);
  const double one = e == 2 ? 0.30 : 0.75, two = e == 2 ? 0.45 : 1.15, read = 2.0 * no * ni * e / 4.9e6;
  double least = 1e30;
  for (int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
    if (splits > 1 && steps < 4 * splits) break;
    const long n = mm::ceil_div((long)p.tm * p.tn * splits, 256);
    double t = std::max(read, mm::ceil_div(steps, splits) * ((n / 2) * two + (n % 2) * one));
    if (splits > 1) t += 5.0 + 2.0 * splits * B * p.tn * 64 * 4 / 3e6;
    if (t < least) least = t, p.splits = splits;
  }
  return p;
}

GatedLayout gated_layout(int dtype, int B, int ni, int no, bool grad) {
  const size_t e = esize(dtype), row = mm::padded(e, ni) * e;
  const int two = 2 * mm::ceil_div(no, mm::PAIR_BLOCK) * mm::PAIR_BLOCK;
  GatedLayout l{};
  // (a pair's tile holds half a tile's features of each: the tiles of a product of 2 no features)
  l.z = pair_plan(e, B, ni, no);
  if (B == 1 && !grad) l.z = mm::Plan{1, 1, 1, mm::ceil_div(no, mm::one_features(2L * no) / 2)};
  size_t part = l.z.part_bytes();
  Parts p;
  if (grad) {
    l.zx = mm::plan_of(e, B, ni, two);
    l.zw = mm::plan_of(e, two, ni, B);
    const double stages = mm::ceil_div((long)std::max(two, B) * (long)e, mm::STAGE_BYTES);
    l.both = l.zx.tile == 64 && l.zw.tile == 64 && stages <= both_stages(e);
    if (l.both) l.zx.splits = l.zw.splits = 1;
    part = std::max({part, l.zx.part_bytes(), l.zw.part_bytes()});
    // (and the layer itself, whose plan differs for one row only and then has no sums to join)
    l.dz = p.take((size_t)B * two * e);
  }
  l.x = p.take(B * row);
  l.Wg = p.take(no * row);
  l.Wu = p.take(no * row);
  l.part = p.take(part);
  l.total = p.total();
  return l;
}

// Matrices are taken a chunk at a time, whose X, A and P take ORTH_CHUNK at most: enough that launches and their uneven
// ends do not count (2048 of 220 x 220 f32: 7.2 ms by 64 MiB, 6.2 by 128, which the last cache would hold, 5.4 by 512, 5.0).
constexpr size_t ORTH_CHUNK = (size_t)1 << 30;

// A symmetric product over rows, tiles of 192 where they are estimated faster: n = 4096 has 253 of them (136 of 256, 528
// of 128), one for every CU.
static mm::Plan sym_plan(size_t e, int n, int k, int batch, bool duo) {
  const mm::Plan p = mm::plan_of(e, n, n, k, batch, true, duo);
  const int tm = mm::ceil_div(n, 192);
  const double us = mm::ceil_div(k * (long)e, 128) * (double)mm::ceil_div((long)batch * tm * (tm + 1) / 2, 256) * (duo ? 1.6 : 1.1);
  return us < p.us ? mm::Plan{192, 1, tm, tm, us} : p;
}

OrthLayout orth_layout(int dtype, int N, int no, int ni) {
  const size_t e = esize(dtype);  // (of the products: f16 for both 16-bit types)
  const int n = std::min(no, ni), k = std::max(no, ni);
  OrthLayout l{};
  if (orth_small(no, ni)) {
    l.total = 256;
    return l;
  }
  const bool duo = dtype == LP_F32;
  l.ld = (mm::padded(e, ni) + 7) / 8 * 8;
  l.lda = (mm::padded(e, n) + 7) / 8 * 8;
  l.ldlo = duo ? 0 : (l.ld + 15) / 16 * 16;
  const size_t x = (size_t)no * l.ld * e, a = (size_t)n * l.lda * e, lo = (size_t)no * l.ldlo;
  l.chunk = (int)std::min<size_t>(std::max(N, 1), std::min<size_t>(std::max<size_t>(ORTH_CHUNK / (2 * (x + a) + lo), 1), 16384));
  l.parts = (int)std::min<size_t>(((size_t)no * ni + 4095) / 4096, 2048);
  l.gram = no > ni ? mm::plan_of(e, n, n, k, l.chunk, true, duo) : sym_plan(e, n, k, l.chunk, duo);
  l.poly = sym_plan(e, n, n, l.chunk, duo);
  l.next = mm::plan_of(e, no, ni, n, l.chunk, false, duo);
  const auto part = [&](const mm::Plan& p, bool sym) {
    return p.splits > 1 ? (size_t)l.chunk * p.splits * tiles_of(p, sym) * p.tile * p.tile * 4 : 0;
  };
  Parts p;
  l.norms = p.take((size_t)l.chunk * l.parts * 8);
  for (size_t& at : l.X) at = p.take(l.chunk * x);
  l.lo = p.take(l.chunk * lo);
  l.A = p.take(l.chunk * a);
  l.P = p.take(l.chunk * a);
  l.part = p.take(std::max({part(l.gram, true), part(l.poly, true), part(l.next, false)}));
  l.total = p.total();
  return l;
}

}  // namespace lp

#define LP_BY_TYPE(dtype, call, ...)                     \
  ((dtype) == LP_F32    ? lp::call##_f32(__VA_ARGS__)    \
   : (dtype) == LP_BF16 ? lp::call##_bf16(__VA_ARGS__)   \
                        : lp::call##_f16(__VA_ARGS__))

extern "C" {

size_t lp_norm_workspace_bytes(const lp_norm* n) {
  if (check_norm(n) != LP_OK) return 0;
  lp::clear_error();
  return lp::norm_layout(n->dtype, n->B, n->q).total;
}

int32_t lp_norm_forward(const lp_norm* n, const void* x, const void* gamma, const void* beta, void* y, void* stream) {
  int rc = check_norm(n);
  if (rc) return rc;
  if (n->B && (!x || !y)) return fail(LP_EINVAL, "NULL array argument");
  if (n->B && any_same({y}, {gamma, beta})) return fail(LP_EINVAL, "y aliases a weight");
  if (n->B == 0) return LP_OK;
  lp::NormArgs a{};
  a.dtype = n->dtype, a.B = n->B, a.q = n->q, a.eps = n->eps;
  a.x = x, a.gamma = gamma, a.beta = beta, a.y = y;
  const hipError_t e = LP_BY_TYPE(n->dtype, norm_forward, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "norm forward");
}

int32_t lp_norm_backward(const lp_norm* n, const void* x, const void* gamma, const void* dy, const void* dr, void* dx,
                         void* dgamma, void* dbeta, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_norm(n);
  if (rc) return rc;
  if (n->B && (!x || !dy)) return fail(LP_EINVAL, "NULL array argument");
  if (any_same({dx, dgamma, dbeta}, {x, gamma, dy}) || any_same({dgamma, dbeta}, {dr}))
    return fail(LP_EINVAL, "an output aliases an input or another output");
  if ((rc = check_ws(ws, ws_bytes, lp::norm_layout(n->dtype, n->B, n->q).total))) return rc;
  if (!dx && !dgamma && !dbeta) return LP_OK;
  lp::NormArgs a{};
  a.dtype = n->dtype, a.B = n->B, a.q = n->q, a.eps = n->eps;
  a.x = x, a.gamma = gamma, a.dy = dy, a.dr = dr, a.dx = dx, a.dgamma = dgamma, a.dbeta = dbeta, a.ws = ws;
  const hipError_t e = LP_BY_TYPE(n->dtype, norm_backward, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "norm backward");
}

size_t lp_gated_workspace_bytes(const lp_gated* g, int32_t grad) {
  if (check_gated(g) != LP_OK) return 0;
  lp::clear_error();
  return lp::gated_layout(g->dtype, g->B, g->ni, g->no, grad != 0).total;
}

int32_t lp_gated_forward(const lp_gated* g, const void* x, const void* Wg, const void* Wu, void* y, void* ws,
                         size_t ws_bytes, void* stream) {
  int rc = check_gated(g);
  if (rc) return rc;
  if (!Wg || !Wu || (g->B && (!x || !y))) return fail(LP_EINVAL, "NULL array argument");
  if (g->B && any_same({y}, {x, Wg, Wu})) return fail(LP_EINVAL, "y aliases an input");
  if ((rc = check_ws(ws, ws_bytes, lp::gated_layout(g->dtype, g->B, g->ni, g->no, false).total))) return rc;
  if (g->B == 0) return LP_OK;
  lp::GatedArgs a{};
  a.dtype = g->dtype, a.act = g->act, a.B = g->B, a.ni = g->ni, a.no = g->no;
  a.x = x, a.Wg = Wg, a.Wu = Wu, a.y = y, a.ws = ws;
  const hipError_t e = LP_BY_TYPE(g->dtype, gated_forward, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "gated forward");
}

int32_t lp_gated_backward(const lp_gated* g, const void* x, const void* Wg, const void* Wu, const void* dy, void* dx,
                          void* dWg, void* dWu, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_gated(g);
  if (rc) return rc;
  if (!Wg || !Wu || (g->B && (!x || !dy))) return fail(LP_EINVAL, "NULL array argument");
  if (any_same({dx, dWg, dWu}, {x, Wg, Wu, dy})) return fail(LP_EINVAL, "an output aliases an input or another output");
  if ((rc = check_ws(ws, ws_bytes, lp::gated_layout(g->dtype, g->B, g->ni, g->no, true).total))) return rc;
  if (!dx && !dWg && !dWu) return LP_OK;
  lp::GatedArgs a{};
  a.dtype = g->dtype, a.act = g->act, a.B = g->B, a.ni = g->ni, a.no = g->no;
  a.x = x, a.Wg = Wg, a.Wu = Wu, a.dy = dy, a.dx = dx, a.dWg = dWg, a.dWu = dWu, a.ws = ws;
  const hipError_t e = LP_BY_TYPE(g->dtype, gated_backward, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "gated backward");
}

size_t lp_orth_workspace_bytes(const lp_orth* o) {
  if (check_orth(o) != LP_OK) return 0;
  lp::clear_error();
  return lp::orth_layout(o->dtype, o->N, o->no, o->ni).total;
}

int32_t lp_orth_update(const lp_orth* o, const void* g, const float* m, float* mo, double alpha, double beta, const void* r,
                       void* W, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_orth(o);
  if (rc) return rc;
  if (!isfinite(alpha) || !isfinite((float)alpha) || !isfinite(beta) || !isfinite((float)beta))
    return fail(LP_EINVAL, "alpha and beta must be finite in fp32");
  if (o->N && (!g || !W)) return fail(LP_EINVAL, "NULL array argument");
  if (m && !mo) return fail(LP_EINVAL, "m is given without mo");
  if (o->nesterov && !mo) return fail(LP_EINVAL, "nesterov without a momentum");
  if (any_same({W, mo}, {g}) || any_same({W}, {m}) || any_same({mo}, {r}))
    return fail(LP_EINVAL, "an output aliases an input or another output");
  if ((rc = check_ws(ws, ws_bytes, lp::orth_layout(o->dtype, o->N, o->no, o->ni).total))) return rc;
  if (o->N == 0) return LP_OK;
  lp::OrthArgs a{o->dtype, o->N, o->no, o->ni, o->steps, o->nesterov, o->a, o->b, o->c, o->eps, o->mu, alpha, beta, g, m, mo, r, W, ws};
  const hipError_t e = LP_BY_TYPE(o->dtype, orth_update, a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LP_OK : hip_fail(e, "orthogonalised update");
}

}  // extern "C"
