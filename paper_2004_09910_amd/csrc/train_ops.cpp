// C entry points of the operators around a stage's tasks: argument checks on
// the host, then the launchers of train_ops.h.
#include "train_ops.h"

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <numeric>

#include "error.h"
#include "tgp.h"

using tgpk::fail;

namespace {

bool at(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// The shape both directions share; `who` names the call.
tgp_status check_norm(const char* who, int64_t rows, int C, int dtype) {
  if (dtype != TGP_BF16 && dtype != TGP_FP32) return fail(TGP_EINVAL, "%s: bad dtype %d", who, dtype);
  if (rows < 0 || C < 1)
    return fail(TGP_EINVAL, "%s: bad shape %lld x %d", who, (long long)rows, C);
  // byte offsets stay far inside 64 bits, and row counts inside the kernels' 32-bit block maths
  if (rows > ((int64_t)1 << 40) / C)
    return fail(TGP_EINVAL, "%s: %lld x %d values are too many", who, (long long)rows, C);
  // a block steps through a row's channels in 32 bits
  if (C > 1 << 30) return fail(TGP_EUNSUPPORTED, "%s: rows of %d channels are too long", who, C);
  return TGP_OK;
}

tgp_status check_rows(const char* who, const char* name, const void* p, int64_t ld, int C, int dtype,
                      int64_t rows) {
  if (!p) return fail(TGP_EINVAL, "%s: %s is NULL", who, name);
  if (ld < C) return fail(TGP_EINVAL, "%s: rows of %s are %lld apart, less than %d", who, name,
                          (long long)ld, C);
  if (ld > ((int64_t)1 << 42) / (rows > 0 ? rows : 1))
    return fail(TGP_EINVAL, "%s: rows of %s are %lld apart: too far", who, name, (long long)ld);
  if (!at(p, dtype == TGP_BF16 ? 2 : 4))
    return fail(TGP_EINVAL, "%s: %s (%p) is not aligned to its elements", who, name, p);
  return TGP_OK;
}

// Whether rows of wa bytes, la apart from a on, share bytes with rows of wb, lb
// apart from b on.
bool rows_meet(int64_t a, int64_t la, int64_t wa, int64_t b, int64_t lb, int64_t wb, int64_t rows) {
  if (a + (rows - 1) * la + wa <= b || b + (rows - 1) * lb + wb <= a) return false;
  // every distance of a row of b from one of a is that of a and b but for
  // multiples of what divides both la and lb
  const int64_t g = std::gcd(la, lb), d = ((b - a) % g + g) % g;
  if (d >= wa && g - d >= wb) return false;
  // row by row of a: the rows of b that start last at or before it and next
  // (where those of very many rows do not keep clear as above, they meet)
  if (la != lb && rows > 1 << 16) return true;
  const int64_t step = la == lb ? 1 : rows;
  for (int64_t i = 0; i < step; ++i) {
    const int64_t at = a + i * la - b, k = (at >= 0 ? at : at - lb + 1) / lb;
    for (int64_t j = k; j <= k + 1; ++j) {
      // (of equal distances only the difference of the rows' numbers counts)
      const bool there = la == lb ? std::abs(j) < rows : j >= 0 && j < rows;
      const int64_t past = at - j * lb;   // from the row of b to that of a
      if (there && past < wb && -past < wa) return true;
    }
  }
  return false;
}

// Rows of a tensor for the overlap checks.
struct Place {
  const char* name;
  const void* p;
  int64_t ld, rows, C;
};

// `out` may lie on `in` row by row (itself: whether it may), and share nothing with
// it otherwise.
tgp_status check_apart(const char* who, const Place& out, const Place& in, int dtype, bool itself = true) {
  if (!out.p || !in.p || out.rows == 0 || in.rows == 0) return TGP_OK;
  const int64_t e = dtype == TGP_BF16 ? 2 : 4, rows = std::min(out.rows, in.rows);
  if (itself && out.p == in.p && out.C == in.C && out.rows == in.rows && (out.ld == in.ld || rows == 1))
    return TGP_OK;
  const int64_t a = (int64_t)(uintptr_t)in.p, b = (int64_t)(uintptr_t)out.p;
  // of tensors of different numbers of rows, all that lies between first and last
  const bool meet = out.rows == in.rows
      ? rows_meet(a, in.ld * e, in.C * e, b, out.ld * e, out.C * e, rows)
      : !(a + ((in.rows - 1) * in.ld + in.C) * e <= b || b + ((out.rows - 1) * out.ld + out.C) * e <= a);
  if (!meet) return TGP_OK;
  return itself ? fail(TGP_EINVAL, "%s: %s overlaps %s and is not %s itself at its row distance", who, out.name,
                       in.name, in.name)
                : fail(TGP_EINVAL, "%s: %s overlaps %s", who, out.name, in.name);
}
tgp_status check_apart(const char* who, const char* out, const void* p, int64_t ldp, const char* in,
                       const void* q, int64_t ldq, int64_t rows, int C, int dtype) {
  return check_apart(who, Place{out, p, ldp, rows, C}, Place{in, q, ldq, rows, C}, dtype);
}

tgp_status check_ptr(const char* who, const char* name, int k, const void* p, size_t align,
                     bool required) {
  if (!p && required) return fail(TGP_EINVAL, "%s: tensor %d: %s is NULL", who, k, name);
  if (!at(p, align))
    return fail(TGP_EINVAL, "%s: tensor %d: %s (%p) is not at a multiple of %zu bytes", who, k, name,
                p, align);
  return TGP_OK;
}

#define TRY(expr)                     \
  do {                                \
    tgp_status s_ = (expr);           \
    if (s_ != TGP_OK) return s_;      \
  } while (0)

tgp_status check_list(const char* who, int n, const void* t) {
  if (n < 0) return fail(TGP_EINVAL, "%s: n = %d", who, n);
  if (n > 0 && !t) return fail(TGP_EINVAL, "%s: the tensor list is NULL", who);
  return TGP_OK;
}

tgp_status check_muon(const char* who, int n, const tgp_muon_tensor* t) {
  TRY(check_list(who, n, t));
  for (int k = 0; k < n; ++k) {
    if (t[k].rows < 1 || t[k].cols < 1)
      return fail(TGP_EINVAL, "%s: tensor %d: bad shape %d x %d", who, k, t[k].rows, t[k].cols);
    const int64_t r = ((int64_t)t[k].rows + 127) / 128 * 128, c = ((int64_t)t[k].cols + 127) / 128 * 128;
    if (r * c >= (int64_t)1 << 30)
      return fail(TGP_EUNSUPPORTED, "%s: tensor %d: %d x %d is too large", who, k, t[k].rows,
                  t[k].cols);
  }
  return TGP_OK;
}

tgp_status check_gated(const char* who, const tgp_gated_shape* s, int64_t rows) {
  if (!s) return fail(TGP_EINVAL, "%s: shape is NULL", who);
  if (s->dtype != TGP_BF16 && s->dtype != TGP_FP32) return fail(TGP_EINVAL, "%s: bad dtype %d", who, s->dtype);
  if (s->act != TGP_ACT_SILU && s->act != TGP_ACT_GELU) return fail(TGP_EINVAL, "%s: bad act %d", who, s->act);
  if (rows < 0 || s->cin < 1 || s->hidden < 1 || s->cout < 1)
    return fail(TGP_EINVAL, "%s: bad shape %lld x %d x %d x %d", who, (long long)rows, s->cin, s->hidden, s->cout);
  // a tile steps through a matrix in 32 bits, and counts rows in 31
  const int64_t most = (int64_t)1 << 30;
  if (s->cin > 1 << 20 || s->hidden > 1 << 20 || s->cout > 1 << 20 || (int64_t)s->hidden * s->cin >= most ||
      (int64_t)s->hidden * s->cout >= most || rows >= (int64_t)1 << 31)
    return fail(TGP_EUNSUPPORTED, "%s: %lld x %d x %d x %d is too large", who, (long long)rows, s->cin, s->hidden,
                s->cout);
  return TGP_OK;
}

tgp_status check_gated_weights(const char* who, const tgp_gated_shape* s, const tgp_gated_weights* w) {
  if (!w) return fail(TGP_EINVAL, "%s: weights is NULL", who);
  if (!w->gate || !w->up || !w->down) return fail(TGP_EINVAL, "%s: a weight matrix is NULL", who);
  const size_t e = s->dtype == TGP_BF16 ? 2 : 4;
  if (!at(w->gate, e) || !at(w->up, e) || !at(w->down, e))
    return fail(TGP_EINVAL, "%s: a weight matrix is not aligned to its elements", who);
  if (!at(w->b_gate, 4) || !at(w->b_up, 4) || !at(w->b_down, 4))
    return fail(TGP_EINVAL, "%s: a bias is not aligned", who);
  return TGP_OK;
}

tgp_status check_ws(const char* who, const void* ws, size_t bytes, size_t need, size_t align) {
  if (need == 0) return TGP_OK;
  if (!ws) return fail(TGP_EINVAL, "%s: ws is NULL", who);
  if (!at(ws, align)) return fail(TGP_EINVAL, "%s: ws is not at a multiple of %zu bytes", who, align);
  if (bytes < need) return fail(TGP_ENOSPACE, "%s: workspace of %zu bytes, %zu needed", who, bytes, need);
  return TGP_OK;
}

// The shape and what both directions read; `gate`: whether there is one.
tgp_status check_residual(const char* who, const tgp_residual_shape* s, bool gate) {
  if (!s) return fail(TGP_EINVAL, "%s: shape is NULL", who);
  TRY(check_norm(who, s->rows, s->C, s->dtype));
  if (s->C > tgpk::kResidualMaxC)
    return fail(TGP_EUNSUPPORTED, "%s: rows of %d channels are too long", who, s->C);
  if (s->post != 0 && s->post != 1) return fail(TGP_EINVAL, "%s: post is %d, not 0 or 1", who, s->post);
  if (!(s->eps >= 0.f) || std::isinf(s->eps)) return fail(TGP_EINVAL, "%s: bad eps %g", who, s->eps);
  if (gate && (s->group < 1 || s->rows % s->group))
    return fail(TGP_EINVAL, "%s: %lld rows are not whole groups of %lld", who, (long long)s->rows,
                (long long)s->group);
  return TGP_OK;
}

tgp_status check_residual_params(const char* who, const tgp_residual_params* w) {
  if (!w) return fail(TGP_EINVAL, "%s: params is NULL", who);
  if (!at(w->scale, 4) || !at(w->post_gain, 4) || !at(w->post_bias, 4) || !at(w->pre_gain, 4) || !at(w->pre_bias, 4))
    return fail(TGP_EINVAL, "%s: a scale, gain or bias is not aligned", who);
  return TGP_OK;
}

// Each of outs against every in, on which it may lie row by row, and every other out.
tgp_status check_places(const char* who, const Place* ins, int n_in, const Place* outs, int n_out, int dtype) {
  for (int o = 0; o < n_out; ++o) {
    for (int i = 0; i < n_in; ++i) TRY(check_apart(who, outs[o], ins[i], dtype));
    for (int q = 0; q < o; ++q) TRY(check_apart(who, outs[o], outs[q], dtype, false));
  }
  return TGP_OK;
}

}  // namespace

extern "C" {

tgp_status tgp_layer_norm_forward(int64_t rows, int C, int dtype, const void* x, int64_t ldx,
                                  const float* gain, const float* bias, float eps, void* y,
                                  int64_t ldy, float* stats, void* stream) {
  const char* who = "layer_norm_forward";
  TRY(check_norm(who, rows, C, dtype));
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(TGP_EINVAL, "%s: bad eps %g", who, eps);
  if (!at(gain, 4) || !at(bias, 4) || !at(stats, 8))
    return fail(TGP_EINVAL, "%s: gain, bias or stats is not aligned", who);
  if (rows == 0) return TGP_OK;
  TRY(check_rows(who, "x", x, ldx, C, dtype, rows));
  TRY(check_rows(who, "y", y, ldy, C, dtype, rows));
  TRY(check_apart(who, "y", y, ldy, "x", x, ldx, rows, C, dtype));
  HIPCHK(tgpk::layer_norm_forward(dtype, {(long)rows, C}, x, ldx, gain, bias, eps, y, ldy, stats,
                                  (hipStream_t)stream),
         who);
  return TGP_OK;
}

tgp_status tgp_layer_norm_backward_workspace(int64_t rows, int C, int dtype, size_t* bytes) {
  const char* who = "layer_norm_backward_workspace";
  if (!bytes) return fail(TGP_EINVAL, "%s: bytes is NULL", who);
  TRY(check_norm(who, rows, C, dtype));
  *bytes = tgpk::layer_norm_partial_floats(dtype, {(long)rows, C}) * sizeof(float);
  return TGP_OK;
}

tgp_status tgp_layer_norm_backward(int64_t rows, int C, int dtype, const void* dy, int64_t lddy,
                                   const void* x, int64_t ldx, const float* gain,
                                   const float* stats, void* dx, int64_t lddx, float* dgain,
                                   float* dbias, int overwrite, void* ws, size_t ws_bytes,
                                   void* stream) {
  const char* who = "layer_norm_backward";
  TRY(check_norm(who, rows, C, dtype));
  if (!dgain != !dbias) return fail(TGP_EINVAL, "%s: dgain and dbias are both set or both NULL", who);
  if (!dgain && !dx) return fail(TGP_EINVAL, "%s: nothing to compute (dx and dgain are NULL)", who);
  if (overwrite != 0 && overwrite != 1)
    return fail(TGP_EINVAL, "%s: overwrite is %d, not 0 or 1", who, overwrite);
  if (!at(gain, 4) || !at(stats, 8) || !at(dgain, 4) || !at(dbias, 4))
    return fail(TGP_EINVAL, "%s: gain, stats, dgain or dbias is not aligned", who);
  if (rows > 0) {
    TRY(check_rows(who, "dy", dy, lddy, C, dtype, rows));
    TRY(check_rows(who, "x", x, ldx, C, dtype, rows));
    if (dx) {
      TRY(check_rows(who, "dx", dx, lddx, C, dtype, rows));
      TRY(check_apart(who, "dx", dx, lddx, "dy", dy, lddy, rows, C, dtype));
      TRY(check_apart(who, "dx", dx, lddx, "x", x, ldx, rows, C, dtype));
    }
    if (!stats) return fail(TGP_EINVAL, "%s: stats is NULL", who);
    const size_t need = dgain ? tgpk::layer_norm_partial_floats(dtype, {(long)rows, C}) * 4 : 0;
    if (need) {
      if (!ws) return fail(TGP_EINVAL, "%s: ws is NULL", who);
      if (!at(ws, 16)) return fail(TGP_EINVAL, "%s: ws is not at a multiple of 16 bytes", who);
      if (ws_bytes < need)
        return fail(TGP_ENOSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
    }
  }
  HIPCHK(tgpk::layer_norm_backward(dtype, {(long)rows, C}, dy, lddy, x, ldx, gain, stats, dx, lddx,
                                   dgain, dbias, overwrite != 0, (float*)ws, (hipStream_t)stream),
         who);
  return TGP_OK;
}

tgp_status tgp_gated_workspace(const tgp_gated_shape* shape, int64_t rows, int backward, size_t* bytes) {
  const char* who = "gated_workspace";
  if (!bytes) return fail(TGP_EINVAL, "%s: bytes is NULL", who);
  TRY(check_gated(who, shape, rows));
  if (backward != 0 && backward != 1) return fail(TGP_EINVAL, "%s: backward is %d, not 0 or 1", who, backward);
  *bytes = rows ? tgpk::gated_bytes(*shape, (long)rows, backward != 0) : 0;
  return TGP_OK;
}

tgp_status tgp_gated_forward(const tgp_gated_shape* shape, int64_t rows, const tgp_gated_weights* weights,
                             const void* x, int64_t ldx, void* y, int64_t ldy, void* ws, size_t ws_bytes,
                             void* stream) {
  const char* who = "gated_forward";
  TRY(check_gated(who, shape, rows));
  TRY(check_gated_weights(who, shape, weights));
  if (rows == 0) return TGP_OK;
  const int dtype = shape->dtype;
  TRY(check_rows(who, "x", x, ldx, shape->cin, dtype, rows));
  TRY(check_rows(who, "y", y, ldy, shape->cout, dtype, rows));
  TRY(check_apart(who, Place{"y", y, ldy, rows, shape->cout}, Place{"x", x, ldx, rows, shape->cin}, dtype, false));
  TRY(check_ws(who, ws, ws_bytes, tgpk::gated_bytes(*shape, (long)rows, false), 256));
  HIPCHK(tgpk::gated_forward({*shape, (long)rows, *weights}, x, ldx, y, ldy, ws, (hipStream_t)stream), who);
  return TGP_OK;
}

tgp_status tgp_gated_backward(const tgp_gated_shape* shape, int64_t rows, const tgp_gated_weights* weights,
                              const void* dy, int64_t lddy, const void* x, int64_t ldx, void* dx, int64_t lddx,
                              const tgp_gated_grads* grads, int overwrite, void* ws, size_t ws_bytes,
                              void* stream) {
  const char* who = "gated_backward";
  TRY(check_gated(who, shape, rows));
  TRY(check_gated_weights(who, shape, weights));
  if (overwrite != 0 && overwrite != 1)
    return fail(TGP_EINVAL, "%s: overwrite is %d, not 0 or 1", who, overwrite);
  const tgp_gated_grads g = grads ? *grads : tgp_gated_grads{};
  if (!at(g.gate, 4) || !at(g.up, 4) || !at(g.down, 4) || !at(g.b_gate, 4) || !at(g.b_up, 4) || !at(g.b_down, 4))
    return fail(TGP_EINVAL, "%s: a gradient is not aligned", who);
  if (!dx && !g.gate && !g.up && !g.down && !g.b_gate && !g.b_up && !g.b_down)
    return fail(TGP_EINVAL, "%s: nothing to compute (dx and every gradient are NULL)", who);
  if (rows > 0) {
    const int dtype = shape->dtype;
    TRY(check_rows(who, "dy", dy, lddy, shape->cout, dtype, rows));
    TRY(check_rows(who, "x", x, ldx, shape->cin, dtype, rows));
    if (dx) {
      TRY(check_rows(who, "dx", dx, lddx, shape->cin, dtype, rows));
      const Place to{"dx", dx, lddx, rows, shape->cin};
      TRY(check_apart(who, to, Place{"dy", dy, lddy, rows, shape->cout}, dtype));
      TRY(check_apart(who, to, Place{"x", x, ldx, rows, shape->cin}, dtype));
    }
    TRY(check_ws(who, ws, ws_bytes, tgpk::gated_bytes(*shape, (long)rows, true), 256));
  }
  HIPCHK(tgpk::gated_backward({*shape, (long)rows, *weights}, dy, lddy, x, ldx, dx, lddx, g, overwrite != 0, ws,
                              (hipStream_t)stream),
         who);
  return TGP_OK;
}

tgp_status tgp_residual_norm_forward(const tgp_residual_shape* shape, const tgp_residual_params* params,
                                     const void* r, int64_t ldr, const void* f, int64_t ldf, const void* gate,
                                     int64_t ldgate, void* out, int64_t ldout, void* z, int64_t ldz, float* stats,
                                     void* stream) {
  const char* who = "residual_norm_forward";
  TRY(check_residual(who, shape, gate != nullptr));
  TRY(check_residual_params(who, params));
  if (!at(stats, 16)) return fail(TGP_EINVAL, "%s: stats is not at a multiple of 16 bytes", who);
  const int64_t rows = shape->rows, groups = gate ? rows / shape->group : 0;
  const int C = shape->C, dtype = shape->dtype;
  if (rows == 0) return TGP_OK;
  TRY(check_rows(who, "r", r, ldr, C, dtype, rows));
  TRY(check_rows(who, "f", f, ldf, C, dtype, rows));
  TRY(check_rows(who, "out", out, ldout, C, dtype, rows));
  if (gate) TRY(check_rows(who, "gate", gate, ldgate, C, dtype, groups));
  if (z) TRY(check_rows(who, "z", z, ldz, C, dtype, rows));
  const Place ins[] = {{"r", r, ldr, rows, C}, {"f", f, ldf, rows, C}, {"gate", gate, ldgate, groups, C}};
  const Place outs[] = {{"out", out, ldout, rows, C}, {"z", z, ldz, rows, C}};
  TRY(check_places(who, ins, 3, outs, 2, dtype));
  if (gate && shape->group > 1)   // one row for several pixels: read after the first of them is written
    for (const Place& o : outs) TRY(check_apart(who, o, ins[2], dtype, false));
  HIPCHK(tgpk::residual_norm_forward({*shape, *params, {(void*)r, ldr}, {(void*)f, ldf}, {(void*)gate, ldgate},
                                      {out, ldout}, {z, ldz}, stats},
                                     (hipStream_t)stream),
         who);
  return TGP_OK;
}

tgp_status tgp_residual_norm_backward_workspace(const tgp_residual_shape* shape, size_t* bytes) {
  const char* who = "residual_norm_backward_workspace";
  if (!bytes) return fail(TGP_EINVAL, "%s: bytes is NULL", who);
  TRY(check_residual(who, shape, false));
  *bytes = shape->rows ? tgpk::residual_norm_partial_floats(*shape) * sizeof(float) : 0;
  return TGP_OK;
}

tgp_status tgp_residual_norm_backward(const tgp_residual_shape* shape, const tgp_residual_params* params,
                                      const void* dz, int64_t lddz, const void* dout, int64_t lddout,
                                      const void* out, int64_t ldout, const void* f, int64_t ldf, const void* gate,
                                      int64_t ldgate, const float* stats, void* dr, int64_t lddr, void* df,
                                      int64_t lddf, void* dgate, int64_t lddgate, const tgp_residual_grads* grads,
                                      int overwrite, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "residual_norm_backward";
  TRY(check_residual(who, shape, gate != nullptr));
  TRY(check_residual_params(who, params));
  if (overwrite != 0 && overwrite != 1)
    return fail(TGP_EINVAL, "%s: overwrite is %d, not 0 or 1", who, overwrite);
  const tgp_residual_grads g = grads ? *grads : tgp_residual_grads{};
  if (!at(g.scale, 4) || !at(g.post_gain, 4) || !at(g.post_bias, 4) || !at(g.pre_gain, 4) || !at(g.pre_bias, 4) ||
      !at(stats, 16))
    return fail(TGP_EINVAL, "%s: stats or a gradient is not aligned", who);
  if (!shape->post && (g.post_gain || g.post_bias))
    return fail(TGP_EINVAL, "%s: gradients of the post norm without one", who);
  if (dgate && !gate) return fail(TGP_EINVAL, "%s: dgate without a gate", who);
  const int64_t rows = shape->rows, groups = gate ? rows / shape->group : 0;
  const int C = shape->C, dtype = shape->dtype;
  if (rows > 0) {
    if (!dz && !dout) return fail(TGP_EINVAL, "%s: dz and dout are NULL", who);
    if (!dz && (g.pre_gain || g.pre_bias))
      return fail(TGP_EINVAL, "%s: gradients of the pre norm without dz", who);
    TRY(check_rows(who, "f", f, ldf, C, dtype, rows));
    TRY(check_rows(who, "dr", dr, lddr, C, dtype, rows));
    TRY(check_rows(who, "df", df, lddf, C, dtype, rows));
    if (dz) {
      TRY(check_rows(who, "dz", dz, lddz, C, dtype, rows));
      TRY(check_rows(who, "out", out, ldout, C, dtype, rows));
    }
    if (dout) TRY(check_rows(who, "dout", dout, lddout, C, dtype, rows));
    if (gate) TRY(check_rows(who, "gate", gate, ldgate, C, dtype, groups));
    if (dgate) TRY(check_rows(who, "dgate", dgate, lddgate, C, dtype, groups));
    if (!stats) return fail(TGP_EINVAL, "%s: stats is NULL", who);
    const void* read_out = dz ? out : nullptr;
    const Place ins[] = {{"dz", dz, lddz, rows, C}, {"dout", dout, lddout, rows, C}, {"out", read_out, ldout, rows, C},
                         {"f", f, ldf, rows, C}, {"gate", gate, ldgate, groups, C}};
    const Place outs[] = {{"dr", dr, lddr, rows, C}, {"df", df, lddf, rows, C}, {"dgate", dgate, lddgate, groups, C}};
    TRY(check_places(who, ins, 5, outs, 3, dtype));
    if (gate && shape->group > 1)   // sums over pixels still read the gate and the tensors of others
      for (const Place& o : outs)
        for (const Place& i : ins)
          if (o.p == dgate || i.p == gate) TRY(check_apart(who, o, i, dtype, false));
    TRY(check_ws(who, ws, ws_bytes, tgpk::residual_norm_partial_floats(*shape) * 4, 16));
  }
  {
    const tgpk::ResidualBackward a{*shape, *params, {(void*)dz, lddz}, {(void*)dout, lddout}, {(void*)out, ldout},
                                   {(void*)f, ldf}, {(void*)gate, ldgate}, stats, {dr, lddr}, {df, lddf},
                                   {dgate, lddgate}, g, overwrite != 0, (float*)ws};
    HIPCHK(tgpk::residual_norm_backward(a, (hipStream_t)stream), who);
  }
  return TGP_OK;
}

tgp_status tgp_muon_workspace(int n, const tgp_muon_tensor* t, size_t* bytes) {
  const char* who = "muon_workspace";
  if (!bytes) return fail(TGP_EINVAL, "%s: bytes is NULL", who);
  TRY(check_muon(who, n, t));
  *bytes = tgpk::muon_bytes(n, t);
  return TGP_OK;
}

tgp_status tgp_muon_update(int n, const tgp_muon_tensor* t, float mu, int nesterov, int steps,
                           float eps, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "muon_update";
  TRY(check_muon(who, n, t));
  if (!std::isfinite(mu)) return fail(TGP_EINVAL, "%s: bad mu %g", who, mu);
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(TGP_EINVAL, "%s: bad eps %g", who, eps);
  if (nesterov != 0 && nesterov != 1)
    return fail(TGP_EINVAL, "%s: nesterov is %d, not 0 or 1", who, nesterov);
  if (steps < 1) return fail(TGP_EINVAL, "%s: steps is %d", who, steps);
  for (int k = 0; k < n; ++k) {
    TRY(check_ptr(who, "grad", k, t[k].grad, 16, true));
    TRY(check_ptr(who, "momentum", k, t[k].momentum, 16, false));
    TRY(check_ptr(who, "update", k, t[k].update, 16, true));
  }
  if (n == 0) return TGP_OK;
  const size_t need = tgpk::muon_bytes(n, t);
  if (!ws) return fail(TGP_EINVAL, "%s: ws is NULL", who);
  if (!at(ws, 256)) return fail(TGP_EINVAL, "%s: ws is not at a multiple of 256 bytes", who);
  if (ws_bytes < need)
    return fail(TGP_ENOSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
  HIPCHK(tgpk::muon_update(n, t, mu, nesterov != 0, steps, eps, ws, (hipStream_t)stream), who);
  return TGP_OK;
}

tgp_status tgp_weight_step(int n, const tgp_step_tensor* t, float decay, void* stream) {
  const char* who = "weight_step";
  TRY(check_list(who, n, t));
  if (!std::isfinite(decay)) return fail(TGP_EINVAL, "%s: bad decay %g", who, decay);
  for (int k = 0; k < n; ++k) {
    if (t[k].count < 0 || t[k].count > (int64_t)1 << 40)
      return fail(TGP_EINVAL, "%s: tensor %d: bad count %lld", who, k, (long long)t[k].count);
    if (!std::isfinite(t[k].rate)) return fail(TGP_EINVAL, "%s: tensor %d: bad rate", who, k);
    TRY(check_ptr(who, "w", k, t[k].w, 16, t[k].count > 0));
    TRY(check_ptr(who, "update", k, t[k].update, 16, t[k].count > 0));
    TRY(check_ptr(who, "w16", k, t[k].w16, 16, false));
  }
  HIPCHK(tgpk::weight_step(n, t, decay, (hipStream_t)stream), who);
  return TGP_OK;
}

tgp_status tgp_adamw_step(int n, const tgp_adamw_tensor* t, float rate, float beta1, float beta2,
                          float eps, float decay, int64_t step, void* stream) {
  const char* who = "adamw_step";
  TRY(check_list(who, n, t));
  if (!std::isfinite(rate) || !std::isfinite(decay) || !(beta1 >= 0.f && beta1 < 1.f) ||
      !(beta2 >= 0.f && beta2 < 1.f) || !(eps >= 0.f) || std::isinf(eps))
    return fail(TGP_EINVAL, "%s: bad rate, beta, eps or decay", who);
  if (step < 1) return fail(TGP_EINVAL, "%s: step is %lld", who, (long long)step);
  for (int k = 0; k < n; ++k) {
    const bool some = t[k].count > 0;
    if (t[k].count < 0 || t[k].count > (int64_t)1 << 40)
      return fail(TGP_EINVAL, "%s: tensor %d: bad count %lld", who, k, (long long)t[k].count);
    TRY(check_ptr(who, "w", k, t[k].w, 16, some));
    TRY(check_ptr(who, "w16", k, t[k].w16, 16, false));
    TRY(check_ptr(who, "grad", k, t[k].grad, 16, some));
    TRY(check_ptr(who, "m", k, t[k].m, 16, some));
    TRY(check_ptr(who, "v", k, t[k].v, 16, some));
  }
  const float c1 = (float)(1.0 / (1.0 - std::pow((double)beta1, (double)step)));
  const float c2 = (float)(1.0 / (1.0 - std::pow((double)beta2, (double)step)));
  HIPCHK(tgpk::adamw_step(n, t, rate, beta1, beta2, eps, decay, c1, c2, (hipStream_t)stream), who);
  return TGP_OK;
}

tgp_status tgp_adamw8_step(int n, const tgp_adamw8_tensor* t, float rate, double beta1, double beta2, float eps,
                           float decay, int64_t step, uint64_t seed, void* stream) {
  const char* who = "adamw8_step";
  TRY(check_list(who, n, t));
  if (!std::isfinite(rate) || !std::isfinite(decay) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
      !(eps >= 0.f) || std::isinf(eps))
    return fail(TGP_EINVAL, "%s: bad rate, beta, eps or decay", who);
  if (step < 1) return fail(TGP_EINVAL, "%s: step is %lld", who, (long long)step);
  for (int k = 0; k < n; ++k) {
    const bool some = t[k].count > 0;
    if (t[k].count < 0 || t[k].count > (int64_t)1 << 40)
      return fail(TGP_EINVAL, "%s: tensor %d: bad count %lld", who, k, (long long)t[k].count);
    TRY(check_ptr(who, "w", k, t[k].w, 16, some));
    TRY(check_ptr(who, "w16", k, t[k].w16, 16, false));
    TRY(check_ptr(who, "grad", k, t[k].grad, 16, some));
    TRY(check_ptr(who, "m", k, t[k].m, 16, some));
    TRY(check_ptr(who, "root", k, t[k].root, 16, some));
    TRY(check_ptr(who, "exps", k, t[k].exps, 2, some));
  }
  const float c1 = (float)(1.0 / (1.0 - std::pow(beta1, (double)step)));
  const float rc2 = (float)std::sqrt(1.0 / (1.0 - std::pow(beta2, (double)step)));
  HIPCHK(tgpk::adamw8_step(n, t, rate, beta1, beta2, eps, decay, c1, rc2, seed, (hipStream_t)stream), who);
  return TGP_OK;
}

}  // extern "C"
