// C entry points of the operators around a stage's tasks: argument checks on
// the host, then the launchers of train_ops.h.
#include "train_ops.h"

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

// Whether rows of w bytes, la apart from a on, share bytes with rows lb apart
// from b on.
bool rows_meet(int64_t a, int64_t la, int64_t b, int64_t lb, int64_t rows, int64_t w) {
  if (a + (rows - 1) * la + w <= b || b + (rows - 1) * lb + w <= a) return false;
  // every distance of a row of b from one of a is that of a and b but for
  // multiples of what divides both la and lb
  const int64_t g = std::gcd(la, lb), d = ((b - a) % g + g) % g;
  if (d >= w && g - d >= w) return false;
  // row by row of a: the rows of b that start last at or before it and next
  // (where those of very many rows do not keep clear as above, they meet)
  if (la != lb && rows > 1 << 16) return true;
  const int64_t step = la == lb ? 1 : rows;
  for (int64_t i = 0; i < step; ++i) {
    const int64_t at = a + i * la - b, k = (at >= 0 ? at : at - lb + 1) / lb;
    for (int64_t j = k; j <= k + 1; ++j) {
      // (of equal distances only the difference of the rows' numbers counts)
      const bool there = la == lb ? std::abs(j) < rows : j >= 0 && j < rows;
      if (there && std::abs(at - j * lb) < w) return true;
    }
  }
  return false;
}

// `out` may lie on `in` row by row, and share nothing with it otherwise.
tgp_status check_apart(const char* who, const char* out, const void* p, int64_t ldp, const char* in,
                       const void* q, int64_t ldq, int64_t rows, int C, int dtype) {
  if (p == q && (ldp == ldq || rows == 1)) return TGP_OK;
  const int64_t e = dtype == TGP_BF16 ? 2 : 4;
  if (rows_meet((int64_t)(uintptr_t)q, ldq * e, (int64_t)(uintptr_t)p, ldp * e, rows, C * e))
    return fail(TGP_EINVAL, "%s: %s overlaps %s and is not %s itself at its row distance", who, out, in, in);
  return TGP_OK;
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

}  // extern "C"
