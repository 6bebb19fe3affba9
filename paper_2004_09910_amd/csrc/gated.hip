// A gated feed-forward block over the channels of each pixel, forward and
// backward: y = (act(x Wg^T + bg) * (x Wu^T + bu)) Wd^T + bd.
#include <algorithm>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256;

// act(g) and act'(g).
__device__ __forceinline__ float2 act_of(float g, int act) {
  if (act == TGP_ACT_SILU) {
    const float p = 1.f / (1.f + expf(-g));
    return make_float2(g * p, p * (1.f + g * (1.f - p)));
  }
  const float p = 0.5f * (1.f + erff(g * 0.70710678f));
  return make_float2(g * p, p + g * expf(-0.5f * g * g) * 0.39894228f);
}

// h (and dg, du) of one pixel and hidden channel a thread.
template <typename T>
__global__ __launch_bounds__(kT) void hidden_any(tgp_gated_shape s, long rows, tgp_gated_weights w, const T* x,
                                                 long ldx, const T* dy, long lddy, float* h, float* dg, float* du) {
  const long e = (long)blockIdx.x * kT + threadIdx.x, r = e / s.hidden;
  const int j = (int)(e % s.hidden);
  if (r >= rows) return;
  float g = w.b_gate ? w.b_gate[j] : 0.f, u = w.b_up ? w.b_up[j] : 0.f, d = 0.f;
  for (int c = 0; c < s.cin; ++c) {
    const float v = Elt<T>::ld(x + r * ldx + c);
    g += v * Elt<T>::ld((const T*)w.gate + (long)j * s.cin + c);
    u += v * Elt<T>::ld((const T*)w.up + (long)j * s.cin + c);
  }
  const float2 a = act_of(g, s.act);
  h[e] = a.x * u;
  if (!dy) return;
  for (int c = 0; c < s.cout; ++c)
    d += Elt<T>::ld(dy + r * lddy + c) * Elt<T>::ld((const T*)w.down + (long)c * s.hidden + j);
  dg[e] = d * u * a.y;
  du[e] = d * a.x;
}

template <typename T>
__global__ __launch_bounds__(kT) void out_any(tgp_gated_shape s, long rows, const T* down, const float* bias,
                                              const float* h, T* y, long ldy) {
  const long e = (long)blockIdx.x * kT + threadIdx.x, r = e / s.cout;
  const int c = (int)(e % s.cout);
  if (r >= rows) return;
  float v = bias ? bias[c] : 0.f;
  for (int j = 0; j < s.hidden; ++j) v += h[r * s.hidden + j] * Elt<T>::ld(down + (long)c * s.hidden + j);
  Elt<T>::st(y + r * ldy + c, v);
}

template <typename T>
__global__ __launch_bounds__(kT) void dx_any(tgp_gated_shape s, long rows, const T* gate, const T* up, const float* dg,
                                             const float* du, T* dx, long lddx) {
  const long e = (long)blockIdx.x * kT + threadIdx.x, r = e / s.cin;
  const int c = (int)(e % s.cin);
  if (r >= rows) return;
  float v = 0.f;
  for (int j = 0; j < s.hidden; ++j)
    v += dg[r * s.hidden + j] * Elt<T>::ld(gate + (long)j * s.cin + c) +
         du[r * s.hidden + j] * Elt<T>::ld(up + (long)j * s.cin + c);
  Elt<T>::st(dx + r * lddx + c, v);
}

// to (+)= a^T b over the rows, a of m and b of n columns (b NULL: ones).
template <typename A, typename B>
__global__ __launch_bounds__(kT) void outer_any(long rows, const A* a, long lda, int m, const B* b, long ldb, int n,
                                                float* to, int overwrite) {
  const long e = (long)blockIdx.x * kT + threadIdx.x;
  const long i = e / n;
  const int j = (int)(e % n);
  if (i >= m) return;
  double v = 0;
  for (long r = 0; r < rows; ++r) v += (double)Elt<A>::ld(a + r * lda + i) * (b ? Elt<B>::ld(b + r * ldb + j) : 1.f);
  to[e] = overwrite ? (float)v : to[e] + (float)v;
}

unsigned grid(long n) { return (unsigned)((n + kT - 1) / kT); }

template <typename T>
hipError_t forward_t(const Gated& g, const void* x, long ldx, void* y, long ldy, void* ws, hipStream_t st) {
  float* h = (float*)ws;
  {
    ProfScope ps("gated_hidden", 0, 0, st);
    TGP_LAUNCH(ps, hidden_any<T>, dim3(grid(g.rows * g.s.hidden)), dim3(kT), 0, st, g.s, g.rows, g.w, (const T*)x, ldx,
               (const T*)nullptr, 0l, h, (float*)nullptr, (float*)nullptr);
  }
  ProfScope ps("gated_out", 0, 0, st);
  TGP_LAUNCH(ps, out_any<T>, dim3(grid(g.rows * g.s.cout)), dim3(kT), 0, st, g.s, g.rows, (const T*)g.w.down,
             g.w.b_down, h, (T*)y, ldy);
  return launch_status();
}

template <typename T>
hipError_t backward_t(const Gated& g, const void* dyp, long lddy, const void* xp, long ldx, void* dx, long lddx,
                      const tgp_gated_grads& gr, int overwrite, void* ws, hipStream_t st) {
  const int cin = g.s.cin, hidden = g.s.hidden, cout = g.s.cout;
  const T *x = (const T*)xp, *dy = (const T*)dyp;
  float *h = (float*)ws, *dg = h + g.rows * hidden, *du = dg + g.rows * hidden;
  {
    ProfScope ps("gated_hidden", 0, 0, st);
    TGP_LAUNCH(ps, hidden_any<T>, dim3(grid(g.rows * hidden)), dim3(kT), 0, st, g.s, g.rows, g.w, x, ldx, dy, lddy, h,
               dg, du);
  }
  auto outer = [&](auto* a, long lda, int m, auto* b, long ldb, int n, float* to) {
    if (!to) return;
    typedef std::remove_cv_t<std::remove_pointer_t<decltype(a)>> A;
    typedef std::remove_cv_t<std::remove_pointer_t<decltype(b)>> B;
    ProfScope ps("gated_outer", 0, 0, st);
    TGP_LAUNCH(ps, (outer_any<A, B>), dim3(grid((long)m * n)), dim3(kT), 0, st, g.rows, (const A*)a, lda, m,
               (const B*)b, ldb, n, to, overwrite);
  };
  outer(dg, hidden, hidden, x, ldx, cin, gr.gate);
  outer(du, hidden, hidden, x, ldx, cin, gr.up);
  outer(dy, lddy, cout, h, hidden, hidden, gr.down);
  const T* ones = nullptr;
  outer(dg, hidden, hidden, ones, 0, 1, gr.b_gate);
  outer(du, hidden, hidden, ones, 0, 1, gr.b_up);
  outer(dy, lddy, cout, ones, 0, 1, gr.b_down);
  if (dx) {   // last: it may be written over x or dy
    ProfScope ps("gated_dx", 0, 0, st);
    TGP_LAUNCH(ps, dx_any<T>, dim3(grid(g.rows * cin)), dim3(kT), 0, st, g.s, g.rows, (const T*)g.w.gate,
               (const T*)g.w.up, dg, du, (T*)dx, lddx);
  }
  return launch_status();
}

__global__ void zero_k(float* p, long n) {
  const long i = (long)blockIdx.x * kT + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

}  // namespace

size_t gated_bytes(const tgp_gated_shape& s, long rows, bool backward) {
  return (size_t)rows * s.hidden * 4 * (backward ? 3 : 1);
}

hipError_t gated_forward(const Gated& g, const void* x, long ldx, void* y, long ldy, void* ws, hipStream_t st) {
  return g.s.dtype == TGP_BF16 ? forward_t<bf16_t>(g, x, ldx, y, ldy, ws, st)
                               : forward_t<float>(g, x, ldx, y, ldy, ws, st);
}

hipError_t gated_backward(const Gated& g, const void* dy, long lddy, const void* x, long ldx, void* dx, long lddx,
                          const tgp_gated_grads& gr, bool overwrite, void* ws, hipStream_t st) {
  if (g.rows == 0) {
    if (!overwrite) return hipSuccess;
    const long m = (long)g.s.hidden * g.s.cin, k = (long)g.s.hidden * g.s.cout;
    const std::pair<float*, long> all[] = {{gr.gate, m}, {gr.up, m}, {gr.down, k}, {gr.b_gate, g.s.hidden},
                                           {gr.b_up, g.s.hidden}, {gr.b_down, g.s.cout}};
    for (const auto& a : all) {
      if (!a.first) continue;
      ProfScope ps("gated_zero", 0, 4.0 * a.second, st);
      TGP_LAUNCH(ps, zero_k, dim3(grid(a.second)), dim3(kT), 0, st, a.first, a.second);
    }
    return launch_status();
  }
  return g.s.dtype == TGP_BF16 ? backward_t<bf16_t>(g, dy, lddy, x, ldx, dx, lddx, gr, overwrite, ws, st)
                               : backward_t<float>(g, dy, lddy, x, ldx, dx, lddx, gr, overwrite, ws, st);
}

}  // namespace tgpk
