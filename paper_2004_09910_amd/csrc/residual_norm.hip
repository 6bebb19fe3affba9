// What stands between two blocks of a residual stream, in one pass over the
// tensors: the norm of a block's output, its gate and scale, the sum, and the
// norm that the next block reads.
//
// Forward: n = post_gain fhat + post_bias, out = r + scale gate n, z = pre_gain
// ohat + pre_bias, fhat and ohat a row less its mean, times rstd.
// Backward, G = dout + rstd_out (a - mean(a) - ohat mean(a ohat)) with a =
// pre_gain dz: dr = G, dn = scale gate G, df the same of b = post_gain dn and
// fhat.  Four sums over rows give all gradients of vectors: of dz ohat and dz,
// and of
//   S1 = gate G fhat, S2 = gate G:   dpost_gain = scale S1, dpost_bias = scale S2,
//   dscale = post_gain S1 + post_bias S2
// (without a post norm fhat stands for f: dscale = S1).  Over the pixels of one
// gate the same two sums without the gate, U1 and U2, give its gradient, scale
// (post_gain U1 + post_bias U2), and S1 and S2 are gate U1 and gate U2 added up.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256;   // threads of a block

// Sum over the block's kT threads, the same value in every thread.
template <typename F>
__device__ __forceinline__ F block_sum(F v, F* s4) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (s4[0] + s4[1]) + (s4[2] + s4[3]);
  __syncthreads();
  return v;
}

// Mean and rstd of the row in LDS.
__device__ __forceinline__ float2 row_stats(const float* row, int C, float eps, float* s4, double* d4, float* rest) {
  double s = 0;
  for (int c = threadIdx.x; c < C; c += kT) s += row[c];
  s = block_sum(s, d4) / C;
  const float mean = (float)s;
  *rest = (float)(s - mean);
  float q = 0.f;
  for (int c = threadIdx.x; c < C; c += kT) {
    const float d = row[c] - mean - *rest;
    q += d * d;
  }
  return make_float2(mean, 1.f / sqrtf(block_sum(q, s4) / C + eps));
}

__device__ __forceinline__ float at_or(const float* p, int c, float none) { return p ? p[c] : none; }

struct Vectors {
  const float *scale, *post_gain, *post_bias, *pre_gain, *pre_bias;
};

// A row a block at a time, held in LDS (kResidualMaxC values), one value a lane
// and access.
template <typename T>
__global__ __launch_bounds__(kT) void res_fwd_any(const T* r, long ldr, const T* f, long ldf, const T* gate,
                                                  long ldgate, long group, Vectors w, float eps, int post, T* out,
                                                  long ldout, T* z, long ldz, float4* stats, long rows, int C) {
  extern __shared__ float row[];
  __shared__ float s4[4];
  __shared__ double d4[4];
  for (long p = blockIdx.x; p < rows; p += gridDim.x) {
    const T* fr = f + p * ldf;
    for (int c = threadIdx.x; c < C; c += kT) row[c] = Elt<T>::ld(fr + c);
    __syncthreads();
    float2 a = make_float2(0.f, 0.f), b = a;
    float rest = 0.f;
    if (post) a = row_stats(row, C, eps, s4, d4, &rest);
    const T* q = gate ? gate + p / group * ldgate : nullptr;
    for (int c = threadIdx.x; c < C; c += kT) {
      float n = row[c];
      if (post) n = (n - a.x - rest) * a.y * at_or(w.post_gain, c, 1.f) + at_or(w.post_bias, c, 0.f);
      n *= at_or(w.scale, c, 1.f);
      if (q) n *= Elt<T>::ld(q + c);
      row[c] = Elt<T>::ld(r + p * ldr + c) + n;
      Elt<T>::st(out + p * ldout + c, row[c]);
    }
    __syncthreads();
    if (z) {
      b = row_stats(row, C, eps, s4, d4, &rest);
      for (int c = threadIdx.x; c < C; c += kT)
        Elt<T>::st(z + p * ldz + c,
                   (row[c] - b.x - rest) * b.y * at_or(w.pre_gain, c, 1.f) + at_or(w.pre_bias, c, 0.f));
    }
    if (stats && threadIdx.x == 0) stats[p] = make_float4(a.x, a.y, b.x, b.y);
    __syncthreads();
  }
}

// One gate's pixels (without a gate: one pixel) a block at a time, G of a row in
// LDS; a column's sums belong to one thread of the block and lie in part[block][6][C]:
// dz ohat, dz, S1, S2, and U1 and U2 of the present gate.
template <typename T>
__global__ __launch_bounds__(kT) void res_bwd_any(const T* dz, long lddz, const T* dout, long lddout, const T* out,
                                                  long ldout, const T* f, long ldf, const T* gate, long ldgate,
                                                  long group, Vectors w, int post, const float4* stats, T* dr,
                                                  long lddr, T* df, long lddf, T* dgate, long lddgate, float* part,
                                                  long rows, int C) {
  extern __shared__ float row[];
  __shared__ float s4[4];
  float* mine = part + (long)blockIdx.x * 6 * C;
  float *P0 = mine, *P1 = P0 + C, *S1 = P1 + C, *S2 = S1 + C, *U1 = S2 + C, *U2 = U1 + C;
  for (int c = threadIdx.x; c < C; c += kT) P0[c] = P1[c] = S1[c] = S2[c] = 0.f;
  const float inv_c = 1.f / C;
  for (long u = blockIdx.x; u * group < rows; u += gridDim.x) {
    const T* q = gate ? gate + u * ldgate : nullptr;
    for (int c = threadIdx.x; c < C; c += kT) U1[c] = U2[c] = 0.f;
    for (long p = u * group; p < (u + 1) * group; ++p) {
      const float4 st = stats[p];
      float ms = 0.f, mp = 0.f;
      if (dz) {
        for (int c = threadIdx.x; c < C; c += kT) {
          const float d = Elt<T>::ld(dz + p * lddz + c), a = d * at_or(w.pre_gain, c, 1.f);
          const float o = (Elt<T>::ld(out + p * ldout + c) - st.z) * st.w;
          ms += a;
          mp += a * o;
          P0[c] += d * o;
          P1[c] += d;
        }
        ms = block_sum(ms, s4) * inv_c;
        mp = block_sum(mp, s4) * inv_c;
      }
      float ns = 0.f, np = 0.f;
      for (int c = threadIdx.x; c < C; c += kT) {
        float G = dout ? Elt<T>::ld(dout + p * lddout + c) : 0.f;
        if (dz) {
          const float a = Elt<T>::ld(dz + p * lddz + c) * at_or(w.pre_gain, c, 1.f);
          const float o = (Elt<T>::ld(out + p * ldout + c) - st.z) * st.w;
          G += st.w * (a - ms - o * mp);
        }
        row[c] = G;
        if (!post) continue;
        const float fh = (Elt<T>::ld(f + p * ldf + c) - st.x) * st.y;
        const float b = G * at_or(w.scale, c, 1.f) * (q ? Elt<T>::ld(q + c) : 1.f) * at_or(w.post_gain, c, 1.f);
        ns += b;
        np += b * fh;
      }
      if (post) {
        ns = block_sum(ns, s4) * inv_c;
        np = block_sum(np, s4) * inv_c;
      }
      // all that a thread reads of a channel before what it writes there: outputs may lie on inputs
      for (int c = threadIdx.x; c < C; c += kT) {
        const float G = row[c], sc = at_or(w.scale, c, 1.f), g = q ? Elt<T>::ld(q + c) : 1.f;
        float fh = Elt<T>::ld(f + p * ldf + c), v = G * sc * g, n = fh;
        if (post) {
          const float pg = at_or(w.post_gain, c, 1.f);
          fh = (fh - st.x) * st.y;
          n = pg * fh + at_or(w.post_bias, c, 0.f);
          v = st.y * (v * pg - ns - fh * np);
        }
        if (group == 1) {
          S1[c] += g * G * fh;
          S2[c] += g * G;
          if (dgate) Elt<T>::st(dgate + p * lddgate + c, sc * G * n);
        } else {
          U1[c] += G * fh;
          U2[c] += G;
        }
        Elt<T>::st(dr + p * lddr + c, G);
        Elt<T>::st(df + p * lddf + c, v);
      }
    }
    for (int c = threadIdx.x; c < C && group > 1; c += kT) {
      const float g = q ? Elt<T>::ld(q + c) : 1.f;
      S1[c] += g * U1[c];
      S2[c] += g * U2[c];
      if (dgate) {
        const float n = post ? at_or(w.post_gain, c, 1.f) * U1[c] + at_or(w.post_bias, c, 0.f) * U2[c] : U1[c];
        Elt<T>::st(dgate + u * lddgate + c, at_or(w.scale, c, 1.f) * n);
      }
    }
  }
}

// The vectors' gradients from the partial sums of S blocks, `stride` sums of C a
// block: sixteen columns a block, sixteen threads a column.
__global__ __launch_bounds__(256) void res_sums(const float* part, int S, int stride, Vectors w, int post,
                                                tgp_residual_grads g, int overwrite, int C) {
  __shared__ float sh[4][16][17];
  const int l = threadIdx.x & 15, k = threadIdx.x >> 4, c = blockIdx.x * 16 + l;
  float s[4] = {};
  if (c < C)
    for (int b = k; b < S; b += 16)
#pragma unroll
      for (int z = 0; z < 4; ++z) s[z] += part[((long)b * stride + z) * C + c];
#pragma unroll
  for (int z = 0; z < 4; ++z) sh[z][k][l] = s[z];
  __syncthreads();
  if (k || c >= C) return;
#pragma unroll
  for (int z = 0; z < 4; ++z)
    for (int i = 1; i < 16; ++i) s[z] += sh[z][i][l];
  auto put = [&](float* p, float v) {
    if (p) p[c] = overwrite ? v : p[c] + v;
  };
  const float sc = at_or(w.scale, c, 1.f);
  put(g.pre_gain, s[0]);
  put(g.pre_bias, s[1]);
  put(g.post_gain, sc * s[2]);
  put(g.post_bias, sc * s[3]);
  put(g.scale, post ? at_or(w.post_gain, c, 1.f) * s[2] + at_or(w.post_bias, c, 0.f) * s[3] : s[2]);
}

Vectors vectors(const tgp_residual_params& p) {
  return {p.scale, p.post_gain, p.post_bias, p.pre_gain, p.pre_bias};
}

constexpr int kAnyBlocks = 512;

bool any_sum(const tgp_residual_grads& g) {
  return g.scale || g.post_gain || g.post_bias || g.pre_gain || g.pre_bias;
}

template <typename T>
hipError_t forward_t(const ResidualForward& a, hipStream_t st) {
  const double n = (double)a.s.rows * a.s.C;
  ProfScope ps("residual_norm_fwd_any", 20 * n, 4 * n * sizeof(T), st);
  TGP_LAUNCH(ps, res_fwd_any<T>, dim3((unsigned)std::min<long>(a.s.rows, 2048)), dim3(kT),
             a.s.C * sizeof(float), st, (const T*)a.r.p, a.r.ld, (const T*)a.f.p, a.f.ld, (const T*)a.gate.p,
             a.gate.ld, (long)a.s.group, vectors(a.w), a.s.eps, a.s.post, (T*)a.out.p, a.out.ld, (T*)a.z.p, a.z.ld,
             (float4*)a.stats, (long)a.s.rows, a.s.C);
  return launch_status();
}

template <typename T>
hipError_t backward_t(const ResidualBackward& a, hipStream_t st) {
  const double n = (double)a.s.rows * a.s.C;
  const long group = a.gate.p ? (long)a.s.group : 1;
  const int S = (int)std::min<long>(kAnyBlocks, a.s.rows / group);
  {
    ProfScope ps("residual_norm_bwd_any", 40 * n, 6 * n * sizeof(T), st);
    TGP_LAUNCH(ps, res_bwd_any<T>, dim3(S), dim3(kT), a.s.C * sizeof(float), st, (const T*)a.dz.p, a.dz.ld,
               (const T*)a.dout.p, a.dout.ld, (const T*)a.out.p, a.out.ld, (const T*)a.f.p, a.f.ld,
               (const T*)a.gate.p, a.gate.ld, group, vectors(a.w), a.s.post, (const float4*)a.stats, (T*)a.dr.p,
               a.dr.ld, (T*)a.df.p, a.df.ld, (T*)a.dgate.p, a.dgate.ld, a.part, (long)a.s.rows, a.s.C);
  }
  if (any_sum(a.g)) {
    ProfScope ps("residual_norm_sums", 4.0 * S * a.s.C, 16.0 * S * a.s.C, st);
    TGP_LAUNCH(ps, res_sums, dim3(cdiv(a.s.C, 16)), dim3(256), 0, st, a.part, S, 6, vectors(a.w), a.s.post, a.g,
               (int)a.overwrite, a.s.C);
  }
  return launch_status();
}

}  // namespace

hipError_t residual_norm_forward(const ResidualForward& a, hipStream_t st) {
  return a.s.dtype == TGP_BF16 ? forward_t<bf16_t>(a, st) : forward_t<float>(a, st);
}

size_t residual_norm_partial_floats(const tgp_residual_shape& s) {
  return 6 * (size_t)std::min<long>(kAnyBlocks, s.rows) * s.C;
}

hipError_t residual_norm_backward(const ResidualBackward& a, hipStream_t st) {
  if (a.s.rows == 0) {
    if (!any_sum(a.g) || !a.overwrite) return hipSuccess;
    ProfScope ps("residual_norm_zero", 0, 20.0 * a.s.C, st);
    TGP_LAUNCH(ps, res_sums, dim3(cdiv(a.s.C, 16)), dim3(256), 0, st, nullptr, 0, 4, Vectors{}, 0, a.g, 1, a.s.C);
    return launch_status();
  }
  return a.s.dtype == TGP_BF16 ? backward_t<bf16_t>(a, st) : backward_t<float>(a, st);
}

}  // namespace tgpk
