// Layer normalisation over the channels of each pixel (a row of an NHWC
// tensor), forward and backward.
//
// Forward: mean and rstd = (var + eps)^-1/2 of each row, the variance taken
// from the differences to the mean, y = gain (x - mean) rstd + bias.
// Backward: with xhat = (x - mean) rstd and g = gain dy, dx = rstd (g -
// mean(g) - xhat mean(g xhat)), and the column sums of dy xhat and dy.
// Column sums are partial sums of row ranges, left in a workspace and added
// up in a fixed order by a second launch.
#include <algorithm>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256;          // threads of a block
constexpr int kColBlocks = 256;  // most row ranges of the column sums

// Sum over the block's kT threads, the same value in every thread: a wave's
// xor tree, then the waves' sums in order.
__device__ __forceinline__ float block_sum(float v, float* s4) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (s4[0] + s4[1]) + (s4[2] + s4[3]);
  __syncthreads();
  return v;
}

// One block a row (rows dealt out over the grid), the row read once for each
// of the mean, the variance and the result.
template <typename T>
__global__ __launch_bounds__(kT) void norm_fwd_any(const T* __restrict__ x, long ldx,
                                                   const float* __restrict__ gain,
                                                   const float* __restrict__ bias, float eps,
                                                   T* y, long ldy, float2* __restrict__ stats,
                                                   long rows, int C) {
  __shared__ float s4[4];
  for (long r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* xr = x + r * ldx;
    T* yr = y + r * ldy;
    float s = 0.f;
    for (int c = threadIdx.x; c < C; c += kT) s += Elt<T>::ld(xr + c);
    const float mean = block_sum(s, s4) / C;
    float q = 0.f;
    for (int c = threadIdx.x; c < C; c += kT) {
      const float d = Elt<T>::ld(xr + c) - mean;
      q += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(q, s4) / C + eps);
    for (int c = threadIdx.x; c < C; c += kT) {
      float v = (Elt<T>::ld(xr + c) - mean) * rstd;
      if (gain) v *= gain[c];
      if (bias) v += bias[c];
      Elt<T>::st(yr + c, v);
    }
    if (stats && threadIdx.x == 0) stats[r] = make_float2(mean, rstd);
  }
}

template <typename T>
__global__ __launch_bounds__(kT) void norm_dx_any(const T* dy, long lddy, const T* x, long ldx,
                                                  const float* __restrict__ gain,
                                                  const float2* __restrict__ stats, T* dx,
                                                  long lddx, long rows, int C) {
  __shared__ float s4[4];
  for (long r = blockIdx.x; r < rows; r += gridDim.x) {
    const T *dr = dy + r * lddy, *xr = x + r * ldx;
    const float2 st = stats[r];
    float s = 0.f, p = 0.f;
    for (int c = threadIdx.x; c < C; c += kT) {
      const float g = Elt<T>::ld(dr + c) * (gain ? gain[c] : 1.f);
      s += g;
      p += g * ((Elt<T>::ld(xr + c) - st.x) * st.y);
    }
    const float ms = block_sum(s, s4) / C, mp = block_sum(p, s4) / C;
    for (int c = threadIdx.x; c < C; c += kT) {
      const float g = Elt<T>::ld(dr + c) * (gain ? gain[c] : 1.f);
      const float xh = (Elt<T>::ld(xr + c) - st.x) * st.y;
      Elt<T>::st(dx + r * lddx + c, st.y * (g - ms - xh * mp));
    }
  }
}

// Column sums of one range of rows (blockIdx.y) for 64 channels: part[range][0]
// = sum dy xhat, part[range][1] = sum dy.
template <typename T>
__global__ __launch_bounds__(kT) void norm_cols_any(const T* __restrict__ dy, long lddy,
                                                    const T* __restrict__ x, long ldx,
                                                    const float2* __restrict__ stats,
                                                    float* __restrict__ part, long rows, int C) {
  __shared__ float sh[2][4][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  const long per = (rows + gridDim.y - 1) / gridDim.y;
  const long r0 = per * blockIdx.y, r1 = r0 + per < rows ? r0 + per : rows;
  float a = 0.f, b = 0.f;
  if (c < C)
    for (long r = r0 + w; r < r1; r += 4) {
      const float2 st = stats[r];
      const float d = Elt<T>::ld(dy + r * lddy + c);
      a += d * ((Elt<T>::ld(x + r * ldx + c) - st.x) * st.y);
      b += d;
    }
  sh[0][w][threadIdx.x & 63] = a;
  sh[1][w][threadIdx.x & 63] = b;
  __syncthreads();
  if (w < 2 && c < C) {
    const int l = threadIdx.x & 63;
    part[((long)blockIdx.y * 2 + w) * C + c] = (sh[w][0][l] + sh[w][1][l]) + (sh[w][2][l] + sh[w][3][l]);
  }
}

// dgain, dbias (+)= the sum over S ranges of part[s][2][C]: 16 sums a block,
// 32 threads a sum (ranges s, s + 32, ..), then their xor tree.
__global__ __launch_bounds__(512) void norm_cols_sum(const float* __restrict__ part, int S, int C,
                                                     float* dgain, float* dbias, int overwrite) {
  __shared__ float sh[32][17];
  const int l = threadIdx.x & 15, k = threadIdx.x >> 4;
  const long e = (long)blockIdx.x * 16 + l, E = 2L * C;
  float s = 0.f;
  if (e < E)
    for (int q = k; q < S; q += 32) s += part[q * E + e];
  sh[k][l] = s;
  __syncthreads();
  for (int o = 16; o > 0; o >>= 1) {
    if (k < o) sh[k][l] += sh[k + o][l];
    __syncthreads();
  }
  if (k == 0 && e < E) {
    float* p = e < C ? dgain + e : dbias + (e - C);
    *p = overwrite ? sh[0][l] : *p + sh[0][l];
  }
}

__global__ void norm_zero(float* a, float* b, int C) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c < C) a[c] = b[c] = 0.f;
}

int row_ranges(const NormShape& s) { return (int)std::min<long>(kColBlocks, std::max<long>(1, s.rows / 32)); }

template <typename T>
hipError_t forward_t(const NormShape& s, const void* x, long ldx, const float* gain,
                     const float* bias, float eps, void* y, long ldy, float* stats,
                     hipStream_t st) {
  const double n = (double)s.rows * s.C;
  ProfScope ps("layer_norm_fwd_any", 8 * n, 2 * n * sizeof(T), st);
  TGP_LAUNCH(ps, norm_fwd_any<T>, dim3((unsigned)std::min<long>(s.rows, 2048)), dim3(kT), 0, st,
             (const T*)x, ldx, gain, bias, eps, (T*)y, ldy, (float2*)stats, s.rows, s.C);
  return launch_status();
}

template <typename T>
hipError_t backward_t(const NormShape& s, const void* dy, long lddy, const void* x, long ldx,
                      const float* gain, const float* stats, void* dx, long lddx, float* dgain,
                      float* dbias, bool overwrite, float* part, hipStream_t st) {
  const double n = (double)s.rows * s.C;
  if (dgain) {   // first: dx may be written over dy or x
    const int S = row_ranges(s);
    {
      ProfScope ps("layer_norm_cols_any", 5 * n, 2 * n * sizeof(T), st);
      TGP_LAUNCH(ps, norm_cols_any<T>, dim3(cdiv(s.C, 64), S), dim3(kT), 0, st, (const T*)dy, lddy,
                 (const T*)x, ldx, (const float2*)stats, part, s.rows, s.C);
    }
    ProfScope ps("layer_norm_cols_sum", 2.0 * S * s.C, 8.0 * S * s.C, st);
    TGP_LAUNCH(ps, norm_cols_sum, dim3(cdiv(2L * s.C, 16)), dim3(512), 0, st, (const float*)part, S,
               s.C, dgain, dbias, (int)overwrite);
  }
  if (dx) {
    ProfScope ps("layer_norm_dx_any", 9 * n, 3 * n * sizeof(T), st);
    TGP_LAUNCH(ps, norm_dx_any<T>, dim3((unsigned)std::min<long>(s.rows, 2048)), dim3(kT), 0, st,
               (const T*)dy, lddy, (const T*)x, ldx, gain, (const float2*)stats, (T*)dx, lddx,
               s.rows, s.C);
  }
  return launch_status();
}

}  // namespace

hipError_t layer_norm_forward(int dt, const NormShape& s, const void* x, long ldx,
                              const float* gain, const float* bias, float eps, void* y, long ldy,
                              float* stats, hipStream_t st) {
  return dt == TGP_BF16 ? forward_t<bf16_t>(s, x, ldx, gain, bias, eps, y, ldy, stats, st)
                        : forward_t<float>(s, x, ldx, gain, bias, eps, y, ldy, stats, st);
}

size_t layer_norm_partial_floats(int, const NormShape& s) {
  return s.rows > 0 ? 2 * (size_t)row_ranges(s) * s.C : 0;
}

hipError_t layer_norm_backward(int dt, const NormShape& s, const void* dy, long lddy,
                               const void* x, long ldx, const float* gain, const float* stats,
                               void* dx, long lddx, float* dgain, float* dbias, bool overwrite,
                               float* part, hipStream_t st) {
  if (s.rows == 0) {
    if (!dgain || !overwrite) return hipSuccess;
    ProfScope ps("layer_norm_zero", 0, 8.0 * s.C, st);
    TGP_LAUNCH(ps, norm_zero, dim3(cdiv(s.C, 256)), dim3(256), 0, st, dgain, dbias, s.C);
    return launch_status();
  }
  return dt == TGP_BF16 ? backward_t<bf16_t>(s, dy, lddy, x, ldx, gain, stats, dx, lddx, dgain,
                                             dbias, overwrite, part, st)
                        : backward_t<float>(s, dy, lddy, x, ldx, gain, stats, dx, lddx, dgain,
                                            dbias, overwrite, part, st);
}

}  // namespace tgpk
