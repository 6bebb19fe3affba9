// Layer normalisation over the channels of each pixel (a row of an NHWC
// tensor), forward and backward.
//
// Forward: mean and rstd = (var + eps)^-1/2 of each row, the variance taken
// from the differences to the mean, y = gain (x - mean) rstd + bias.  A float32
// sum of C values around an offset is rounded at the size of the offset, and
// its mean is off by that many times the spread of a row that varies little
// (a constant row of 1000 values 12345.678 comes out 2e-3 lower, and y with
// eps = 1e-5 at half a unit in every channel): the differences' own mean is
// taken off them, and added to the mean.
// Backward: with xhat = (x - mean) rstd and g = gain dy, dx = rstd (g -
// mean(g) - xhat mean(g xhat)), and the column sums of dy xhat and dy.
// Column sums are partial sums of row ranges, left in a workspace and added
// up in a fixed order by a second launch; of few rows, blocks of their own
// take them in the same launch.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "prof.h"
#include "row_regs.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kFwdBlocks = 2048; // most blocks of a forward launch
constexpr int kColBlocks = 1024; // most row ranges of the column sums
constexpr int kColFlight = 4;    // rows in flight of a lane that sums columns

// One block a row (rows dealt out over the grid), the row read once for each
// of the mean, the variance and the result.  The mean is a float64 sum, exact
// to float32, which costs less than a reading of the differences more.  One
// value a lane and access: 2048 x 20000 bf16 105 us, 1.6 TB/s of what has to be
// read and written.  (y may be x: a thread reads a value before it writes it.)
template <typename T>
__global__ __launch_bounds__(kT) void norm_fwd_any(const T* x, long ldx,
                                                   const float* __restrict__ gain,
                                                   const float* __restrict__ bias, float eps,
                                                   T* y, long ldy, float2* __restrict__ stats,
                                                   long rows, int C) {
  __shared__ float s4[4];
  __shared__ double d4[4];
  for (long r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* xr = x + r * ldx;
    T* yr = y + r * ldy;
    double s = 0;
    for (int c = threadIdx.x; c < C; c += kT) s += Elt<T>::ld(xr + c);
    s = block_sum(s, d4) / C;
    // as a float32 and what that leaves out
    const float mean = (float)s, rest = (float)(s - mean);
    float q = 0.f;
    for (int c = threadIdx.x; c < C; c += kT) {
      const float d = Elt<T>::ld(xr + c) - mean - rest;
      q += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(q, s4) / C + eps);
    for (int c = threadIdx.x; c < C; c += kT) {
      float v = (Elt<T>::ld(xr + c) - mean - rest) * rstd;
      if (gain) v *= gain[c];
      if (bias) v += bias[c];
      Elt<T>::st(yr + c, v);
    }
    if (stats && threadIdx.x == 0) stats[r] = make_float2(mean, rstd);
  }
}

// ------------------------------------------------- rows held in registers

// Memory bounds it, and what comes between a row's loads and its stores: 147456
// x 64 bf16 take 10.2 us (3.8 TB/s of what has to be read and written; a copy of
// that size, out of the caches, 4.7 us and a launch), 0.8 of them for the
// correction of the mean, 144 x 1024 3.7.  Taking the variance beside the
// correction, as the squares' mean less the correction's square, saves nothing
// of that.  One row a lane is on its way at a time: two or four cost registers
// and waves, and come out slower (10.4 us, where one took 9.5 without the
// correction).
template <typename T, int VB, int NV, bool BLK>
__global__ __launch_bounds__(kT) void norm_fwd(const T* x, long ldx, const float* __restrict__ gain,
                                               const float* __restrict__ bias, float eps, T* y,
                                               long ldy, float2* __restrict__ stats, long rows,
                                               int C, int G) {
  typedef Vec<T, VB> VT;
  typedef Share<T, VB, NV, BLK> SH;
  constexpr int V = SH::V;
  __shared__ float s4[4];
  const SH sh(C, G, gridDim.x);
  float gn[NV][V], bs[NV][V];
  sh.channels(gain, 1.f, gn);
  sh.channels(bias, 0.f, bs);
  // the trip count is the same for every lane of the block (block_sum meets a barrier)
  for (long base = 0; base + sh.first() < rows; base += sh.step) {
    const long r = sh.row0 + base;
    typename VT::raw raw[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (r < rows && sh.has(k)) raw[k] = ((const typename VT::mem*)(x + r * ldx))[sh.vec(k)];
      else raw[k] = typename VT::raw{};
    float f[NV][V], s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      VT::un(raw[k], f[k]);
#pragma unroll
      for (int v = 0; v < V; ++v) s += f[k][v];
    }
    float mean = row_sum<BLK>(s, sh.G, s4) / C, e = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        f[k][v] -= mean;
        if (sh.has(k)) e += f[k][v];
      }
    // what the differences leave of a mean: a constant row's are all one small
    // multiple of its last place, whose sum and quotient are exact
    e = row_sum<BLK>(e, sh.G, s4) / C;
    mean += e;
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        f[k][v] -= e;
        if (sh.has(k)) q += f[k][v] * f[k][v];
      }
    const float rstd = 1.f / sqrtf(row_sum<BLK>(q, sh.G, s4) / C + eps);
    if (r < rows) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int v = 0; v < V; ++v) f[k][v] = f[k][v] * rstd * gn[k][v] + bs[k][v];
        if (sh.has(k)) ((typename VT::mem*)(y + r * ldy))[sh.vec(k)] = (typename VT::mem)VT::pk(f[k]);
      }
      if (stats && sh.l == 0) stats[r] = make_float2(mean, rstd);
    }
  }
}

// The whole column sums of four vectors of channels: 64 rows at a time, a
// vector a lane, kColFlight rows a lane in flight.
template <typename T, int VB>
__device__ __forceinline__ void norm_cols(const T* dy, long lddy, const T* x, long ldx, const float2* stats,
                                          long rows, int C, int blk, float* dgain, float* dbias, int overwrite) {
  typedef Vec<T, VB> VT;
  constexpr int V = VB / (int)sizeof(T);
  __shared__ float sums[kT / 64][2 * V][4];
  const int tid = threadIdx.x, q = blk * 4 + (tid & 3);
  const bool has = q < C / V;
  float a[V] = {}, b[V] = {};
  for (long r0 = tid >> 2; r0 < rows; r0 += kColFlight * (kT / 4)) {
    typename VT::raw rd[kColFlight], rx[kColFlight];
    float2 st[kColFlight];
#pragma unroll
    for (int z = 0; z < kColFlight; ++z) {
      const long r = r0 + z * (kT / 4);
      rd[z] = rx[z] = typename VT::raw{};
      st[z] = make_float2(0.f, 0.f);
      if (!has || r >= rows) continue;
      rd[z] = ((const typename VT::mem*)(dy + r * lddy))[q];
      rx[z] = ((const typename VT::mem*)(x + r * ldx))[q];
      st[z] = stats[r];
    }
#pragma unroll
    for (int z = 0; z < kColFlight; ++z) {
      float d[V], f[V];
      VT::un(rd[z], d);
      VT::un(rx[z], f);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        a[v] += d[v] * ((f[v] - st[z].x) * st[z].y);
        b[v] += d[v];
      }
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int o = 4; o < 64; o <<= 1) {
      a[v] += __shfl_xor(a[v], o);
      b[v] += __shfl_xor(b[v], o);
    }
    if ((tid & 63) < 4) {
      sums[tid >> 6][v][tid & 3] = a[v];
      sums[tid >> 6][V + v][tid & 3] = b[v];
    }
  }
  __syncthreads();
  if (tid >= 8 * V) return;
  const int l = tid & 3, e = tid >> 2;   // (lane, one of its 2 V sums)
  const int c = (blk * 4 + l) * V + e % V;
  if (c >= C) return;
  const float s = (sums[0][e][l] + sums[1][e][l]) + (sums[2][e][l] + sums[3][e][l]);
  float* to = (e < V ? dgain : dbias) + c;
  *to = overwrite ? s : *to + s;
}

// dx, and the column sums: those of the block's rows in part[block][2][C]
// (part NULL: none), or (DIRECT) the whole ones by the blocks after the
// row_blocks that take rows.
// Memory bounds it: 131072 x 128 bf16 take 19.8 us (5.1 TB/s) and their sums'
// launch 3.9, 12544 x 256 8.4 and 3.2.
template <typename T, int VB, int NV, bool BLK, bool DIRECT>
__global__ __launch_bounds__(kT) void norm_bwd(const T* dy, long lddy, const T* x, long ldx,
                                               const float* __restrict__ gain,
                                               const float2* __restrict__ stats, T* dx, long lddx,
                                               float* __restrict__ part, long rows, int C, int G,
                                               int row_blocks, float* dgain, float* dbias, int overwrite) {
  if (DIRECT && (int)blockIdx.x >= row_blocks) {
    norm_cols<T, VB>(dy, lddy, x, ldx, stats, rows, C, blockIdx.x - row_blocks, dgain, dbias, overwrite);
    return;
  }
  typedef Vec<T, VB> VT;
  typedef Share<T, VB, NV, BLK> SH;
  constexpr int V = SH::V;
  __shared__ float s4[4];
  const SH sh(C, G, DIRECT ? row_blocks : gridDim.x);
  float gn[NV][V], a[NV][V], b[NV][V];
  sh.channels(gain, 1.f, gn);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) a[k][v] = b[k][v] = 0.f;
  const float inv_c = 1.f / C;
  for (long base = 0; base + sh.first() < rows; base += sh.step) {
    const long r = sh.row0 + base;
    typename VT::raw rd[NV], rx[NV];
    const float2 st = r < rows ? stats[r] : make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (r < rows && sh.has(k)) {
        rd[k] = ((const typename VT::mem*)(dy + r * lddy))[sh.vec(k)];
        rx[k] = ((const typename VT::mem*)(x + r * ldx))[sh.vec(k)];
      } else {
        rd[k] = rx[k] = typename VT::raw{};
      }
    float d[NV][V], xh[NV][V], s = 0.f, p = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      VT::un(rd[k], d[k]);
      VT::un(rx[k], xh[k]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        xh[k][v] = (xh[k][v] - st.x) * st.y;
        if constexpr (!DIRECT) {
          a[k][v] += d[k][v] * xh[k][v];
          b[k][v] += d[k][v];
        }
        const float g = d[k][v] * gn[k][v];
        s += g;
        p += g * xh[k][v];
      }
    }
    if (!dx) continue;
    const float ms = row_sum<BLK>(s, sh.G, s4) * inv_c, mp = row_sum<BLK>(p, sh.G, s4) * inv_c;
    if (r < rows) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float o[V];
#pragma unroll
        for (int v = 0; v < V; ++v) o[v] = st.y * (d[k][v] * gn[k][v] - ms - xh[k][v] * mp);
        if (sh.has(k)) ((typename VT::mem*)(dx + r * lddx))[sh.vec(k)] = (typename VT::mem)VT::pk(o);
      }
    }
  }
  if (DIRECT || !part) return;
  float* out = part + (long)blockIdx.x * 2 * C;
  if constexpr (BLK) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (sh.has(k))
#pragma unroll
        for (int v = 0; v < V; ++v) {
          out[(long)sh.vec(k) * V + v] = a[k][v];
          out[C + (long)sh.vec(k) * V + v] = b[k][v];
        }
  } else {
    // the wave's rows, then the four waves' sums in order
    __shared__ float ws[3][2 * NV * V][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        for (int o = sh.G; o < 64; o <<= 1) {
          a[k][v] += __shfl_xor(a[k][v], o);
          b[k][v] += __shfl_xor(b[k][v], o);
        }
        if (wave > 0) {
          ws[wave - 1][k * V + v][lane] = a[k][v];
          ws[wave - 1][NV * V + k * V + v][lane] = b[k][v];
        }
      }
    __syncthreads();
    if (wave == 0 && lane < sh.G)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (sh.has(k))
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const int e = k * V + v, f = NV * V + e;
            out[(long)sh.vec(k) * V + v] = ((a[k][v] + ws[0][e][lane]) + ws[1][e][lane]) + ws[2][e][lane];
            out[C + (long)sh.vec(k) * V + v] = ((b[k][v] + ws[0][f][lane]) + ws[1][f][lane]) + ws[2][f][lane];
          }
  }
}

// ------------------------------------------------- any row

// One block a row, read once for the two means and once for dx: 2048 x 20000 bf16
// 76 us, 3.3 TB/s.
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
// = sum dy xhat, part[range][1] = sum dy.  2048 x 20000 bf16 42 us (3.9 TB/s), and
// 10 to add up its 64 ranges.
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
// 64 threads a sum (ranges s, s + 64, .., eight loads in flight), then a tree.
__global__ __launch_bounds__(1024) void norm_cols_sum(const float* __restrict__ part, int S, int C,
                                                      float* dgain, float* dbias, int overwrite) {
  __shared__ float sh[64][17];
  const int l = threadIdx.x & 15, k = threadIdx.x >> 4;
  const long e = (long)blockIdx.x * 16 + l, E = 2L * C;
  float s = 0.f;
  if (e < E)
    for (int q0 = k; q0 < S; q0 += 8 * 64) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = q0 + 64 * i < S ? part[(q0 + 64 * i) * E + e] : 0.f;
      s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
  sh[k][l] = s;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
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

// The plan of a register kernel: VB bytes a vector, NV vectors a lane, G lanes
// a row (0: the whole block); VB = 0 where no register kernel takes the row.
struct Plan {
  int vb, nv, g;
};

// The widest vectors that every row's start and length allow; then the lanes
// and vectors a lane that leave the fewest lanes idle, more lanes where two
// leave the same (a row's vectors then lie side by side in one access).  A
// row of more than 4 x 64 vectors takes a block, of more than 4 x 256 (16 x 256
// of 2 or 4 bytes, whose values fit in as many registers) none: 8192 x 4095 bf16
// forward 31 us, backward 77; by the kernels of any row 70 and 106.
Plan plan_of(int dt, int C, uintptr_t bits) {
  const int esz = dt == TGP_BF16 ? 2 : 4;
  bits |= (uintptr_t)C * esz;
  const int vb = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
  const int nvec = C * (long)esz / vb > 1 << 20 ? 1 << 20 : (int)(C * (long)esz / vb);
  if (nvec > (vb == 16 ? 4 : 16) * kT) return {0, 0, 0};
  if (nvec > 4 * 64) {
    const int nv = cdiv(nvec, kT);
    return {vb, nv <= 4 ? nv : nv <= 8 ? 8 : 16, 0};
  }
  Plan best{vb, 1, 64};
  int room = 1 << 30;
  for (int g = 64; g >= 1; g >>= 1) {
    const int nv = cdiv(nvec, g);
    if (nv > 4) break;
    if (nv * g < room) room = nv * g, best = {vb, nv, g};
  }
  return best;
}

// Calls f(Plan's NV, BLK as constants).
template <int VB, typename F>
void with_plan(const Plan& p, F f) {
  auto nv = [&](auto blk) {
    if constexpr (VB < 16 && decltype(blk)::value) {
      if (p.nv == 8) return f(std::integral_constant<int, 8>(), blk);
      if (p.nv == 16) return f(std::integral_constant<int, 16>(), blk);
    }
    switch (p.nv) {
      case 1: f(std::integral_constant<int, 1>(), blk); break;
      case 2: f(std::integral_constant<int, 2>(), blk); break;
      case 3: f(std::integral_constant<int, 3>(), blk); break;
      default: f(std::integral_constant<int, 4>(), blk); break;
    }
  };
  if (p.g == 0) nv(std::true_type());
  else nv(std::false_type());
}

long rows_of_block(const Plan& p) { return p.g == 0 ? 1 : 4 * (64 / p.g); }

template <typename T, int VB>
void forward_regs(const Plan& p, const NormShape& s, const T* x, long ldx, const float* gain,
                  const float* bias, float eps, T* y, long ldy, float2* stats, hipStream_t st) {
  const double n = (double)s.rows * s.C;
  const unsigned grid = even_grid(s.rows, rows_of_block(p), kFwdBlocks);
  with_plan<VB>(p, [&](auto nv, auto blk) {
    constexpr int NV = decltype(nv)::value;
    constexpr bool BLK = decltype(blk)::value;
    ProfScope ps("layer_norm_fwd", 8 * n, 2 * n * sizeof(T), st);
    TGP_LAUNCH(ps, (norm_fwd<T, VB, NV, BLK>), dim3(grid), dim3(kT), 0, st, x, ldx, gain, bias,
               eps, y, ldy, stats, s.rows, s.C, p.g);
  });
}

template <typename T, int VB>
void backward_regs(const Plan& p, bool direct, int row_blocks, int col_blocks, const NormShape& s, const T* dy,
                   long lddy, const T* x, long ldx, const float* gain, const float2* stats, T* dx,
                   long lddx, float* part, float* dgain, float* dbias, bool overwrite, hipStream_t st) {
  const double n = (double)s.rows * s.C;
  with_plan<VB>(p, [&](auto nv, auto blk) {
    constexpr int NV = decltype(nv)::value;
    constexpr bool BLK = decltype(blk)::value;
    ProfScope ps("layer_norm_bwd", 14 * n, (dx ? 3 : 2) * n * sizeof(T), st);
    if (direct)
      TGP_LAUNCH(ps, (norm_bwd<T, VB, NV, BLK, true>), dim3(row_blocks + col_blocks), dim3(kT), 0, st, dy,
                 lddy, x, ldx, gain, stats, dx, lddx, part, s.rows, s.C, p.g, row_blocks, dgain, dbias,
                 (int)overwrite);
    else
      TGP_LAUNCH(ps, (norm_bwd<T, VB, NV, BLK, false>), dim3(row_blocks), dim3(kT), 0, st, dy, lddy, x, ldx,
                 gain, stats, dx, lddx, part, s.rows, s.C, p.g, row_blocks, dgain, dbias, (int)overwrite);
  });
}

// Row ranges (partial column sums) of the backward, at most: enough to fill
// the chip; beyond that 24 rows each, so that the sums' traffic (16 bytes a
// channel and range) stays a ninth of the rows' own (12544 x 256: 11.0 us with
// 24, 11.8 with 16, 13.0 with 48).
int row_ranges(const NormShape& s) {
  return (int)std::min<long>(std::min<long>(kColBlocks, std::max<long>(256, s.rows / 24)), s.rows);
}

// Most rows whose column sums blocks of their own take, reading the rows once
// more, in the one launch.  A launch less is worth more than the reading up to
// there: 64 x 64 bf16 7.3 -> 3.8 us, 1024 x 128 7.3 -> 5.9, 1024 x 3848 21.4
// -> 12.1 (2048 x 128 7.2, 9.0).  What bounds such a block is its CU's loads of
// 64 bytes a row; eight rows in flight a lane take what four take.
constexpr long kDirectRows = 1024;

// Element size, and the bits of every address and row distance that the
// widest vector has to divide.
template <typename T>
uintptr_t place(const void* p, long ld) { return (uintptr_t)p | (uintptr_t)ld * sizeof(T); }

template <typename T>
hipError_t forward_t(const NormShape& s, const void* x, long ldx, const float* gain,
                     const float* bias, float eps, void* y, long ldy, float* stats,
                     hipStream_t st) {
  const Plan p = plan_of(sizeof(T) == 2 ? TGP_BF16 : TGP_FP32, s.C, place<T>(x, ldx) | place<T>(y, ldy));
  auto regs = [&](auto vb) {
    forward_regs<T, decltype(vb)::value>(p, s, (const T*)x, ldx, gain, bias, eps, (T*)y, ldy,
                                         (float2*)stats, st);
  };
  if (p.vb == 16) regs(std::integral_constant<int, 16>());
  else if (p.vb == 4) regs(std::integral_constant<int, 4>());
  else if (p.vb == 2) regs(std::integral_constant<int, sizeof(T) == 2 ? 2 : 4>());
  if (p.vb) return launch_status();
  const double n = (double)s.rows * s.C;
  ProfScope ps("layer_norm_fwd_any", 8 * n, 2 * n * sizeof(T), st);
  TGP_LAUNCH(ps, norm_fwd_any<T>, dim3((unsigned)std::min<long>(s.rows, 2048)), dim3(kT), 0, st,
             (const T*)x, ldx, gain, bias, eps, (T*)y, ldy, (float2*)stats, s.rows, s.C);
  return launch_status();
}

void sum_columns(int S, int C, const float* part, float* dgain, float* dbias, bool overwrite,
                 hipStream_t st) {
  ProfScope ps("layer_norm_cols_sum", 2.0 * S * C, 8.0 * S * C, st);
  TGP_LAUNCH(ps, norm_cols_sum, dim3(cdiv(2L * C, 16)), dim3(1024), 0, st, part, S, C, dgain, dbias,
             (int)overwrite);
}

template <typename T>
hipError_t backward_t(const NormShape& s, const void* dy, long lddy, const void* x, long ldx,
                      const float* gain, const float* stats, void* dx, long lddx, float* dgain,
                      float* dbias, bool overwrite, float* part, hipStream_t st) {
  const double n = (double)s.rows * s.C;
  const int most = row_ranges(s);
  const Plan p = plan_of(sizeof(T) == 2 ? TGP_BF16 : TGP_FP32, s.C,
                         place<T>(dy, lddy) | place<T>(x, ldx) | (dx ? place<T>(dx, lddx) : 0));
  if (p.vb) {
    const int S = (int)even_grid(s.rows, rows_of_block(p), most);
    // the column sums: by blocks of their own, or of the rows' blocks
    const bool direct = dgain && s.rows <= kDirectRows;
    const int cols = direct ? cdiv((long)s.C * sizeof(T), 4 * p.vb) : 0;
    auto launch = [&](int row_blocks, int col_blocks) {
      auto regs = [&](auto vb) {
        backward_regs<T, decltype(vb)::value>(p, direct, row_blocks, col_blocks, s, (const T*)dy, lddy, (const T*)x,
                                              ldx, gain, (const float2*)stats, (T*)dx, lddx,
                                              dgain && !direct ? part : nullptr, dgain, dbias, overwrite, st);
      };
      if (p.vb == 16) regs(std::integral_constant<int, 16>());
      else if (p.vb == 4) regs(std::integral_constant<int, 4>());
      else regs(std::integral_constant<int, sizeof(T) == 2 ? 2 : 4>());
    };
    if (!direct) {
      launch(S, 0);
      if (dgain) sum_columns(S, s.C, part, dgain, dbias, overwrite, st);
    } else if (dx == dy || dx == x) {   // the columns' blocks read what the rows' would write over
      launch(0, cols);
      launch(S, 0);
    } else {
      launch(dx ? S : 0, cols);
    }
    return launch_status();
  }
  if (dgain) {   // first: dx may be written over dy or x
    const int S = (int)std::min<long>(most, std::max<long>(1, s.rows / 32));
    {
      ProfScope ps("layer_norm_cols_any", 5 * n, 2 * n * sizeof(T), st);
      TGP_LAUNCH(ps, norm_cols_any<T>, dim3(cdiv(s.C, 64), S), dim3(kT), 0, st, (const T*)dy, lddy,
                 (const T*)x, ldx, (const float2*)stats, part, s.rows, s.C);
    }
    sum_columns(S, s.C, part, dgain, dbias, overwrite, st);
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
