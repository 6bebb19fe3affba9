// Orthogonalised updates of weight matrices: momentum, then Newton-Schulz
// products that bring the singular values of X near one.
//
// With m the shorter and n the longer side of a matrix, X is held m x n (a
// matrix of more rows than columns transposed), in float16 at a fixed scale,
// padded with zeros to multiples of 64.  One step is
//
//   A = X X^T          P = a I + b A + c A A          X' = P X
//
// three launches over the tiles of all matrices.  A and P are float16 with the
// rounding error of their diagonals beside them in float32: near convergence
// A is nearly a multiple of I, whose one rounding would shift every singular
// value alike and be multiplied by b / p(1) = 7.  A product of two such
// matrices (L + dL)(R + dR), dL and dR diagonal, is taken as L R + dL R + L dR.
#include <algorithm>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

typedef _Float16 f16;
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// Scales of the stored values.  Singular values never pass 1.3, so entries of
// X and A stay under 2^12 and those of P (at most a) under 2^12; rms entries
// start at (m n)^-1/2 for X and 1 / m on A's diagonal, far above float16's
// smallest normal value at these scales.
constexpr float kSX = 2048.f, kSM = 1024.f;

constexpr int kNormBlocks = 256;   // most partial sums of |U|^2 of a matrix
constexpr int kMaxMats = 20;       // matrices of one launch

struct Mat {
  const float* grad;
  float* mom;
  bf16_t* out;
  double* norm;        // partial sums of |U|^2
  f16 *x[2], *a, *p;   // X (mp x np, ping-pong), A and P (mp x mp)
  float *da, *dp;      // diagonals' rounding errors
  int rows, cols, m, n, mp, np, norm_blocks;
};

struct Mats {
  int count;
  Mat t[kMaxMats];
  int blk0[kMaxMats + 1];   // first block of each matrix in the launch
};

__device__ __forceinline__ int find(const Mats& l, int blk) {
  int k = 0;
  while (k + 1 < l.count && blk >= l.blk0[k + 1]) ++k;
  return k;
}

__device__ __forceinline__ float update_of(const Mat& t, long i, float mu, int nesterov) {
  const float g = t.grad[i];
  if (!t.mom) return g;
  return nesterov ? g + mu * t.mom[i] : t.mom[i];
}

// M = mu M + G, and partial sums of U^2.
__global__ __launch_bounds__(256) void muon_momentum(Mats l, float mu, int nesterov) {
  __shared__ double sh[4];
  const int k = find(l, blockIdx.x);
  const Mat& t = l.t[k];
  const int b = blockIdx.x - l.blk0[k];
  const long N = (long)t.rows * t.cols;
  double s = 0;
  for (long i = (long)b * 256 + threadIdx.x; i < N; i += (long)t.norm_blocks * 256) {
    const float g = t.grad[i];
    float u = g;
    if (t.mom) {
      const float m = mu * t.mom[i] + g;
      t.mom[i] = m;
      u = nesterov ? g + mu * m : m;
    }
    s += (double)u * u;
  }
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) t.norm[b] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// X = U / (|U| + eps) as float16, a 64 x 64 tile a block, zeros in the padding.
__global__ __launch_bounds__(256) void muon_normalize(Mats l, float mu, int nesterov, float eps) {
  __shared__ double sh[256];
  __shared__ float tile[64][65];
  const int k = find(l, blockIdx.x);
  const Mat& t = l.t[k];
  const int b = blockIdx.x - l.blk0[k], nt = t.np / 64;
  const int i0 = b / nt * 64, j0 = b % nt * 64;
  sh[threadIdx.x] = (int)threadIdx.x < t.norm_blocks ? t.norm[threadIdx.x] : 0.0;
  const bool flip = t.rows > t.cols;
  const int r0 = flip ? j0 : i0, c0 = flip ? i0 : j0;
  for (int e = threadIdx.x; e < 4096; e += 256) {
    const int r = r0 + e / 64, c = c0 + e % 64;
    tile[e / 64][e % 64] = r < t.rows && c < t.cols ? update_of(t, (long)r * t.cols + c, mu, nesterov) : 0.f;
  }
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) sh[threadIdx.x] += sh[threadIdx.x + o];
    __syncthreads();
  }
  const double norm = sqrt(sh[0]) + eps;
  const float inv = norm > 0 || norm != norm ? (float)(1.0 / norm) : 0.f;
  for (int e = threadIdx.x; e < 4096; e += 256) {
    const int i = e / 64, j = e % 64;
    t.x[0][(long)(i0 + i) * t.np + j0 + j] = (f16)((flip ? tile[j][i] : tile[i][j]) * inv * kSX);
  }
}

enum { GRAM, POLY, APPLY };

// One 64 x 64 tile of C = L R a block, four waves of 32 x 32.
template <int MODE>
__global__ __launch_bounds__(256) void muon_gemm(Mats l, int from, int last) {
  constexpr int PITCH = 72;
  __shared__ __attribute__((aligned(16))) f16 ls[64 * PITCH], rs[64 * PITCH];
  const int k = find(l, blockIdx.x);
  const Mat& t = l.t[k];
  const int b = blockIdx.x - l.blk0[k], nt = (MODE == APPLY ? t.np : t.mp) / 64;
  const int i0 = b / nt * 64, j0 = b % nt * 64;
  const f16* L = MODE == GRAM ? t.x[from] : MODE == POLY ? t.a : t.p;
  const f16* R = MODE == POLY ? t.a : t.x[from];
  const int K = MODE == GRAM ? t.np : t.mp, ld = K;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wi = (w >> 1) * 32, wj = (w & 1) * 32;
  f32x16 acc = {};
  for (int k0 = 0; k0 < K; k0 += 64) {
    __syncthreads();
    for (int e = threadIdx.x; e < 512; e += 256) {
      const int r = e / 8, q = e % 8 * 8;
      *(f16x8*)(ls + r * PITCH + q) = *(const f16x8*)(L + (long)(i0 + r) * ld + k0 + q);
      if (MODE == APPLY) {
        const f16x8 v = *(const f16x8*)(R + (long)(k0 + r) * t.np + j0 + q);
        for (int z = 0; z < 8; ++z) rs[(q + z) * PITCH + r] = v[z];
      } else {
        *(f16x8*)(rs + r * PITCH + q) = *(const f16x8*)(R + (long)(j0 + r) * ld + k0 + q);
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 64; q += 16) {
      const f16x8 a = *(const f16x8*)(ls + (wi + (lane & 31)) * PITCH + q + 8 * (lane >> 5));
      const f16x8 c = *(const f16x8*)(rs + (wj + (lane & 31)) * PITCH + q + 8 * (lane >> 5));
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, c, acc, 0, 0, 0);
    }
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int i = i0 + wi + 8 * (v / 4) + 4 * (lane >> 5) + v % 4, j = j0 + wj + (lane & 31);
    if (MODE == GRAM) {
      const float a = acc[v] * (1.f / (kSX * kSX));
      const f16 h = (f16)(a * kSM);
      t.a[(long)i * t.mp + j] = h;
      if (i == j) t.da[i] = a - (float)h * (1.f / kSM);
    } else if (MODE == POLY) {
      const float a = (float)t.a[(long)i * t.mp + j] * (1.f / kSM);
      const float di = t.da[i], dj = t.da[j];
      float p = kC * (acc[v] * (1.f / (kSM * kSM)) + a * (di + dj)) + kB * a;
      if (i == j) p += kA + kB * di;
      const f16 h = (f16)(p * kSM);
      t.p[(long)i * t.mp + j] = h;
      if (i == j) t.dp[i] = p - (float)h * (1.f / kSM);
    } else {
      const float x = (float)t.x[from][(long)i * t.np + j] * (1.f / kSX);
      const float y = acc[v] * (1.f / (kSM * kSX)) + t.dp[i] * x;
      if (!last)
        t.x[from ^ 1][(long)i * t.np + j] = (f16)(y * kSX);
      else if (i < t.m && j < t.n)
        t.out[t.rows > t.cols ? (long)j * t.cols + i : (long)i * t.cols + j] = (bf16_t)f2bf(y);
    }
  }
}

size_t al256(size_t x) { return (x + 255) & ~size_t(255); }
int up64(int x) { return (x + 63) / 64 * 64; }

// Lays out matrix t at byte `at` of the workspace ws; returns its end.
size_t lay_out(const tgp_muon_tensor& d, char* ws, size_t at, Mat& t) {
  t.grad = d.grad;
  t.mom = d.momentum;
  t.out = (bf16_t*)d.update;
  t.rows = d.rows;
  t.cols = d.cols;
  t.m = std::min(d.rows, d.cols);
  t.n = std::max(d.rows, d.cols);
  t.mp = up64(t.m);
  t.np = up64(t.n);
  t.norm_blocks = (int)std::min<long>(kNormBlocks, cdiv((long)d.rows * d.cols, 1024));
  auto take = [&](size_t bytes) {
    char* p = ws + at;
    at += al256(bytes);
    return p;
  };
  t.norm = (double*)take(kNormBlocks * sizeof(double));
  for (int k = 0; k < 2; ++k) t.x[k] = (f16*)take((size_t)t.mp * t.np * 2);
  t.a = (f16*)take((size_t)t.mp * t.mp * 2);
  t.p = (f16*)take((size_t)t.mp * t.mp * 2);
  t.da = (float*)take((size_t)t.mp * 4);
  t.dp = (float*)take((size_t)t.mp * 4);
  return at;
}

// Fills blk0 with blocks(t) of each matrix; returns the grid.
template <typename F>
unsigned deal(Mats& l, F blocks) {
  int at = 0;
  for (int k = 0; k < l.count; ++k) {
    l.blk0[k] = at;
    at += blocks(l.t[k]);
  }
  l.blk0[l.count] = at;
  return (unsigned)at;
}

hipError_t update_list(Mats& l, float mu, bool nesterov, int steps, float eps, hipStream_t st) {
  double n = 0, gram = 0, poly = 0, cells = 0;
  for (int k = 0; k < l.count; ++k) {
    const Mat& t = l.t[k];
    n += (double)t.rows * t.cols;
    gram += 2.0 * t.m * t.m * t.n;
    poly += 2.0 * t.m * t.m * t.m;
    cells += (double)t.m * t.m;
  }
  {
    const unsigned g = deal(l, [](const Mat& t) { return t.norm_blocks; });
    ProfScope ps("muon_momentum", 4 * n, 12 * n, st);
    TGP_LAUNCH(ps, muon_momentum, dim3(g), dim3(256), 0, st, l, mu, (int)nesterov);
  }
  {
    const unsigned g = deal(l, [](const Mat& t) { return (t.mp / 64) * (t.np / 64); });
    ProfScope ps("muon_normalize", 2 * n, 10 * n, st);
    TGP_LAUNCH(ps, muon_normalize, dim3(g), dim3(256), 0, st, l, mu, (int)nesterov, eps);
  }
  for (int s = 0; s < steps; ++s) {
    const unsigned gm = deal(l, [](const Mat& t) { return (t.mp / 64) * (t.mp / 64); });
    {
      ProfScope ps("muon_gram", gram, 2 * n + 2 * cells, st);
      TGP_LAUNCH(ps, muon_gemm<GRAM>, dim3(gm), dim3(256), 0, st, l, s & 1, 0);
    }
    {
      ProfScope ps("muon_poly", poly, 4 * cells, st);
      TGP_LAUNCH(ps, muon_gemm<POLY>, dim3(gm), dim3(256), 0, st, l, s & 1, 0);
    }
    const unsigned ga = deal(l, [](const Mat& t) { return (t.mp / 64) * (t.np / 64); });
    ProfScope ps("muon_apply", gram, 4 * n + 2 * cells, st);
    TGP_LAUNCH(ps, muon_gemm<APPLY>, dim3(ga), dim3(256), 0, st, l, s & 1, (int)(s + 1 == steps));
  }
  return launch_status();
}

}  // namespace

size_t muon_bytes(int n, const tgp_muon_tensor* t) {
  size_t at = 0;
  Mat m;
  for (int k = 0; k < n; ++k) at = lay_out(t[k], nullptr, at, m);
  return at;
}

hipError_t muon_update(int n, const tgp_muon_tensor* t, float mu, bool nesterov, int steps,
                       float eps, void* ws, hipStream_t st) {
  size_t at = 0;
  for (int k0 = 0; k0 < n; k0 += kMaxMats) {
    Mats l;
    l.count = std::min(kMaxMats, n - k0);
    for (int k = 0; k < l.count; ++k) at = lay_out(t[k0 + k], (char*)ws, at, l.t[k]);
    const hipError_t e = update_list(l, mu, nesterov, steps, eps, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace tgpk
