// Orthogonalised updates of weight matrices: momentum, then Newton-Schulz
// products that bring the singular values of X near one.
//
// With m the shorter and n the longer side of a matrix, X is held m x n (a
// matrix of more rows than columns transposed), in float16 at a fixed scale,
// padded with zeros to multiples of 128.  One step is
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
#include "mfma_util.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

typedef _Float16 f16;
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef f32x16_t f32x16;

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

// ------------------------------------------------- products

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b),
                                                c, 0, 0, 0);
}

// The tile product of a block: WM x WN waves, each MT x NT fragments of 32 x
// 32, over stages of 64 sum values in a ring of NS LDS slots.  L is a panel
// of BM rows, R of BN rows, both contiguous in the sum (128-byte LDS rows,
// 16-byte chunks XOR-swizzled); with TR, R's panel is 64 sum rows of BN
// columns and its fragments are gathered by transpose loads.  With SWAP the
// accumulators hold the transposed tile: a lane has column (row with SWAP)
// l % 32 of a fragment and rows (columns) 8 (v / 4) + 4 (l / 32) + v % 4.
template <int MT, int NT, int WM, int WN, int NS, bool TR, bool SWAP>
struct Tile {
  static constexpr int NW = WM * WN, BM = 32 * MT * WM, BN = 32 * NT * WN;
  static constexpr int LCH = BM / 8, RCH = BN / 8, CH = LCH + RCH;   // 1 KiB DMA chunks of a stage
  static constexpr int SB = CH * 1024, PER = CH / NW;
  static constexpr int RROW = 2 * BN, RPI = 1024 / RROW;             // (TR) bytes of a sum row, rows of a chunk
  static_assert(LCH % NW == 0 && RCH % NW == 0 && NS * SB <= 160 * 1024, "whole DMA rounds, LDS ring");

  f32x16 acc[MT][NT];

  __device__ __forceinline__ static int rswz(int row) { return 2 * (row & 3); }

  // L: first row of the panel (ldl values a row); R: likewise, or (TR) row 0
  // at the panel's first column (ldr values a row); stages k0 .. k1 of the sum.
  __device__ __forceinline__ void run(unsigned char* ring, const f16* L, int ldl, const f16* R, int ldr,
                                      int k0, int k1) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const u32x4 rl = make_rsrc(L, 0x7fffffff), rr = make_rsrc(R, 0x7fffffff);
    int lo[LCH / NW], ro[RCH / NW];
#pragma unroll
    for (int u = 0; u < LCH / NW; ++u) {
      const int row = (NW * u + wave) * 8 + (lane >> 3);
      lo[u] = (row * ldl + 8 * swz(row, lane & 7)) * 2;
    }
#pragma unroll
    for (int u = 0; u < RCH / NW; ++u) {
      const int c = NW * u + wave;
      if constexpr (TR) {
        const int row = c * RPI + lane / (64 / RPI);
        ro[u] = (row * ldr + 8 * ((lane % (64 / RPI)) ^ rswz(row))) * 2;
      } else {
        const int row = c * 8 + (lane >> 3);
        ro[u] = (row * ldr + 8 * swz(row, lane & 7)) * 2;
      }
    }
    auto issue = [&](int k, int slot) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < LCH / NW; ++u)
        dma16(rl, TGP_LDS(ring + slot * SB + (NW * u + wave) * 1024), lo[u], k * 128);
#pragma unroll
      for (int u = 0; u < RCH / NW; ++u)
        dma16(rr, TGP_LDS(ring + slot * SB + (LCH + NW * u + wave) * 1024), ro[u],
              TR ? k * 128 * ldr : k * 128);
    };
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x16{};
    const int total = k1 - k0;
#pragma unroll
    for (int k = 0; k < NS - 1; ++k)
      if (k < total) issue(k0 + k, k);
    const int kb = 8 * (lane >> 5) + ((lane & 15) >> 2);   // (TR) row of the transpose load
    for (int idx = 0; idx < total; ++idx) {
      wait_stages<NS, PER>(min(NS - 2, total - 1 - idx));
      ring_barrier();
      if (idx + NS - 1 < total) issue(k0 + idx + NS - 1, (idx + NS - 1) % NS);
      const unsigned char* Ls = ring + (idx % NS) * SB;
      const unsigned char* Rs = Ls + LCH * 1024;
      u32x4 a[2][MT], b[2][NT];
      auto load = [&](int kk, int buf) __attribute__((always_inline)) {
        const int q = 2 * kk + (lane >> 5);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int row = (wm * MT + i) * 32 + (lane & 31);
          a[buf][i] = *(const u32x4*)(Ls + row * 128 + swz(row, q) * 16);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if constexpr (TR) {
            const int cb = ((wn * NT + j) * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
            b[buf][j] = frag_tr(Rs + (16 * kk + kb) * RROW + (((cb >> 4) ^ rswz(kb)) << 4) + (cb & 15), RROW);
          } else {
            const int row = (wn * NT + j) * 32 + (lane & 31);
            b[buf][j] = *(const u32x4*)(Rs + row * 128 + swz(row, q) * 16);
          }
        }
      };
      load(0, 0);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        if (kk + 1 < 4) load(kk + 1, (kk + 1) & 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            acc[i][j] = SWAP ? mfma(b[kk & 1][j], a[kk & 1][i], acc[i][j])
                             : mfma(a[kk & 1][i], b[kk & 1][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// Eight consecutive values of a fragment's lane as one 16-byte chunk: lanes l
// and l + 32 hold values 8 g + 0..3 and 8 g + 4..7; swapping the halves of
// groups 2 h and 2 h + 1 leaves each lane one whole group, 2 h + l / 32.
// Calls put(h, chunk) for h = 0, 1; the chunk starts at 16 h + 8 (l / 32).
template <typename F>
__device__ __forceinline__ void put8(const unsigned (&pk)[8], F put) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto s0 = __builtin_amdgcn_permlane32_swap(pk[4 * h], pk[4 * h + 2], false, false);
    const auto s1 = __builtin_amdgcn_permlane32_swap(pk[4 * h + 1], pk[4 * h + 3], false, false);
    put(h, u32x4{s0[0], s1[0], s0[1], s1[1]});
  }
}

__device__ __forceinline__ unsigned pack_f16(float a, float b) {
  typedef f16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 v = {(f16)a, (f16)b};
  return __builtin_bit_cast(unsigned, v);
}

// Stores one 32 x 32 fragment of a symmetric matrix at rows i0, columns j0
// (value(v, i, j): what element v, row i, column j, becomes, already scaled)
// and, off the diagonal tiles, its mirror image.
template <typename F>
__device__ __forceinline__ void store_sym(f16* m, float* d, int mp, int i0, int j0, bool mirror, F value) {
  const int lane = threadIdx.x & 63, j = j0 + (lane & 31);
  unsigned pk[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    float f[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int v = 2 * g + z, i = i0 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
      f[z] = value(v, i, j);
      const f16 h = (f16)(f[z] * kSM);
      if (i == j) d[i] = f[z] - (float)h * (1.f / kSM);
      if (mirror) m[(long)i * mp + j] = h;
    }
    pk[g] = pack_f16(f[0] * kSM, f[1] * kSM);
  }
  put8(pk, [&](int h, u32x4 c) { *(u32x4*)(m + (long)j * mp + i0 + 16 * h + 8 * (lane >> 5)) = c; });
}

// Row and column of tile b of the upper triangle (row <= column), row by row
// of an nt x nt grid.
__device__ __forceinline__ void upper(int b, int nt, int& r, int& c) {
  r = 0;
  while (b >= nt - r) {
    b -= nt - r;
    ++r;
  }
  c = r + b;
}

enum { GRAM, POLY, APPLY };

// Symmetric products, upper tiles only: A = X X^T (GRAM) or P = a I + b A + c
// A A (POLY).
template <int MODE, int MT, int WM, int NS>
__global__ __launch_bounds__(64 * WM * WM) void muon_sym(Mats l, int from) {
  typedef Tile<MT, MT, WM, WM, NS, false, false> TL;
  __shared__ __attribute__((aligned(16))) unsigned char ring[NS * TL::SB];
  const int blk = xcd_remap(blockIdx.x, gridDim.x);
  const int k = find(l, blk);
  const Mat& t = l.t[k];
  int ti, tj;
  upper(blk - l.blk0[k], t.mp / TL::BM, ti, tj);
  const int i0 = ti * TL::BM, j0 = tj * TL::BM, K = MODE == GRAM ? t.np : t.mp;
  const f16* src = MODE == GRAM ? t.x[from] : t.a;
  TL tl;
  tl.run(ring, src + (long)i0 * K, K, src + (long)j0 * K, K, 0, K / 64);
  const int wave = threadIdx.x >> 6, wi = i0 + wave / WM * MT * 32, wj = j0 + wave % WM * MT * 32;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const f32x16& acc = tl.acc[i][j];
      if constexpr (MODE == GRAM)
        store_sym(t.a, t.da, t.mp, wi + 32 * i, wj + 32 * j, ti != tj,
                  [&](int v, int, int) { return acc[v] * (1.f / (kSX * kSX)); });
      else
        store_sym(t.p, t.dp, t.mp, wi + 32 * i, wj + 32 * j, ti != tj, [&](int v, int r, int c) {
          const float a = (float)t.a[(long)r * t.mp + c] * (1.f / kSM);
          float p = kC * (acc[v] * (1.f / (kSM * kSM)) + a * (t.da[r] + t.da[c])) + kB * a;
          if (r == c) p += kA + kB * t.da[r];
          return p;
        });
    }
}

// X' = P X, or (last) the update itself.
template <int MT, int WM, int NS>
__global__ __launch_bounds__(64 * WM * WM) void muon_apply(Mats l, int from, int last) {
  typedef Tile<MT, MT, WM, WM, NS, true, true> TL;
  __shared__ __attribute__((aligned(16))) unsigned char ring[NS * TL::SB];
  const int blk = xcd_remap(blockIdx.x, gridDim.x);
  const int k = find(l, blk);
  const Mat& t = l.t[k];
  const int b = blk - l.blk0[k], nt = t.mp / TL::BM;
  const int i0 = b % nt * TL::BM, j0 = b / nt * TL::BN;
  const f16* x = t.x[from];
  TL tl;
  tl.run(ring, t.p + (long)i0 * t.mp, t.mp, x + j0, t.np, 0, t.mp / 64);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool flip = t.rows > t.cols, whole = !flip && t.cols % 8 == 0;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int r = i0 + (wave / WM * MT + i) * 32 + (lane & 31);
    const float d = t.dp[r] * (1.f / kSX);
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int c0 = j0 + (wave % WM * MT + j) * 32;
      const f32x16& acc = tl.acc[i][j];
      unsigned pk[8];
      float y[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = c0 + 8 * g + 4 * (lane >> 5);
        const uint2 raw = *(const uint2*)(x + (long)r * t.np + c);
        typedef f16 f16x4 __attribute__((ext_vector_type(4)));
        const f16x4 xv = __builtin_bit_cast(f16x4, raw);
#pragma unroll
        for (int z = 0; z < 4; ++z) y[4 * g + z] = acc[4 * g + z] * (1.f / (kSM * kSX)) + d * (float)xv[z];
      }
      if (!last) {
#pragma unroll
        for (int g = 0; g < 8; ++g) pk[g] = pack_f16(y[2 * g] * kSX, y[2 * g + 1] * kSX);
        f16* out = t.x[from ^ 1] + (long)r * t.np + c0;
        put8(pk, [&](int h, u32x4 c) { *(u32x4*)(out + 16 * h + 8 * (lane >> 5)) = c; });
      } else if (whole) {
#pragma unroll
        for (int g = 0; g < 8; ++g) pk[g] = f2bf(y[2 * g]) | (f2bf(y[2 * g + 1]) << 16);
        put8(pk, [&](int h, u32x4 c) {
          const int cc = c0 + 16 * h + 8 * (lane >> 5);
          if (r < t.m && cc < t.n) *(u32x4*)(t.out + (long)r * t.cols + cc) = c;
        });
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int c = c0 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
          if (r < t.m && c < t.n) t.out[flip ? (long)c * t.cols + r : (long)r * t.cols + c] = (bf16_t)f2bf(y[v]);
        }
      }
    }
  }
}

size_t al256(size_t x) { return (x + 255) & ~size_t(255); }
constexpr int kTile = 128;         // X, A and P are padded to multiples of it
int up(int x) { return (x + kTile - 1) / kTile * kTile; }
int uppers(int nt) { return nt * (nt + 1) / 2; }

// Lays out matrix t at byte `at` of the workspace ws; returns its end.
size_t lay_out(const tgp_muon_tensor& d, char* ws, size_t at, Mat& t) {
  t.grad = d.grad;
  t.mom = d.momentum;
  t.out = (bf16_t*)d.update;
  t.rows = d.rows;
  t.cols = d.cols;
  t.m = std::min(d.rows, d.cols);
  t.n = std::max(d.rows, d.cols);
  t.mp = up(t.m);
  t.np = up(t.n);
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
  const unsigned gs = deal(l, [](const Mat& t) { return uppers(t.mp / kTile); });
  Mats la = l;
  const unsigned ga = deal(la, [](const Mat& t) { return (t.mp / kTile) * (t.np / kTile); });
  for (int s = 0; s < steps; ++s) {
    {
      ProfScope ps("muon_gram", gram / 2, 2 * n + 2 * cells, st);
      TGP_LAUNCH(ps, (muon_sym<GRAM, 2, 2, 2>), dim3(gs), dim3(256), 0, st, l, s & 1);
    }
    {
      ProfScope ps("muon_poly", poly / 2, 4 * cells, st);
      TGP_LAUNCH(ps, (muon_sym<POLY, 2, 2, 2>), dim3(gs), dim3(256), 0, st, l, s & 1);
    }
    ProfScope ps("muon_apply", gram, 4 * n + 2 * cells, st);
    TGP_LAUNCH(ps, (muon_apply<2, 2, 2>), dim3(ga), dim3(256), 0, st, la, s & 1, (int)(s + 1 == steps));
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
