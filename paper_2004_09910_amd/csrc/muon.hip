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

constexpr int kNormBlocks = 1024;  // most partial sums of |U|^2 of a matrix
constexpr int kNormPer = 4;         // pieces of 4096 values a block of the normalisation takes
constexpr int kMaxMats = 20;       // matrices of one launch

struct Mat {
  const float* grad;
  float* mom;
  bf16_t* out;
  double* norm;        // partial sums of |U|^2
  f16 *x[2], *a, *p;   // X (mp x np, ping-pong), A and P (mp x mp)
  float *da, *dp;      // diagonals' rounding errors
  float* part;         // partial tiles of A, of `split` ranges of its sum (1: none)
  int rows, cols, m, n, mp, np, norm_blocks, split;
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

// Sum over the block's 256 threads (the same value in all of them).
__device__ __forceinline__ double block_sum(double s, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// M = mu M + G, and partial sums of U^2 (in float64: squares of float32 values
// neither overflow nor vanish).  Purely a matter of memory: 16-byte accesses,
// two of each tensor in flight a thread.
__global__ __launch_bounds__(256) void muon_momentum(Mats l, float mu, int nesterov) {
  __shared__ double sh[4];
  const int k = find(l, blockIdx.x);
  const Mat& t = l.t[k];
  const int b = blockIdx.x - l.blk0[k];
  const long N = (long)t.rows * t.cols, N4 = N / 4, step = (long)t.norm_blocks * 256;
  const float4* g4 = (const float4*)t.grad;
  float4* m4 = (float4*)t.mom;
  double s = 0;
  auto one = [&](float g, float& m) {
    float u = g;
    if (m4) {
      m = mu * m + g;
      u = nesterov ? g + mu * m : m;
    }
    s += (double)u * u;
  };
  for (long i = (long)b * 256 + threadIdx.x; i < N4; i += 2 * step) {
    const bool two = i + step < N4;
    float4 g[2], m[2];
    g[0] = g4[i];
    g[1] = two ? g4[i + step] : make_float4(0, 0, 0, 0);
    m[0] = m4 ? m4[i] : make_float4(0, 0, 0, 0);
    m[1] = m4 && two ? m4[i + step] : make_float4(0, 0, 0, 0);
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      one(g[z].x, m[z].x);
      one(g[z].y, m[z].y);
      one(g[z].z, m[z].z);
      one(g[z].w, m[z].w);
    }
    if (m4) {
      m4[i] = m[0];
      if (two) m4[i + step] = m[1];
    }
  }
  const long e = 4 * N4 + threadIdx.x;   // the last one to three values
  if (b == 0 && e < N) {
    float m = t.mom ? t.mom[e] : 0.f;
    one(t.grad[e], m);
    if (t.mom) t.mom[e] = m;
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) t.norm[b] = s;
}

// X = U / (|U| + eps) as float16, kNormPer pieces of 4096 values a block, zeros
// in the padding: a piece is 64 rows x 64 columns through LDS where the matrix
// is transposed, else 512 consecutive chunks of eight.
__global__ __launch_bounds__(256) void muon_normalize(Mats l, float mu, int nesterov, float eps) {
  __shared__ double sh[4];
  __shared__ float tile[64][65];
  const int k = find(l, blockIdx.x);
  const Mat& t = l.t[k];
  const bool flip = t.rows > t.cols;
  double s = 0;
  for (int q = threadIdx.x; q < t.norm_blocks; q += 256) s += t.norm[q];
  const double norm = sqrt(block_sum(s, sh)) + eps;
  // a zero matrix stays zero; 1 / |U| may pass float32's range, so the product
  // below is taken in float64
  const double inv = norm > 0 || norm != norm ? kSX / norm : 0.0;
  auto put = [&](int i, int j, const float* f) {
    f16x8 h;
#pragma unroll
    for (int v = 0; v < 8; ++v) h[v] = (f16)(float)(f[v] * inv);
    *(f16x8*)(t.x[0] + (long)i * t.np + j) = h;
  };
  const int b0 = (blockIdx.x - l.blk0[k]) * kNormPer;
  for (int b = b0; b < b0 + kNormPer; ++b) {
    if (flip) {
      const int nt = t.np / 64, i0 = b / nt * 64, j0 = b % nt * 64;
      float u[16];
#pragma unroll
      for (int z = 0; z < 16; ++z) {
        const int r = j0 + z * 4 + (threadIdx.x >> 6), c = i0 + (threadIdx.x & 63);
        u[z] = r < t.rows && c < t.cols ? update_of(t, (long)r * t.cols + c, mu, nesterov) : 0.f;
      }
      __syncthreads();   // the previous piece has been read
#pragma unroll
      for (int z = 0; z < 16; ++z) tile[z * 4 + (threadIdx.x >> 6)][threadIdx.x & 63] = u[z];
      __syncthreads();
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int i = (z * 256 + threadIdx.x) / 8, j = threadIdx.x % 8 * 8;
        float f[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) f[v] = tile[j + v][i];
        put(i0 + i, j0 + j, f);
      }
      continue;
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int e = (b * 512 + z * 256 + threadIdx.x) * 8, i = e / t.np, j = e - i * t.np;
      const long at = (long)i * t.cols + j;
      float u[8];
      if (i < t.rows && j + 8 <= t.cols && t.cols % 4 == 0) {
        const float4 g0 = *(const float4*)(t.grad + at), g1 = *(const float4*)(t.grad + at + 4);
        const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
        if (t.mom) {
          const float4 m0 = *(const float4*)(t.mom + at), m1 = *(const float4*)(t.mom + at + 4);
          const float m[8] = {m0.x, m0.y, m0.z, m0.w, m1.x, m1.y, m1.z, m1.w};
#pragma unroll
          for (int v = 0; v < 8; ++v) u[v] = nesterov ? g[v] + mu * m[v] : m[v];
        } else {
#pragma unroll
          for (int v = 0; v < 8; ++v) u[v] = g[v];
        }
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v)
          u[v] = i < t.rows && j + v < t.cols ? update_of(t, at + v, mu, nesterov) : 0.f;
      }
      put(i, j, u);
    }
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

__device__ __forceinline__ f32x4_t from_f16(const f16* p) {
  typedef f16 f16x4 __attribute__((ext_vector_type(4)));
  return __builtin_convertvector(*(const f16x4*)p, f32x4_t);
}

// Stores one 32 x 32 fragment of a symmetric matrix at rows i0, columns j0,
// and its mirror image where the tile is off the diagonal.  value(g, i, j) is
// what elements 4 g .. 4 g + 3 (rows i .. i + 3, column j) become.
template <typename F>
__device__ __forceinline__ void store_sym(f16* m, float* d, int mp, int i0, int j0, bool mirror, F value) {
  const int lane = threadIdx.x & 63, j = j0 + (lane & 31);
  unsigned pk[8];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int i = i0 + 8 * g + 4 * (lane >> 5);
    const f32x4_t f = value(g, i, j);
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const f16 h = (f16)(f[z] * kSM);
      if (i + z == j) d[j] = f[z] - (float)h * (1.f / kSM);
      if (mirror) m[(long)(i + z) * mp + j] = h;
    }
    pk[2 * g] = pack_f16(f[0] * kSM, f[1] * kSM);
    pk[2 * g + 1] = pack_f16(f[2] * kSM, f[3] * kSM);
  }
  put8(pk, [&](int h, u32x4 c) { *(u32x4*)(m + (long)j * mp + i0 + 16 * h + 8 * (lane >> 5)) = c; });
}

__device__ __forceinline__ f32x4_t part_of(const f32x16& a, int g) {
  return f32x4_t{a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]};
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

enum { GRAM, POLY };

// Symmetric products, upper tiles only: A = X X^T (GRAM) or P = a I + b A + c
// A A (POLY).  Where GRAM's sum is split, its ranges' partial tiles go to
// t.part as the accumulators lie, [range][tile][wave][fragment][g][lane].
template <int MODE, int MT, int WM, int NS>
__global__ __launch_bounds__(64 * WM * WM) void muon_sym(Mats l, int from) {
  typedef Tile<MT, MT, WM, WM, NS, false, false> TL;
  __shared__ __attribute__((aligned(16))) unsigned char ring[NS * TL::SB];
  const int blk = xcd_remap(blockIdx.x, gridDim.x);
  const int k = find(l, blk);
  const Mat& t = l.t[k];
  const int nt = t.mp / TL::BM, tiles = nt * (nt + 1) / 2;
  const int b = blk - l.blk0[k], sp = MODE == GRAM ? b / tiles : 0, tile = b - sp * tiles;
  int ti, tj;
  upper(tile, nt, ti, tj);
  const int i0 = ti * TL::BM, j0 = tj * TL::BM, K = MODE == GRAM ? t.np : t.mp, nk = K / 64;
  const int k0 = MODE == GRAM ? (int)((long)nk * sp / t.split) : 0;
  const int k1 = MODE == GRAM ? (int)((long)nk * (sp + 1) / t.split) : nk;
  const f16* src = MODE == GRAM ? t.x[from] : t.a;
  TL tl;
  tl.run(ring, src + (long)i0 * K, K, src + (long)j0 * K, K, k0, k1);
  const int wave = threadIdx.x >> 6, wi = i0 + wave / WM * MT * 32, wj = j0 + wave % WM * MT * 32;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const f32x16& acc = tl.acc[i][j];
      if constexpr (MODE == GRAM) {
        if (t.split > 1) {
          f32x4_t* out = (f32x4_t*)t.part +
                         ((((long)b * WM * WM + wave) * MT + i) * MT + j) * 256 + (threadIdx.x & 63);
#pragma unroll
          for (int g = 0; g < 4; ++g) out[64 * g] = part_of(acc, g);
        } else {
          store_sym(t.a, t.da, t.mp, wi + 32 * i, wj + 32 * j, ti != tj,
                    [&](int g, int, int) { return part_of(acc, g) * (1.f / (kSX * kSX)); });
        }
      } else {
        store_sym(t.p, t.dp, t.mp, wi + 32 * i, wj + 32 * j, ti != tj, [&](int g, int r, int c) {
          const f32x4_t a = from_f16(t.a + (long)c * t.mp + r) * (1.f / kSM);   // A is symmetric
          const f32x4_t dr = *(const f32x4_t*)(t.da + r);
          const float dc = t.da[c];
          f32x4_t p = kC * (part_of(acc, g) * (1.f / (kSM * kSM)) + a * (dr + dc)) + kB * a;
#pragma unroll
          for (int z = 0; z < 4; ++z)
            if (r + z == c) p[z] += kA + kB * dc;
          return p;
        });
      }
    }
}

// A from the ranges' partial tiles, added in order: a wave takes one fragment.
template <int MT, int WM>
__global__ __launch_bounds__(256) void muon_gram_sum(Mats l) {
  const int k = find(l, blockIdx.x);
  const Mat& t = l.t[k];
  constexpr int BM = 32 * MT * WM, FR = WM * WM * MT * MT;
  const int nt = t.mp / BM, tiles = nt * (nt + 1) / 2;
  const int f = (blockIdx.x - l.blk0[k]) * 4 + (threadIdx.x >> 6), tile = f / FR, q = f % FR;
  const int lane = threadIdx.x & 63, wave = q / (MT * MT), i = q / MT % MT, j = q % MT;
  int ti, tj;
  upper(tile, nt, ti, tj);
  const f32x4_t* in = (const f32x4_t*)t.part + ((long)tile * FR + q) * 256 + lane;
  const long step = (long)tiles * FR * 256;
  f32x4_t acc[4] = {};
  for (int s = 0; s < t.split; ++s)
#pragma unroll
    for (int g = 0; g < 4; ++g) acc[g] += in[s * step + 64 * g];
  store_sym(t.a, t.da, t.mp, ti * BM + (wave / WM * MT + i) * 32, tj * BM + (wave % WM * MT + j) * 32,
            ti != tj, [&](int g, int, int) { return acc[g] * (1.f / (kSX * kSX)); });
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
        const f32x4_t xv = from_f16(x + (long)r * t.np + c);
#pragma unroll
        for (int z = 0; z < 4; ++z) y[4 * g + z] = acc[4 * g + z] * (1.f / (kSM * kSX)) + d * xv[z];
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
constexpr int kGramBlocks = 512;
int uppers(int nt) { return nt * (nt + 1) / 2; }

// Describes n (at most kMaxMats) matrices laid out from byte `at` of the
// workspace ws on; returns their end.  The sums of A = X X^T are split where
// the launch has too few tiles to fill the chip: into ranges of about one
// length over all matrices, for kGramBlocks blocks, of 512 values at least.
size_t lay_out(int n, const tgp_muon_tensor* d, char* ws, size_t at, Mats& l) {
  auto take = [&](size_t bytes) {
    char* p = ws + at;
    at += al256(bytes);
    return p;
  };
  l.count = n;
  long work = 0;
  for (int k = 0; k < n; ++k) {
    Mat& t = l.t[k];
    t.grad = d[k].grad;
    t.mom = d[k].momentum;
    t.out = (bf16_t*)d[k].update;
    t.rows = d[k].rows;
    t.cols = d[k].cols;
    t.m = std::min(t.rows, t.cols);
    t.n = std::max(t.rows, t.cols);
    t.mp = up(t.m);
    t.np = up(t.n);
    t.norm_blocks = (int)std::min<long>(kNormBlocks, cdiv((long)t.rows * t.cols, 4096));
    t.norm = (double*)take(kNormBlocks * sizeof(double));
    for (int z = 0; z < 2; ++z) t.x[z] = (f16*)take((size_t)t.mp * t.np * 2);
    t.a = (f16*)take((size_t)t.mp * t.mp * 2);
    t.p = (f16*)take((size_t)t.mp * t.mp * 2);
    t.da = (float*)take((size_t)t.mp * 4);
    t.dp = (float*)take((size_t)t.mp * 4);
    work += (long)uppers(t.mp / kTile) * (t.np / 64);
  }
  const long range = std::max<long>(8, (work + kGramBlocks - 1) / kGramBlocks);
  for (int k = 0; k < n; ++k) {
    Mat& t = l.t[k];
    t.split = (int)((t.np / 64 + range - 1) / range);
    t.part = nullptr;
    if (t.split > 1)
      t.part = (float*)take((size_t)t.split * uppers(t.mp / kTile) * kTile * kTile * sizeof(float));
  }
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
    const unsigned g = deal(l, [](const Mat& t) { return (t.mp / 64) * (t.np / 64) / kNormPer; });
    ProfScope ps("muon_normalize", 2 * n, 10 * n, st);
    TGP_LAUNCH(ps, muon_normalize, dim3(g), dim3(256), 0, st, l, mu, (int)nesterov, eps);
  }
  Mats lp = l, lsum = l, la = l;   // the same matrices, blocks dealt for each product
  const unsigned gg = deal(l, [](const Mat& t) { return uppers(t.mp / kTile) * t.split; });
  const unsigned gsum = deal(lsum, [](const Mat& t) {
    return t.split > 1 ? uppers(t.mp / kTile) * (kTile / 32) * (kTile / 32) / 4 : 0;
  });
  const unsigned gp = deal(lp, [](const Mat& t) { return uppers(t.mp / 64); });
  const unsigned ga = deal(la, [](const Mat& t) { return (t.mp / kTile) * (t.np / kTile); });
  for (int s = 0; s < steps; ++s) {
    {
      ProfScope ps("muon_gram", gram / 2, 2 * n + 2 * cells, st);
      TGP_LAUNCH(ps, (muon_sym<GRAM, 2, 2, 2>), dim3(gg), dim3(256), 0, st, l, s & 1);
    }
    if (gsum) {
      ProfScope ps("muon_gram_sum", 0, 4.0 * gsum * 4096, st);
      TGP_LAUNCH(ps, (muon_gram_sum<2, 2>), dim3(gsum), dim3(256), 0, st, lsum);
    }
    {
      ProfScope ps("muon_poly", poly / 2, 4 * cells, st);
      TGP_LAUNCH(ps, (muon_sym<POLY, 1, 2, 4>), dim3(gp), dim3(256), 0, st, lp, s & 1);
    }
    ProfScope ps("muon_apply", gram, 4 * n + 2 * cells, st);
    TGP_LAUNCH(ps, (muon_apply<2, 2, 2>), dim3(ga), dim3(256), 0, st, la, s & 1, (int)(s + 1 == steps));
  }
  return launch_status();
}

}  // namespace

size_t muon_bytes(int n, const tgp_muon_tensor* t) {
  size_t at = 0;
  Mats l;
  for (int k = 0; k < n; k += kMaxMats) at = lay_out(std::min(kMaxMats, n - k), t + k, nullptr, at, l);
  return at;
}

hipError_t muon_update(int n, const tgp_muon_tensor* t, float mu, bool nesterov, int steps,
                       float eps, void* ws, hipStream_t st) {
  size_t at = 0;
  for (int k = 0; k < n; k += kMaxMats) {
    Mats l;
    at = lay_out(std::min(kMaxMats, n - k), t + k, (char*)ws, at, l);
    const hipError_t e = update_list(l, mu, nesterov, steps, eps, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace tgpk
