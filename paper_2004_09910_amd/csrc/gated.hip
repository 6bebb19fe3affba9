// A gated feed-forward block over the channels of each pixel, forward and
// backward: y = (act(x Wg^T + bg) * (x Wu^T + bu)) Wd^T + bd.
//
// Forward: one launch has both projections of a tile of hidden channels in
// registers and leaves h = act(g) u; a second multiplies it by Wd^T.
// Backward, from x and dy: one launch has g, u and dh = dy Wd of a tile and leaves
// h, dg = dh u act'(g) and du = dh act(g); one takes dx = dg Wg + du Wu as one sum
// over twice the hidden channels; one takes the three weight gradients, sums over
// pixels, in ranges whose partial tiles the last adds up in order, together
// with the column sums of dg, du and dy (a product of the left factor with ones).
//
// Matrix instructions take bfloat16.  Of a TGP_BF16 network x, dy and the weights
// are that; h, dg and du are rounded once for y and dx, which are rounded to
// bfloat16 themselves, and kept as two bfloat16s (16 bits) for the weights'
// gradients, float32 sums.  Of a TGP_FP32 network every factor is three
// bfloat16s, its 24 bits, and six of the nine products are summed, small ones
// first: what is left out is 2^-24 of a term.  A sum over split factors is one
// sum over pairs of their parts.
//
// Tensors that are not bfloat16 in 16-byte pieces are copied into the workspace
// first, split or as they are, rows padded with zeros.  Many pixels are taken some
// thousands at a time, so that what one launch leaves for the next stays in the
// caches.
#include <algorithm>
#include <utility>

#include "common.h"
#include "gemm_tile.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256;
constexpr int kMaxParts = 3;

long round_up(long v, long m) { return (v + m - 1) / m * m; }

// A matrix of bfloat16s in `parts` parts, each at a multiple of 16 bytes, rows ld
// values apart.
struct Matrix {
  bf16_t* part[kMaxParts];
  long ld;
};

// ------------------------------------------------- copies

// One matrix of a copying launch: rows x cols of T, rows lds apart, to `parts`
// bfloat16 matrices of rows of ld (a multiple of 8, zeros beyond cols).
struct CopyJob {
  const void* from;
  long lds, rows, ld, blk0;
  int cols;
  bf16_t* to[kMaxParts];
};
constexpr int kMaxCopies = 5;
struct Copies {
  CopyJob j[kMaxCopies];
  int n;
};

// Memory bounds it: eight values a thread.  A float32 is split by rounding to
// bfloat16 and rounding what is left; an infinity or NaN has no rest.
template <typename T>
__global__ __launch_bounds__(kT) void copy_k(Copies c) {
  int k = 0;
  while (k + 1 < c.n && (long)blockIdx.x >= c.j[k + 1].blk0) ++k;
  const CopyJob j = c.j[k];
  const long e = ((long)blockIdx.x - j.blk0) * kT + threadIdx.x, per = j.ld / 8;
  const long r = e / per;
  const int c0 = (int)(e - r * per) * 8;
  if (r >= j.rows) return;
  const T* from = (const T*)j.from + r * j.lds;
  float v[8];
#pragma unroll
  for (int z = 0; z < 8; ++z) v[z] = c0 + z < j.cols ? Elt<T>::ld(from + c0 + z) : 0.f;
  constexpr int P = sizeof(T) == 2 ? 1 : 3;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    unsigned w[4];
#pragma unroll
    for (int z = 0; z < 4; ++z) w[z] = f2bf(v[2 * z]) | f2bf(v[2 * z + 1]) << 16;
    *(u32x4*)(j.to[p] + r * j.ld + c0) = u32x4{w[0], w[1], w[2], w[3]};
    if (p + 1 < P)
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const float hi = bf2f(z & 1 ? w[z / 2] >> 16 : w[z / 2] & 0xffffu);
        v[z] = (__float_as_uint(hi) & 0x7f800000u) == 0x7f800000u ? 0.f : v[z] - hi;
      }
  }
}

// ------------------------------------------------- hidden channels

// act(g) and act'(g), to float32's accuracy.  GELU's Phi(g) = (1 + erf(g / sqrt 2)) /
// 2 is by the rational approximation 7.1.26 of Abramowitz and Stegun's Handbook
// (1.5e-7), whose exponential act' has as well.
template <int ACT>
__device__ __forceinline__ void act_of(float g, float* a, float* slope) {
  if constexpr (ACT == TGP_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f));
    *a = g * p;
    *slope = p + *a * (1.f - p);
  } else {
    const float e = __builtin_amdgcn_exp2f(g * g * -0.72134752f);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678f * fabsf(g));
    const float q =
        0.5f * e * t *
        (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float p = g < 0.f ? q : 1.f - q;
    *a = g * p;
    *slope = p + g * e * 0.39894228f;
  }
}

// Sixteen values of a lane's fragment (columns 8 (v / 4) + 4 (l / 32) + v % 4 of row l %
// 32) as P parts to m's rows r and columns from c on.
template <int P>
__device__ __forceinline__ void put_parts(const Matrix& m, long r, int c, bool in, int cols, float (&v)[16]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    unsigned pk[8];
#pragma unroll
    for (int z = 0; z < 8; ++z) pk[z] = pack_bf16(v[2 * z], v[2 * z + 1]);
    put8(pk, [&](int h, u32x4 u) {
      const int at = c + 16 * h + 8 * (lane >> 5);
      if (in && at < cols) *(u32x4*)(m.part[p] + r * m.ld + at) = u;
    });
    if (p + 1 < P)
#pragma unroll
      for (int z = 0; z < 16; ++z) {
        const float hi = z & 1 ? __uint_as_float(pk[z / 2] & 0xffff0000u) : __uint_as_float(pk[z / 2] << 16);
        v[z] = (__float_as_uint(hi) & 0x7f800000u) == 0x7f800000u ? 0.f : v[z] - hi;
      }
  }
}

struct HiddenArgs {
  Segs<2> s;           // x and (Wg, Wu)
  Segs<1> d;           // (backward) dy and Wd
  long lda, ldb, lddy, ldwd;
  int rows, cin, hidden, cout, ldh;
  const float *bg, *bu;
  Matrix h, dg, du;
  int tm, tn;
};

// The lane's sixteen biases of a fragment from column c on.
__device__ __forceinline__ void biases(const float* b, int c, int n, float (&v)[16]) {
  const int c0 = c + 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
  for (int z = 0; z < 16; ++z) {
    const int at = c0 + 8 * (z / 4) + z % 4;
    v[z] = b && at < n ? b[at] : 0.f;
  }
}

// h of a tile.  P: parts of a factor.
template <typename PR, int ACT, int P>
__global__ __launch_bounds__(PR::T, 2) void hidden_k(HiddenArgs a) {
  __shared__ __align__(1024) unsigned char ring[PR::LDS];
  int ti, tj;
  tile_of(xcd_remap(blockIdx.x, gridDim.x), a.tm, a.tn, &ti, &tj);
  const int i0 = ti * PR::BM, j0 = tj * PR::BN, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  PR p;
  p.zero();
  p.run(ring, a.s, a.lda, a.ldb, a.rows, a.hidden, i0, j0, 0, a.cin, [](u32x4, int, int) {});
#pragma unroll
  for (int j = 0; j < PR::NT; ++j) {
    const int c = j0 + (wave % PR::WN * PR::NT + j) * 32;
#pragma unroll
    for (int i = 0; i < PR::MT; ++i) {
      float bg[16], bu[16];
      biases(a.bg, c, a.hidden, bg);
      biases(a.bu, c, a.hidden, bu);
      const long r = i0 + (wave / PR::WN * PR::MT + i) * 32 + (lane & 31);
      float v[16];
#pragma unroll
      for (int z = 0; z < 16; ++z) {
        float act, slope;
        act_of<ACT>(p.acc[0][i][j][z] + bg[z], &act, &slope);
        v[z] = act * (p.acc[1][i][j][z] + bu[z]);
      }
      put_parts<P>(a.h, r, c, r < a.rows, a.ldh, v);
    }
  }
}

// h, dg and du of a tile, each in P parts (one, and no h, where no weight's gradient
// is wanted).
template <typename PR, typename PD, int ACT, int P, bool GRADS>
__global__ __launch_bounds__(PR::T, 2) void back_k(HiddenArgs a) {
  static_assert(PR::BM == PD::BM && PR::BN == PD::BN && PR::MT == PD::MT && PR::WN == PD::WN, "one tile");
  __shared__ __align__(1024) unsigned char ring[PR::LDS > PD::LDS ? PR::LDS : PD::LDS];
  int ti, tj;
  tile_of(xcd_remap(blockIdx.x, gridDim.x), a.tm, a.tn, &ti, &tj);
  const int i0 = ti * PR::BM, j0 = tj * PR::BN, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  PR p;
  PD d;
  p.zero();
  d.zero();
  p.run(ring, a.s, a.lda, a.ldb, a.rows, a.hidden, i0, j0, 0, a.cin, [](u32x4, int, int) {});
  ring_barrier();   // every wave has read the last stage
  d.run(ring, a.d, a.lddy, a.ldwd, a.rows, a.hidden, i0, j0, 0, a.cout, [](u32x4, int, int) {});
#pragma unroll
  for (int j = 0; j < PR::NT; ++j) {
    const int c = j0 + (wave % PR::WN * PR::NT + j) * 32;
#pragma unroll
    for (int i = 0; i < PR::MT; ++i) {
      float bg[16], bu[16];
      biases(a.bg, c, a.hidden, bg);
      biases(a.bu, c, a.hidden, bu);
      const long r = i0 + (wave / PR::WN * PR::MT + i) * 32 + (lane & 31);
      float h[16], dg[16], du[16];
#pragma unroll
      for (int z = 0; z < 16; ++z) {
        float act, slope;
        act_of<ACT>(p.acc[0][i][j][z] + bg[z], &act, &slope);
        const float u = p.acc[1][i][j][z] + bu[z], dh = d.acc[0][i][j][z];
        h[z] = act * u;
        dg[z] = dh * u * slope;
        du[z] = dh * act;
      }
      constexpr int Q = GRADS ? P : (P == 2 ? 1 : P);
      if constexpr (GRADS) put_parts<Q>(a.h, r, c, r < a.rows, a.ldh, h);
      put_parts<Q>(a.dg, r, c, r < a.rows, a.ldh, dg);
      put_parts<Q>(a.du, r, c, r < a.rows, a.ldh, du);
      __builtin_amdgcn_sched_barrier(0);   // one fragment's values at a time: registers
    }
  }
}

// ------------------------------------------------- y, dx

struct OutArgs {
  Segs<1> s;
  long lda, ldb;
  int rows, k, n;
  const float* bias;
  void* y;
  long ldy;
  int vec;   // 16-byte pieces of y's rows lie at multiples of 16
  int tm, tn;
};

template <typename PR, typename T>
__global__ __launch_bounds__(PR::T, 2) void out_k(OutArgs a) {
  __shared__ __align__(1024) unsigned char ring[PR::LDS];
  int ti, tj;
  tile_of(xcd_remap(blockIdx.x, gridDim.x), a.tm, a.tn, &ti, &tj);
  const int i0 = ti * PR::BM, j0 = tj * PR::BN, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  PR p;
  p.zero();
  p.run(ring, a.s, a.lda, a.ldb, a.rows, a.n, i0, j0, 0, a.k, [](u32x4, int, int) {});
#pragma unroll
  for (int j = 0; j < PR::NT; ++j) {
    const int c = j0 + (wave % PR::WN * PR::NT + j) * 32;
    float b[16];
    biases(a.bias, c, a.n, b);
#pragma unroll
    for (int i = 0; i < PR::MT; ++i) {
      const long r = i0 + (wave / PR::WN * PR::MT + i) * 32 + (lane & 31);
      T* y = (T*)a.y + r * a.ldy;
      float v[16];
#pragma unroll
      for (int z = 0; z < 16; ++z) v[z] = p.acc[0][i][j][z] + b[z];
      if constexpr (sizeof(T) == 2) {
        unsigned pk[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) pk[z] = pack_bf16(v[2 * z], v[2 * z + 1]);
        put8(pk, [&](int h, u32x4 u) {
          const int at = c + 16 * h + 8 * (lane >> 5);
          if (r >= a.rows) return;
          if (a.vec && at + 8 <= a.n) {
            *(u32x4*)(y + at) = u;
          } else {
#pragma unroll
            for (int z = 0; z < 8; ++z)
              if (at + z < a.n) y[at + z] = (bf16_t)(u[z / 2] >> (16 * (z & 1)));
          }
        });
      } else {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int at = c + 8 * g + 4 * (lane >> 5);
          if (r >= a.rows) continue;
          if (a.vec && at + 4 <= a.n) {
            *(float4*)(y + at) = make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
          } else {
#pragma unroll
            for (int z = 0; z < 4; ++z)
              if (at + z < a.n) y[at + z] = v[4 * g + z];
          }
        }
      }
    }
  }
}

// ------------------------------------------------- weights' gradients

// One matrix's gradient, a^T b over the pixels: m columns of a, n of b; partial sums
// of range q at part + q stride (rows of ldp floats), column sums of a at cols +
// q stride.
struct OuterJob {
  Segs<1> s;
  long lda, ldb;
  int m, n, ldp, tm, tn, blk0;
  int sums;   // the pairs, a bit each, whose a's go into the column sums: every part once
  float *part, *cols;
};
struct OuterArgs {
  OuterJob j[3];
  int n, rows, per;    // jobs, pixels, pixels of a range (a multiple of the stage)
  long stride;
};

template <typename PR>
__global__ __launch_bounds__(PR::T, 2) void outer_k(OuterArgs a) {
  __shared__ __align__(1024) unsigned char ring[PR::LDS];
  const int blk = xcd_remap(blockIdx.x, gridDim.x);
  int k = 0;
  while (k + 1 < a.n && blk >= a.j[k + 1].blk0) ++k;
  const OuterJob& J = a.j[k];
  const int tiles = J.tm * J.tn, t = (blk - J.blk0) % tiles, q = (blk - J.blk0) / tiles;
  const int ti = t % J.tm, tj = t / J.tm, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i0 = ti * PR::BM, j0 = tj * PR::BN, k0 = q * a.per, k1 = min(a.rows, k0 + a.per);
  PR p;
  p.zero();
  f32x16_t ones[PR::MT];
#pragma unroll
  for (int i = 0; i < PR::MT; ++i) ones[i] = f32x16_t{};
  // the waves of the first columns take the column sums
  const int sums = __builtin_amdgcn_readfirstlane(tj == 0 && wave % PR::WN == 0 ? J.sums : 0);
  const u32x4 one{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  p.run(ring, J.s, J.lda, J.ldb, J.m, J.n, i0, j0, k0, k1, [&](u32x4 f, int i, int pair) {
    if (sums >> pair & 1) ones[i] = mfma32(as_bf16x8(one), as_bf16x8(f), ones[i]);
  });
#pragma unroll
  for (int i = 0; i < PR::MT; ++i) {
    const int r = i0 + (wave / PR::WN * PR::MT + i) * 32 + (lane & 31);
    if (r >= J.m) continue;
    if (sums && lane < 32) J.cols[q * a.stride + r] = ones[i][0];
#pragma unroll
    for (int j = 0; j < PR::NT; ++j) {
      float* to = J.part + q * a.stride + (long)r * J.ldp;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int at = j0 + (wave % PR::WN * PR::NT + j) * 32 + 8 * g + 4 * (lane >> 5);
        const f32x16_t& v = p.acc[0][i][j];
        if (at < J.ldp) *(float4*)(to + at) = make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
      }
    }
  }
}

// to (+)= the ranges' partial sums, in order.
struct SumJob {
  const float* part;
  float* to;
  int rows, n, ldp, blk0;
};
struct SumArgs {
  SumJob j[6];
  int jobs, ranges, add;
  long stride;
};

// Four columns a thread; with many ranges four waves share them (WAVES = 4).
template <int WAVES>
__global__ __launch_bounds__(256) void sum_k(SumArgs a) {
  __shared__ float4 sh[WAVES][64];
  int k = 0;
  while (k + 1 < a.jobs && (int)blockIdx.x >= a.j[k + 1].blk0) ++k;
  const SumJob j = a.j[k];
  constexpr int E = 256 / WAVES;   // pieces of a block
  const int w = WAVES == 1 ? 0 : threadIdx.x >> 6, l = threadIdx.x % E;
  const long e = (long)(blockIdx.x - j.blk0) * E + l;
  const int per = j.ldp / 4;
  const long r = e / per;
  const int c = (int)(e - r * per) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (r < j.rows) {
    const float* p = j.part + r * j.ldp + c;
#pragma unroll 4
    for (int q = w; q < a.ranges; q += WAVES) {
      const float4 v = *(const float4*)(p + q * a.stride);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  if constexpr (WAVES > 1) {
    sh[w][l] = s;
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int q = 1; q < WAVES; ++q) {
      const float4 v = sh[q][l];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  if (r >= j.rows) return;
  float* to = j.to + r * j.n + c;
  const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int z = 0; z < 4; ++z)
    if (c + z < j.n) to[z] = a.add ? to[z] + v[z] : v[z];
}

__global__ void zero_k(float* p, long n) {
  const long i = (long)blockIdx.x * kT + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

// ------------------------------------------------- plans

// Large and small tiles of each launch.
typedef Product<2, 2, 2, 2, 32, 3, false, false, 2> HidL;
typedef Product<1, 1, 2, 2, 64, 3, false, false, 2> HidS;
typedef Product<2, 2, 2, 2, 32, 3, false, true, 1> DhL;
typedef Product<1, 1, 2, 2, 64, 3, false, true, 1> DhS;
typedef Product<2, 2, 2, 2, 64, 2, false, false, 1> OutL;
typedef Product<1, 1, 2, 2, 64, 4, false, false, 1> OutS;
typedef Product<2, 2, 2, 2, 64, 2, false, true, 1> DxL;
typedef Product<1, 1, 2, 2, 64, 4, false, true, 1> DxS;
typedef Product<2, 2, 2, 2, 64, 2, true, true, 1> OuterL;
typedef Product<1, 1, 2, 2, 64, 4, true, true, 1> OuterS;

constexpr long kFill = 256;   // tiles that fill the chip

// A call's workspace and how its pixels are taken.
struct Plan {
  int parts, low;        // of a factor; of h, dg and du (backward)
  long cinp, hidp, coutp;
  long chunk;            // pixels at a time
  bool small_outer;
  int ranges, per;       // of the pixels of a chunk, at most
  long stride;           // floats of a range's partial sums
  size_t x, dy, wg, wu, wd, h, dg, du, part, bytes;   // offsets
};

int ranges_of(long rows, int per) { return (int)((rows + per - 1) / per); }

Plan plan_of(const tgp_gated_shape& s, long rows, bool backward) {
  Plan p{};
  p.parts = s.dtype == TGP_BF16 ? 1 : 3;
  p.low = s.dtype == TGP_BF16 ? 2 : 3;
  p.cinp = round_up(s.cin, 8);
  p.hidp = round_up(s.hidden, 8);
  p.coutp = round_up(s.cout, 8);
  // so many pixels that what lies between launches stays in the caches, but that
  // a launch fills the chip
  const long a_row = 2 * (backward ? 3 * p.low * p.hidp + p.parts * (p.cinp + p.coutp)
                                   : p.parts * (p.hidp + p.cinp));
  const long most = (long)128 << 20;
  p.chunk = std::min(rows, std::max<long>(4096, most / a_row / 128 * 128));
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += (n + 255) / 256 * 256;
    return here;
  };
  p.wg = take((size_t)2 * p.parts * s.hidden * p.cinp);
  p.wu = take((size_t)2 * p.parts * s.hidden * p.cinp);
  p.wd = take((size_t)2 * p.parts * s.cout * p.hidp);
  p.x = take((size_t)2 * p.parts * p.chunk * p.cinp);
  if (!backward) {
    p.h = take((size_t)2 * p.parts * p.chunk * p.hidp);
  } else {
    p.dy = take((size_t)2 * p.parts * p.chunk * p.coutp);
    p.h = take((size_t)2 * p.low * p.chunk * p.hidp);
    p.dg = take((size_t)2 * p.low * p.chunk * p.hidp);
    p.du = take((size_t)2 * p.low * p.chunk * p.hidp);
    auto tiles = [&](long t) { return 2 * cdiv(s.hidden, t) * (long)cdiv(s.cin, t) + cdiv(s.cout, t) * (long)cdiv(s.hidden, t); };
    const long large = tiles(128);
    p.small_outer = large * std::max<long>(1, p.chunk / 512) < kFill;
    const long n = p.small_outer ? tiles(64) : large;
    // ranges of four stages at least, as many as fill the chip twice
    const long want = std::max<long>(1, std::min<long>(2 * kFill / n, p.chunk / 256));
    p.per = (int)round_up((p.chunk + want - 1) / want, 64);
    p.ranges = ranges_of(p.chunk, p.per);
    p.stride = 2 * (long)s.hidden * round_up(s.cin, 4) + (long)s.cout * round_up(s.hidden, 4) +
               2 * round_up(s.hidden, 4) + round_up(s.cout, 4);
    p.part = take((size_t)4 * p.stride * p.ranges);
  }
  p.bytes = at;
  return p;
}

// p of `parts` matrices of rows x ld, one after the other from `at` on.
Matrix matrix_at(void* ws, size_t at, int parts, long rows, long ld) {
  Matrix m{};
  for (int k = 0; k < parts; ++k) m.part[k] = (bf16_t*)((char*)ws + at) + k * rows * ld;
  m.ld = ld;
  return m;
}

// What a bfloat16 tensor needs to be read where it is.
bool as_is(int dtype, const void* p, long ld, int cols) {
  return dtype == TGP_BF16 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 && ld < 1 << 22;
}

struct Call {
  const Gated& g;
  const Plan p;
  char* ws;
  hipStream_t st;
  Copies copies{};
  long copy_blocks = 0;
  double copy_bytes = 0;

  // The matrix itself, or its copy's place in the workspace, to be filled by flush().
  Matrix operand(const void* from, long ld, long rows, int cols, size_t at, long room) {
    const int dtype = g.s.dtype;
    Matrix m{};
    if (as_is(dtype, from, ld, cols)) {
      m.part[0] = (bf16_t*)from;
      m.ld = ld;
      return m;
    }
    m = matrix_at(ws, at, p.parts, room, round_up(cols, 8));
    CopyJob& j = copies.j[copies.n++];
    j = {from, ld, rows, m.ld, copy_blocks, cols, {m.part[0], m.part[1], m.part[2]}};
    copy_blocks += (rows * (m.ld / 8) + kT - 1) / kT;
    copy_bytes += (double)rows * cols * (dtype == TGP_BF16 ? 4 : 10);
    return m;
  }
  hipError_t flush() {
    if (!copies.n) return hipSuccess;
    ProfScope ps("gated_copy", 0, copy_bytes, st);
    if (g.s.dtype == TGP_BF16) TGP_LAUNCH(ps, copy_k<bf16_t>, dim3((unsigned)copy_blocks), dim3(kT), 0, st, copies);
    else TGP_LAUNCH(ps, copy_k<float>, dim3((unsigned)copy_blocks), dim3(kT), 0, st, copies);
    copies.n = 0;
    copy_blocks = 0;
    copy_bytes = 0;
    return launch_status();
  }
};

// Pairs of parts of two factors whose products are summed, small ones first; f(i, j).
template <typename F>
void pairs(int na, int nb, F f) {
  for (int d = std::min(na + nb - 2, 2); d >= 0; --d)
    for (int i = std::min(d, na - 1); i >= 0 && d - i < nb; --i) f(i, d - i);
}
void add_pairs(Segs<1>* s, const Matrix& a, int na, const Matrix& b, int nb) {
  pairs(na, nb, [&](int i, int j) {
    s->a[s->n] = a.part[i];
    s->b[s->n++][0] = b.part[j];
  });
}

bool fills(long rows, long cols) { return (long)cdiv(rows, 128) * cdiv(cols, 128) >= kFill; }

template <typename PR, typename T>
void launch_out(const char* name, OutArgs a, hipStream_t st) {
  a.tm = cdiv(a.rows, PR::BM);
  a.tn = cdiv(a.n, PR::BN);
  ProfScope ps(name, 2.0 * a.rows * a.k * a.n * a.s.n, 2.0 * a.rows * (a.k + a.n), st);
  TGP_LAUNCH(ps, (out_k<PR, T>), dim3((unsigned)a.tm * a.tn), dim3(PR::T), 0, st, a);
}

HiddenArgs hidden_args(const Call& c, const Matrix& x, const Matrix& wg, const Matrix& wu, long rows) {
  const tgp_gated_shape& s = c.g.s;
  HiddenArgs a{};
  pairs(c.p.parts, c.p.parts, [&](int i, int j) {
    a.s.a[a.s.n] = x.part[i];
    a.s.b[a.s.n][0] = wg.part[j];
    a.s.b[a.s.n++][1] = wu.part[j];
  });
  a.lda = x.ld;
  a.ldb = wg.ld;
  a.rows = (int)rows;
  a.cin = s.cin;
  a.hidden = s.hidden;
  a.cout = s.cout;
  a.ldh = (int)c.p.hidp;
  a.bg = c.g.w.b_gate;
  a.bu = c.g.w.b_up;
  return a;
}

// f(ACT as a constant)
template <typename F>
void with_act(int act, F f) {
  if (act == TGP_ACT_SILU) f(std::integral_constant<int, TGP_ACT_SILU>());
  else f(std::integral_constant<int, TGP_ACT_GELU>());
}

template <typename T>
hipError_t forward_t(const Gated& g, const T* x, long ldx, T* y, long ldy, void* ws, hipStream_t st) {
  constexpr int P = sizeof(T) == 2 ? 1 : 3;
  const tgp_gated_shape& s = g.s;
  Call c{g, plan_of(s, g.rows, false), (char*)ws, st};
  const Matrix wg = c.operand(g.w.gate, s.cin, s.hidden, s.cin, c.p.wg, s.hidden);
  const Matrix wu = c.operand(g.w.up, s.cin, s.hidden, s.cin, c.p.wu, s.hidden);
  const Matrix wd = c.operand(g.w.down, s.hidden, s.cout, s.hidden, c.p.wd, s.cout);
  const Matrix h = matrix_at(ws, c.p.h, P, c.p.chunk, c.p.hidp);
  for (long r0 = 0; r0 < g.rows; r0 += c.p.chunk) {
    const long rows = std::min(c.p.chunk, g.rows - r0);
    const Matrix xm = c.operand(x + r0 * ldx, ldx, rows, s.cin, c.p.x, c.p.chunk);
    if (hipError_t e = c.flush(); e != hipSuccess) return e;
    HiddenArgs a = hidden_args(c, xm, wg, wu, rows);
    a.h = h;
    auto hidden = [&](auto pr, auto act) {
      typedef decltype(pr) PR;
      a.tm = cdiv(rows, PR::BM);
      a.tn = cdiv(s.hidden, PR::BN);
      ProfScope ps("gated_hidden", 4.0 * rows * s.cin * s.hidden * a.s.n, 2.0 * rows * (s.cin + s.hidden), st);
      TGP_LAUNCH(ps, (hidden_k<PR, decltype(act)::value, P>), dim3((unsigned)a.tm * a.tn), dim3(PR::T), 0, st, a);
    };
    with_act(s.act, [&](auto act) {
      if (fills(rows, s.hidden)) hidden(HidL(), act);
      else hidden(HidS(), act);
    });
    OutArgs o{};
    add_pairs(&o.s, h, P, wd, P);
    o.lda = h.ld;
    o.ldb = wd.ld;
    o.rows = (int)rows;
    o.k = s.hidden;
    o.n = s.cout;
    o.bias = g.w.b_down;
    o.y = y + r0 * ldy;
    o.ldy = ldy;
    o.vec = ((uintptr_t)o.y & 15) == 0 && ldy * sizeof(T) % 16 == 0;
    if (fills(rows, s.cout)) launch_out<OutL, T>("gated_out", o, st);
    else launch_out<OutS, T>("gated_out", o, st);
  }
  return launch_status();
}

template <typename T>
hipError_t backward_t(const Gated& g, const T* dy, long lddy, const T* x, long ldx, T* dx, long lddx,
                      const tgp_gated_grads& gr, bool overwrite, void* ws, hipStream_t st) {
  constexpr int P = sizeof(T) == 2 ? 1 : 3, L = sizeof(T) == 2 ? 2 : 3;
  const tgp_gated_shape& s = g.s;
  const bool grads = gr.gate || gr.up || gr.down || gr.b_gate || gr.b_up || gr.b_down;
  Call c{g, plan_of(s, g.rows, true), (char*)ws, st};
  const Plan& p = c.p;
  const Matrix wg = c.operand(g.w.gate, s.cin, s.hidden, s.cin, p.wg, s.hidden);
  const Matrix wu = c.operand(g.w.up, s.cin, s.hidden, s.cin, p.wu, s.hidden);
  const Matrix wd = c.operand(g.w.down, s.hidden, s.cout, s.hidden, p.wd, s.cout);
  const Matrix h = matrix_at(ws, p.h, L, p.chunk, p.hidp), dg = matrix_at(ws, p.dg, L, p.chunk, p.hidp),
               du = matrix_at(ws, p.du, L, p.chunk, p.hidp);
  for (long r0 = 0; r0 < g.rows; r0 += p.chunk) {
    const long rows = std::min(p.chunk, g.rows - r0);
    const Matrix xm = c.operand(x + r0 * ldx, ldx, rows, s.cin, p.x, p.chunk);
    const Matrix dym = c.operand(dy + r0 * lddy, lddy, rows, s.cout, p.dy, p.chunk);
    if (hipError_t e = c.flush(); e != hipSuccess) return e;
    HiddenArgs a = hidden_args(c, xm, wg, wu, rows);
    add_pairs(&a.d, dym, P, wd, P);
    a.lddy = dym.ld;
    a.ldwd = wd.ld;
    a.h = h;
    a.dg = dg;
    a.du = du;
    auto back = [&](auto pr, auto pd, auto act, auto all) {
      typedef decltype(pr) PR;
      a.tm = cdiv(rows, PR::BM);
      a.tn = cdiv(s.hidden, PR::BN);
      ProfScope ps("gated_back", 2.0 * rows * (2 * s.cin + s.cout) * s.hidden * a.s.n, 2.0 * rows * (s.cin + s.cout + 6 * s.hidden), st);
      TGP_LAUNCH(ps, (back_k<PR, decltype(pd), decltype(act)::value, L, decltype(all)::value>),
                 dim3((unsigned)a.tm * a.tn), dim3(PR::T), 0, st, a);
    };
    with_act(s.act, [&](auto act) {
      if (fills(rows, s.hidden)) {
        if (grads) back(HidL(), DhL(), act, std::true_type());
        else back(HidL(), DhL(), act, std::false_type());
      } else {
        if (grads) back(HidS(), DhS(), act, std::true_type());
        else back(HidS(), DhS(), act, std::false_type());
      }
    });
    if (grads) {
      OuterArgs o{};
      SumArgs m{};
      o.rows = (int)rows;
      o.per = p.per;
      o.stride = p.stride;
      m.ranges = ranges_of(rows, p.per);
      m.stride = p.stride;
      m.add = !overwrite || r0 > 0;
      float* at = (float*)((char*)ws + p.part);
      int blocks = 0;
      const int wide = p.small_outer ? OuterS::BM : OuterL::BM;
      auto job = [&](const Matrix& u, int nu, int rows_w, const Matrix& v, int nv, int cols_w, float* w, float* b) {
        const int ldp = (int)round_up(cols_w, 4);
        if (w || b) {
          OuterJob& J = o.j[o.n++];
          add_pairs(&J.s, u, nu, v, nv);
          J.lda = u.ld;
          J.ldb = v.ld;
          J.m = rows_w;
          J.n = cols_w;
          J.ldp = ldp;
          J.tm = cdiv(rows_w, wide);
          J.tn = w ? cdiv(cols_w, wide) : 1;   // the column sums alone: the first columns
          J.blk0 = blocks;
          int bit = 0;
          pairs(nu, nv, [&](int, int k) { J.sums |= (b && k == 0) << bit++; });
          J.part = at;
          J.cols = at + (long)rows_w * ldp;
          blocks += J.tm * J.tn * m.ranges;
          if (w) m.j[m.jobs++] = {J.part, w, rows_w, cols_w, ldp, 0};
          if (b) m.j[m.jobs++] = {J.cols, b, 1, rows_w, (int)round_up(rows_w, 4), 0};
        }
        at += (long)rows_w * ldp + round_up(rows_w, 4);
      };
      job(dg, L, s.hidden, xm, P, s.cin, gr.gate, gr.b_gate);
      job(du, L, s.hidden, xm, P, s.cin, gr.up, gr.b_up);
      job(dym, P, s.cout, h, L, s.hidden, gr.down, gr.b_down);
      {
        ProfScope ps("gated_outer", 2.0 * rows * (2 * s.cin + s.cout) * s.hidden * o.j[0].s.n, 2.0 * rows * (s.cin + s.cout + 6 * s.hidden), st);
        if (p.small_outer) TGP_LAUNCH(ps, outer_k<OuterS>, dim3((unsigned)blocks), dim3(OuterS::T), 0, st, o);
        else TGP_LAUNCH(ps, outer_k<OuterL>, dim3((unsigned)blocks), dim3(OuterL::T), 0, st, o);
      }
      const bool deep = m.ranges >= 8;
      int sb = 0;
      for (int k = 0; k < m.jobs; ++k) {
        m.j[k].blk0 = sb;
        sb += cdiv((long)m.j[k].rows * (m.j[k].ldp / 4), deep ? 64 : 256);
      }
      ProfScope ps("gated_sum", 0, 4.0 * m.ranges * p.stride, st);
      if (deep) TGP_LAUNCH(ps, sum_k<4>, dim3((unsigned)sb), dim3(256), 0, st, m);
      else TGP_LAUNCH(ps, sum_k<1>, dim3((unsigned)sb), dim3(256), 0, st, m);
    }
    if (dx) {   // last: it may be written over x or dy
      OutArgs o{};
      const int nd = sizeof(T) == 2 ? 1 : 3;
      add_pairs(&o.s, dg, nd, wg, P);
      add_pairs(&o.s, du, nd, wu, P);
      o.lda = p.hidp;
      o.ldb = wg.ld;
      o.rows = (int)rows;
      o.k = s.hidden;
      o.n = s.cin;
      o.y = dx + r0 * lddx;
      o.ldy = lddx;
      o.vec = ((uintptr_t)o.y & 15) == 0 && lddx * sizeof(T) % 16 == 0;
      if (fills(rows, s.cin)) launch_out<DxL, T>("gated_dx", o, st);
      else launch_out<DxS, T>("gated_dx", o, st);
    }
  }
  return launch_status();
}

}  // namespace

size_t gated_bytes(const tgp_gated_shape& s, long rows, bool backward) { return plan_of(s, rows, backward).bytes; }

hipError_t gated_forward(const Gated& g, const void* x, long ldx, void* y, long ldy, void* ws, hipStream_t st) {
  return g.s.dtype == TGP_BF16 ? forward_t<bf16_t>(g, (const bf16_t*)x, ldx, (bf16_t*)y, ldy, ws, st)
                               : forward_t<float>(g, (const float*)x, ldx, (float*)y, ldy, ws, st);
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
      TGP_LAUNCH(ps, zero_k, dim3((unsigned)((a.second + kT - 1) / kT)), dim3(kT), 0, st, a.first, a.second);
    }
    return launch_status();
  }
  return g.s.dtype == TGP_BF16
             ? backward_t<bf16_t>(g, (const bf16_t*)dy, lddy, (const bf16_t*)x, ldx, (bf16_t*)dx, lddx, gr, overwrite,
                                  ws, st)
             : backward_t<float>(g, (const float*)dy, lddy, (const float*)x, ldx, (float*)dx, lddx, gr, overwrite, ws,
                                 st);
}

}  // namespace tgpk
