// A gated feed-forward block over the channels of each pixel, forward and
// backward: y = (act(x Wg^T + bg) * (x Wu^T + bu)) Wd^T + bd.
//
// Forward: up to 256 channels (float32: 128) on both sides one launch (gated_narrow) keeps a
// tile's hidden channels in LDS; for at most 64 pixels two (gated_few) read the weights
// once, straight into registers; else one launch has both projections of a tile of
// hidden channels in registers and leaves h = act(g) u, and a second multiplies it by
// Wd^T.
// Backward, from x and dy: one launch has g, u and dh = dy Wd of a tile and leaves
// h, dg = dh u act'(g) and du = dh act(g); one takes the three weight gradients, sums
// over pixels, together with the column sums of dg, du and dy (a product of the left
// factor with ones), where the tiles are few in ranges whose partial sums another adds
// up in order; one takes dx = dg Wg + du Wu as one sum over twice the hidden channels.
// Up to 64 channels on both sides and 65 to 256 hidden ones of bfloat16 all that is one launch
// (gated_slim) and the ranges' sums.
//
// Matrix instructions take bfloat16.  Of a TGP_BF16 network x, dy and the weights
// are that.  h, dg and du are two bfloat16s each (16 bits, 2^-16 of a value) for y and
// dx, which are then rounded once, and three, their 24 bits, for the weights' gradients,
// float32 sums (two parts, a third of the products less, leave 3e-6 of a gradient's
// norm where float32 sums have 1e-7; one part 2e-3).  Of a TGP_FP32 network every factor is three
// bfloat16s, its 24 bits, and six of the nine products are summed, small ones
// first: what is left out is 2^-24 of a term.  A sum over split factors is one
// sum over pairs of their parts.
//
// Tensors that are not bfloat16 in 16-byte pieces are copied into the workspace
// first, split or as they are, rows padded with zeros.  Many pixels are taken some
// thousands at a time, so that what one launch leaves for the next stays in the
// caches.
#include <algorithm>
#include <type_traits>
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
__global__ __launch_bounds__(kT) void gated_copy(Copies c) {
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

// 2^(c v) for v the sum of `v` and `rest`, c the sum of `c` and `tail`.  FINE: to some 2^-22
// of itself; else of c v alone, whose rounding is up to 2^-24 |c v| of it.
template <bool FINE>
__device__ __forceinline__ float exp2_of(float v, float rest, float c, float tail) {
  const float y = v * c, e = __builtin_amdgcn_exp2f(y);
  if constexpr (!FINE) return e;
  const float d = fmaf(v, c, -y) + (v * tail + rest * c);
  return fabsf(y) < 126.f ? fmaf(e, d * 0.69314718f, e) : e;   // (no inf - inf)
}

// act(g) and act'(g), relative to themselves also where g is far below zero.  SiLU is g p,
// p = 1 / (1 + exp(-g)).  GELU is g Phi(g) with Phi(-|g|) = exp(-g g / 2) R(|g|) and R as
// t times a polynomial in t = 1 / (1 + 0.265 |g|), a least-squares fit of erfcx(|g| / sqrt
// 2) / 2 whose largest relative error up to |g| = 15 was brought down to 1.6e-8; in float32
// arithmetic 4e-7.  Without FINE the exponential adds 5e-8 g g of the value (2e-6 at -6):
// for y of bfloat16, whose h is two bfloat16s.
template <int ACT, bool FINE>
__device__ __forceinline__ void act_of(float g, float* a, float* slope) {
  if constexpr (ACT == TGP_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + exp2_of<FINE>(g, 0.f, -1.44269502f, -1.92596303e-8f));
    *a = g * p;
    *slope = p + *a * (1.f - p);
  } else {
    const float s = g * g, rest = FINE ? fmaf(g, g, -s) : 0.f;
    const float e = exp2_of<FINE>(s, rest, -0.72134751f, -9.62981517e-9f);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.265f, fabsf(g), 1.f));
    float r = 0.0304386261f;
    r = fmaf(r, t, -0.142422333f);
    r = fmaf(r, t, 0.214186966f);
    r = fmaf(r, t, -0.112326354f);
    r = fmaf(r, t, 0.135238826f);
    r = fmaf(r, t, 0.0614404269f);
    r = fmaf(r, t, 0.102419138f);
    r = fmaf(r, t, 0.105285376f);
    r = fmaf(r, t, 0.105739325f);
    const float q = e * t * r;
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

// h of a tile, in P parts (three where the factors have as many, else two).
template <typename PR, int ACT, int P>
__global__ __launch_bounds__(PR::T, PR::NW == 8 || PR::LDS <= 80 * 1024 ? 2 : 1) void gated_hidden(HiddenArgs a) {
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
        act_of<ACT, P == 3>(p.acc[0][i][j][z] + bg[z], &act, &slope);
        v[z] = act * (p.acc[1][i][j][z] + bu[z]);
      }
      put_parts<P>(a.h, r, c, r < a.rows, a.ldh, v);
    }
  }
}

// h, dg and du of a tile, each in P parts: three, or of bfloat16 two, and no h, where no
// weight's gradient is wanted.
template <typename PR, typename PD, int ACT, int P, bool GRADS>
__global__ __launch_bounds__(PR::T, PR::NW == 8 || PR::LDS <= 80 * 1024 ? 2 : 1) void gated_back(HiddenArgs a) {
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
        act_of<ACT, true>(p.acc[0][i][j][z] + bg[z], &act, &slope);
        const float u = p.acc[1][i][j][z] + bu[z], dh = d.acc[0][i][j][z];
        h[z] = act * u;
        dg[z] = dh * u * slope;
        du[z] = dh * act;
      }
      if constexpr (GRADS) put_parts<P>(a.h, r, c, r < a.rows, a.ldh, h);
      put_parts<P>(a.dg, r, c, r < a.rows, a.ldh, dg);
      put_parts<P>(a.du, r, c, r < a.rows, a.ldh, du);
      __builtin_amdgcn_sched_barrier(0);   // one fragment's values at a time: registers
    }
  }
}

// ------------------------------------------------- y, dx

struct OutArgs {
  Segs<1, 2> s;        // (of bfloat16 both parts of the left factor at once)
  long lda, ldb;
  int rows, k, n;
  const float* bias;
  void* y;
  long ldy;
  int vec;   // 16-byte pieces of y's rows lie at multiples of 16
  int tm, tn;
  float* part;   // the ranges' sums, rows of ldp floats
  int ldp, per;
};

// Sixteen values of a lane's fragment, with the bias, as T to row r and columns from c
// on of y.
template <typename T>
__device__ __forceinline__ void put_out(const f32x16_t& acc, const float (&b)[16], T* y, bool in, int c, int n, int vec) {
  const int lane = threadIdx.x & 63;
  float v[16];
#pragma unroll
  for (int z = 0; z < 16; ++z) v[z] = acc[z] + b[z];
  if constexpr (sizeof(T) == 2) {
    unsigned pk[8];
#pragma unroll
    for (int z = 0; z < 8; ++z) pk[z] = pack_bf16(v[2 * z], v[2 * z + 1]);
    put8(pk, [&](int h, u32x4 u) {
      const int at = c + 16 * h + 8 * (lane >> 5);
      if (!in) return;
      if (vec && at + 8 <= n) {
        *(u32x4*)(y + at) = u;
      } else {
#pragma unroll
        for (int z = 0; z < 8; ++z)
          if (at + z < n) y[at + z] = (bf16_t)(u[z / 2] >> (16 * (z & 1)));
      }
    });
  } else {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int at = c + 8 * g + 4 * (lane >> 5);
      if (!in) continue;
      if (vec && at + 4 <= n) {
        *(float4*)(y + at) = make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
      } else {
#pragma unroll
        for (int z = 0; z < 4; ++z)
          if (at + z < n) y[at + z] = v[4 * g + z];
      }
    }
  }
}

// SPLIT: ranges of `per` of the sum, each into rows of its own at part.
template <typename PR, typename T, bool SPLIT>
__global__ __launch_bounds__(PR::T, PR::NW == 8 || PR::LDS <= 80 * 1024 ? 2 : 1) void gated_out(OutArgs a) {
  __shared__ __align__(1024) unsigned char ring[PR::LDS];
  const int tiles = a.tm * a.tn, blk = xcd_remap(blockIdx.x, gridDim.x), q = SPLIT ? blk / tiles : 0;
  const int k0 = SPLIT ? q * a.per : 0, k1 = SPLIT ? min(a.k, k0 + a.per) : a.k;
  int ti, tj;
  tile_of(blk - q * tiles, a.tm, a.tn, &ti, &tj);
  const int i0 = ti * PR::BM, j0 = tj * PR::BN, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  PR p;
  p.zero();
  p.run(ring, a.s, a.lda, a.ldb, a.rows, a.n, i0, j0, k0, k1, [](u32x4, int, int) {});
#pragma unroll
  for (int j = 0; j < PR::NT; ++j) {
    const int c = j0 + (wave % PR::WN * PR::NT + j) * 32;
    float b[16];
    biases(SPLIT ? nullptr : a.bias, c, a.n, b);
#pragma unroll
    for (int i = 0; i < PR::MT; ++i) {
      const long r = i0 + (wave / PR::WN * PR::MT + i) * 32 + (lane & 31);
      if constexpr (SPLIT)
        put_out<float>(p.acc[0][i][j], b, a.part + ((long)q * a.rows + r) * a.ldp, r < a.rows, c, a.ldp, 1);
      else
        put_out<T>(p.acc[0][i][j], b, (T*)a.y + r * a.ldy, r < a.rows, c, a.n, a.vec);
    }
  }
}

// y = the ranges' sums, in order, + bias; four columns a thread.
template <typename T>
__global__ __launch_bounds__(kT) void gated_join(OutArgs a, int ranges) {
  const int per = a.ldp / 4, e = blockIdx.x * kT + threadIdx.x, r = e / per, c = (e - r * per) * 4;
  if (r >= a.rows) return;
  const float* p = a.part + (long)r * a.ldp + c;
  float4 s = *(const float4*)p;
#pragma unroll 4
  for (int q = 1; q < ranges; ++q) {
    const float4 v = *(const float4*)(p + (long)q * a.rows * a.ldp);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  const float v[4] = {s.x, s.y, s.z, s.w};
  T* y = (T*)a.y + r * a.ldy + c;
#pragma unroll
  for (int z = 0; z < 4; ++z)
    if (c + z < a.n) Elt<T>::st(y + z, v[z] + (a.bias ? a.bias[c + z] : 0.f));
}

// ------------------------------------------------- narrow blocks in one launch

struct NarrowArgs {
  const bf16_t *x[kMaxParts], *w[2][kMaxParts], *wd[kMaxParts];
  long lda, ldb, ldwd;
  int rows, cin, hidden, cout;
  const float *bg, *bu, *bd;
  void* y;
  long ldy;
  int vec;
};

// The 32 biases from column c on (the same for the wave), by scalar loads: vector loads
// would wait behind the ring's.  Lane l's sixteen, as in a fragment.  (Columns from n on
// get some bias: what becomes of them meets zeros.)
__device__ __forceinline__ void wave_biases(const float* b, int c, int n, float (&v)[16]) {
  typedef const __attribute__((address_space(4))) float* uniform_p;
  const bool hi = (threadIdx.x & 63) >= 32;
  float s[32];
#pragma unroll
  for (int z = 0; z < 32; ++z) s[z] = 0.f;
  if (b) {
    const uniform_p p = (uniform_p)(unsigned long)b;
    if (c + 32 <= n) {
#pragma unroll
      for (int z = 0; z < 32; ++z) s[z] = p[c + z];
    } else {
#pragma unroll
      for (int z = 0; z < 32; ++z) s[z] = p[min(c + z, n - 1)];
    }
  }
#pragma unroll
  for (int z = 0; z < 16; ++z) v[z] = hi ? s[8 * (z / 4) + 4 + z % 4] : s[8 * (z / 4) + z % 4];
}

// y of 64 pixels, 32 NW hidden channels at a time: a wave has 64 pixels x 32 channels of
// g and u, and leaves their h in LDS, the next product's left factor; nothing of the
// hidden channels goes to memory.  The pixels' fragments (KSX stages of 64 channels,
// P parts) stay in registers.  The ring's stages are all of one size and hold one
// matrix's part: first the pixels', then 64 channels of Wg or Wu for the tile's hidden
// channels, or of Wd for 32 CG output channels, KG = NW / CG ranges of 64 hidden
// channels at once, by as many groups of waves, whose sums meet at the end.
//
// A turn multiplies a stage's fragments, and between its products reads the next
// stage's and sends one load of the stage NS ahead after the other: a CU takes a KiB
// of such loads in 19 clocks (55 bytes a clock, of rows of 128 bytes or more; half of
// that of rows of 64), and a wave that sends four at once waits that long.  12544 x
// 256, 1024 hidden channels: 58 us with the loads before the products.
template <int P, int KSX, int NW, int CG, int ACT, typename T>
__global__ __launch_bounds__(64 * NW, P == 1 ? 2 : 1) void gated_narrow(NarrowArgs a) {
  // from three stages of 64 channels on the pixels stay in LDS, which leaves the ring
  // less, and the fragments of one are in registers: all of them spill
  constexpr bool XL = P == 1 && KSX >= 3;
  constexpr int XK = XL ? 1 : KSX;   // stages of pixels in registers
  // Of bfloat16 h is two parts, 16 bits, so that y is rounded once.  A ring of three leaves
  // LDS for them; where the pixels take that as well, it holds half of the tile's channels
  // at a time.  (131072 x 128, 512 hidden channels, as two launches: 116 us, with a ring of
  // four and halves 132, with h in one part, which single values of y show, 92; as one 106.)
  constexpr int Q = P == 1 ? 2 : P;
  constexpr bool HALF = XL;
  constexpr int NS = P == 1 ? 3 : 6, BK = 64, BH = 32 * NW, KG = NW / CG, H = BK / 16, L = 4;
  constexpr int HK = BH / (HALF ? 128 : 64);   // 64s of channels that LDS holds
  typedef Feed<BH, BK, false, NW> FW;
  typedef Feed<64, BK, false, 2> FH;   // (its layout)
  constexpr int SLOT = FW::BYTES, HB = FH::BYTES, DUAL = 2 * P * KSX, SPT = DUAL + P * CG / 2;
  static_assert(FW::LOADS == L && H == L && KSX * HB <= SLOT && P < NS, "a load between the products of a step");
  __shared__ __align__(1024) unsigned char ring[NS * SLOT + Q * HK * HB + XL * SLOT];
  static_assert(!HALF || (P == 1 && CG >= 4), "two stages of Wd at least");
  static_assert(sizeof(ring) <= 160 * 1024 && NS * SLOT >= NW * 8192, "LDS");
  unsigned char* const hs = ring + NS * SLOT;   // [part][64 channels], as stages of 64 rows
  unsigned char* const xs = XL ? hs + Q * HK * HB : ring;   // the pixels, [64 channels][64 rows]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = blockIdx.x * 64;
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long)TGP_LDS(ring) + wave * 1024);
  const int tiles = (a.hidden + BH - 1) / BH;
  const long ldw = a.ldb * 2, ldd = a.ldwd * 2;
  // the lane's chunks: of Wg and Wu, and of Wd (LDS row r is output channel r % (32 CG), of
  // range r / (32 CG))
  int vw[L], vd[L], kd[L];
#pragma unroll
  for (int u = 0; u < L; ++u) {
    const int r = (wave + u * NW) * 8 + lane / 8, q = (lane % 8) ^ FW::swz(r), row = r % (32 * CG);
    vw[u] = (int)(r * ldw) + q * 16;
    kd[u] = 64 * (r / (32 * CG)) + q * 8;
    vd[u] = row < a.cout ? (int)(row * ldd) + kd[u] * 2 : kOob;
  }
  const int kq = kd[0] & 63;   // (the same in all: swz sees the wave's parity alone)
  auto desc = [&](unsigned long p, long bytes) __attribute__((always_inline)) {
    return u32x4{(unsigned)p, (unsigned)(p >> 32) & 0xffffu, (unsigned)max(0l, min(bytes, 0x7fffffffl)), 0x00020000u};
  };
  // load u of stage `step` of tile t, into slot (beyond the last tile: zeros)
  auto load = [&](auto stepc, int t, int slot, auto uc) __attribute__((always_inline)) {
    constexpr int step = decltype(stepc)::value, u = decltype(uc)::value;
    const unsigned d = lds + slot * SLOT + u * NW * 1024;
    int v[1];
    if constexpr (step < DUAL) {
      constexpr int k = step / (2 * P), m = step & 1, j = P - 1 - step / 2 % P;
      // rows from `hidden` on are past the matrix's end
      const long at = t * (BH * ldw) + k * BK * 2;
      v[0] = k < KSX - 1 || kq < a.cin - k * BK ? vw[u] : kOob;
      dma_n<1, 0>(desc((unsigned long)a.w[m][j] + at, (long)a.hidden * ldw - at), d, v);
    } else {
      constexpr int o = (step - DUAL) / P, j = P - 1 - (step - DUAL) % P;
      const int at = t * BH + o * (64 * KG);
      v[0] = kd[u] < a.hidden - at ? vd[u] : kOob;
      dma_n<1, 0>(desc((unsigned long)(a.wd[j] + at), t < tiles ? 0x7fffffff : 0), d, v);
    }
  };
  auto stage = [&](auto stepc, int t, int slot) __attribute__((always_inline)) {
    each<L>([&](auto u) { load(stepc, t, slot, u); });
  };
  // the pixels, part p in slot p: [64 channels][64 rows]
#pragma unroll
  for (int p = 0; p < P; ++p) {
    int v[L];
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int c8 = wave + u * NW, row = (c8 % 8) * 8 + lane / 8, k = c8 / 8, q = (lane % 8) ^ FH::swz(row);
      v[u] = k < KSX && row < a.rows - i0 && k * BK + q * 8 < a.cin ? (int)(row * a.lda * 2) + k * BK * 2 + q * 16 : kOob;
    }
    const unsigned d = lds + (unsigned)(xs - ring) + p * SLOT;
    dma_n<L, NW * 1024>(desc((unsigned long)(a.x[p] + (long)i0 * a.lda), 0x7fffffff), d, v);
  }
  // (in the first slots, where they do not stay)
  constexpr int S0 = XL ? 0 : P;   // the first stage's slot
  each<NS - S0>([&](auto z) {
    constexpr int n = decltype(z)::value;
    stage(std::integral_constant<int, n % SPT>(), n / SPT, S0 + n);
  });
  wait_vmcnt<(NS - S0) * L>();
  ring_barrier();
  u32x4 x[P][XK][H][2];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < XK; ++k)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) x[p][k][h][i] = FH::frag(xs + p * SLOT + k * HB, FH::place(32 * i), h);
  if constexpr (!XL) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ring_barrier();
    each<P>([&](auto z) {
      constexpr int n = NS - P + decltype(z)::value;
      stage(std::integral_constant<int, n % SPT>(), n / SPT, decltype(z)::value);
    });
  }
  const int pb = FW::place(wave * 32);
  u32x4 b[H];   // the fragments of the stage to be multiplied
  int slot = S0;
  wait_vmcnt<(NS - 1) * L>();
  ring_barrier();
#pragma unroll
  for (int h = 0; h < H; ++h) b[h] = FW::frag(ring + slot * SLOT, pb, h);
  // Stage `step` of tile t: mul(h) are the products of step h.  At the barrier the next
  // stage has landed, and every wave has this one's fragments: its slot is free.
  auto turn = [&](auto stepc, int t, auto mul) __attribute__((always_inline)) {
    constexpr int step = decltype(stepc)::value, ahead = step + NS;
    wait_vmcnt<(NS - 2) * L>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // b, and h where this wave has just written it
    ring_barrier();
    const int next = slot + 1 == NS ? 0 : slot + 1;
    each<H>([&](auto hc) {
      constexpr int h = decltype(hc)::value;
      __builtin_amdgcn_sched_barrier(0);
      mul(h);
      b[h] = FW::frag(ring + next * SLOT, pb, h);
      load(std::integral_constant<int, ahead % SPT>(), t + ahead / SPT, slot, hc);
    });
    __builtin_amdgcn_sched_barrier(0);
    slot = next;
  };
  f32x16_t y[2] = {};
  for (int ht = 0; ht < tiles; ++ht) {
    f32x16_t g[2], u[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) g[i] = u[i] = f32x16_t{};
    each<DUAL>([&](auto sc) {
      constexpr int step = decltype(sc)::value, k = step / (2 * P), j = P - 1 - step / 2 % P;
      turn(sc, ht, [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int p = P - 1 - j; p >= 0; --p)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if constexpr (step & 1) u[i] = mfma32(as_bf16x8(b[h]), as_bf16x8(x[p][XL ? 0 : k][h][i]), u[i]);
            else g[i] = mfma32(as_bf16x8(b[h]), as_bf16x8(x[p][XL ? 0 : k][h][i]), g[i]);
            if constexpr (XL && step & 1) x[0][0][h][i] = FH::frag(xs + (k + 1) % KSX * HB, FH::place(32 * i), h);
          }
      });
    });
    const int c = ht * BH + wave * 32;
    float bg[16], bu[16];
    wave_biases(a.bg, c, a.hidden, bg);
    wave_biases(a.bu, c, a.hidden, bu);
    unsigned hp[2][Q][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float v[16];
#pragma unroll
      for (int z = 0; z < 16; ++z) {
        float act, slope;
        act_of<ACT, P == 3>(g[i][z] + bg[z], &act, &slope);
        v[z] = act * (u[i][z] + bu[z]);
      }
#pragma unroll
      for (int p = 0; p < Q; ++p) {
#pragma unroll
        for (int z = 0; z < 8; ++z) hp[i][p][z] = pack_bf16(v[2 * z], v[2 * z + 1]);
        if (p + 1 < Q)
#pragma unroll
          for (int z = 0; z < 16; ++z) {
            const unsigned w = hp[i][p][z / 2];
            const float hi = z & 1 ? __uint_as_float(w & 0xffff0000u) : __uint_as_float(w << 16);
            v[z] = (__float_as_uint(hi) & 0x7f800000u) == 0x7f800000u ? 0.f : v[z] - hi;
          }
      }
      __builtin_amdgcn_sched_barrier(0);   // one fragment's values at a time: registers
    }
    auto put_h = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = 32 * i + (lane & 31);
#pragma unroll
        for (int p = 0; p < Q; ++p)
          put8(hp[i][p], [&](int h, u32x4 w) {
            const int q = (wave & 1) * 4 + 2 * h + (lane >> 5);
            *(u32x4*)(hs + (p * HK + (wave >> 1) % HK) * HB + row * 128 + ((q ^ FH::swz(row)) << 4)) = w;
          });
      }
    };
    // (every wave has met a barrier since the last product read h)
    if (!HALF || wave < NW / 2) put_h();
    // fragments of h: a stage's for its P turns, or (bfloat16) of one step and the next
    constexpr int HF = P == 1 ? 2 : H;
    u32x4 hf[HF][Q][2];
    auto read_h = [&](int o, int z) __attribute__((always_inline)) {
#pragma unroll
      for (int p = 0; p < Q; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          hf[z % HF][p][i] = FH::frag(hs + (p * HK + (o * KG + wave / CG) % HK) * HB, FH::place(32 * i), z);
    };
    each<P * CG / 2>([&](auto sc) {
      constexpr int s = decltype(sc)::value, o = s / P, j = P - 1 - s % P;
      constexpr bool fresh = o == 0 || (HALF && o == CG / 4);   // h is not what the turn before read
      constexpr bool more = s + 1 < P * CG / 2 && !(HALF && o + 1 == CG / 4);
      if constexpr (HALF && o == CG / 4) {   // the other half, when every wave has read the first
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        ring_barrier();
        if (wave >= NW / 2) put_h();
      }
      turn(std::integral_constant<int, DUAL + s>(), ht, [&](int h) __attribute__((always_inline)) {
        if constexpr (P == 1) {
          if (fresh && h == 0) read_h(o, 0);
          if (h + 1 < H) read_h(o, h + 1);
          else if (more) read_h(o + 1, 0);
        } else if (h == 0 && j == P - 1) {
#pragma unroll
          for (int z = 0; z < H; ++z) read_h(o, z);
        }
#pragma unroll
        for (int p = Q - 1 - j; p >= 0; --p)
#pragma unroll
          for (int i = 0; i < 2; ++i) y[i] = mfma32(as_bf16x8(b[h]), as_bf16x8(hf[h % HF][p][i]), y[i]);
      });
    });
  }
  wait_vmcnt<0>();
  if constexpr (KG > 1) {   // the groups' sums, in order
    ring_barrier();         // nothing is on its way into the ring, and nothing read from it
    float* red = (float*)ring;   // [wave][i][value][lane]
    if (wave >= CG)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int z = 0; z < 16; ++z) red[((wave * 2 + i) * 16 + z) * 64 + lane] = y[i][z];
    __syncthreads();
    if (wave >= CG) return;
#pragma unroll
    for (int k = 1; k < KG; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int z = 0; z < 16; ++z) y[i][z] += red[(((wave + k * CG) * 2 + i) * 16 + z) * 64 + lane];
  }
  const int c = wave % CG * 32;
  float bd[16];
  biases(a.bd, c, a.cout, bd);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const long r = i0 + 32 * i + (lane & 31);
    put_out<T>(y[i], bd, (T*)a.y + r * a.ldy, r < a.rows, c, a.cout, a.vec);
  }
}

// ------------------------------------------------- few pixels

// Eight values from k on of a row of n as they are in memory; `in`: whether the row is
// there; vec: rows lie at multiples of 16 bytes.
template <typename T>
struct Eight;
template <>
struct Eight<bf16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t* row, int k, int n, bool in, int vec) {
    if (in && vec && k + 8 <= n) {
      w = *(const u32x4*)(row + k);
    } else {
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const unsigned lo = in && k + 2 * z < n ? row[k + 2 * z] : 0u, hi = in && k + 2 * z + 1 < n ? row[k + 2 * z + 1] : 0u;
        w[z] = lo | hi << 16;
      }
    }
  }
};
template <>
struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* row, int k, int n, bool in, int vec) {
    if (in && vec && k + 8 <= n) {
      const float4 a = *(const float4*)(row + k), b = *(const float4*)(row + k + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int z = 0; z < 8; ++z) v[z] = in && k + z < n ? row[k + z] : 0.f;
    }
  }
};
// A value as two bfloat16s, in the order of fragments: sixteen channels of 32 MF pixels
// are MF times 64 lanes' eight values; the second parts `plane` values behind the first.
struct Pair {
  bf16_t at;
};
template <>
struct Eight<Pair> {
  u32x4 p[2];
  // n: channels from the lane's first on; in: whether the lane's pixel is there
  __device__ __forceinline__ void load(const bf16_t* at, long plane, int n, bool in) {
    p[0] = p[1] = u32x4{};
    if (!in || n <= 0) return;
    p[0] = *(const u32x4*)at;
    p[1] = *(const u32x4*)(at + plane);
    if (n >= 8) return;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int z = 0; z < 4; ++z) p[q][z] = 2 * z + 1 < n ? p[q][z] : 2 * z < n ? p[q][z] & 0xffffu : 0u;
  }
};
template <typename T>
struct Frag {
  static constexpr int P = sizeof(T) == 2 ? 1 : 3;
  u32x4 p[P];
  __device__ __forceinline__ void set(const Eight<T>& e) {
    if constexpr (P == 1) p[0] = e.w;
    else split(e.v);
  }
  __device__ __forceinline__ void split(const float (&f)[8]) {
    float v[8];
#pragma unroll
    for (int z = 0; z < 8; ++z) v[z] = f[z];
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
      for (int z = 0; z < 4; ++z) p[q][z] = pack_bf16(v[2 * z], v[2 * z + 1]);
      if (q + 1 < P)
#pragma unroll
        for (int z = 0; z < 8; ++z) {
          const float hi = z & 1 ? __uint_as_float(p[q][z / 2] & 0xffff0000u) : __uint_as_float(p[q][z / 2] << 16);
          v[z] = (__float_as_uint(hi) & 0x7f800000u) == 0x7f800000u ? 0.f : v[z] - hi;
        }
    }
  }
};
template <>
struct Frag<Pair> {
  static constexpr int P = 2;
  u32x4 p[P];
  __device__ __forceinline__ void set(const Eight<Pair>& e) {
    p[0] = e.p[0];
    p[1] = e.p[1];
  }
};
// c + a's rows times b's: the pairs of parts that a float32 product needs, small ones first
template <typename TA, typename TB>
__device__ __forceinline__ f32x16_t times(const Frag<TA>& a, const Frag<TB>& b, f32x16_t c) {
  constexpr int PA = Frag<TA>::P, PB = Frag<TB>::P;
#pragma unroll
  for (int d = 2; d >= 0; --d)
#pragma unroll
    for (int i = d; i >= 0; --i)
      if (i < PA && d - i < PB) c = mfma32(as_bf16x8(a.p[i < PA ? i : 0]), as_bf16x8(b.p[d - i < PB ? d - i : 0]), c);
  return c;
}

struct FewArgs {
  const void *x, *w[2];
  const float* b[2];
  void* y;
  long ldx, ldw, ldy;
  int rows, k, n, vx, vw;
  int cw;       // channels of a block
  long plane;   // from the first parts of h to the second (Pair)
};

// Up to 32 MF pixels: cw channels of the result a block, NW waves that share the sum; M
// matrices (two: h, else y).  Weights are read once, straight into fragments, and what
// bounds it is how many of their loads are on their way at a time: as many waves as a
// block has, and blocks of fewer channels (the other rows of their fragments are zeros)
// where 32 each leave CUs without one (1 x 1024 through 4096 and back 22.8 us, with 32
// channels a block 41; its 24 MB come in at 1.1 TB/s).  Of a bfloat16 network h is two
// parts in the order of fragments, loads of 1 KB (60 such pixels 43.8 us; in rows, whose
// loads take 32 bytes each of 32 rows, 59.9, and one part in rows 43.8).
template <typename TX, typename TW, typename TY, int M, int MF, int NW, int ACT>
__global__ __launch_bounds__(64 * NW) void gated_few(FewArgs a) {
  constexpr int U = M == 1 && MF == 1 && sizeof(TW) == 2 ? 8 : 4;   // steps of 16 whose loads go out together
  __shared__ float red[NW][M * MF][16][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j0 = blockIdx.x * a.cw, col = j0 + (lane & 31), per = ((a.k + NW - 1) / NW + 15) / 16 * 16;
  const bool here = (lane & 31) < a.cw && col < a.n;
  const int k1 = min(a.k, (wave + 1) * per);
  f32x16_t acc[M][MF];
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[m][f] = f32x16_t{};
  for (int k0 = wave * per; k0 < k1; k0 += 16 * U) {
    Eight<TW> vw[U][M];
    Eight<TX> vx[U][MF];
#pragma unroll
    for (int s = 0; s < U; ++s) {
      const int k = k0 + 16 * s + 8 * (lane >> 5);
#pragma unroll
      for (int m = 0; m < M; ++m) vw[s][m].load((const TW*)a.w[m] + col * a.ldw, k, k1, here, a.vw);
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        const int r = 32 * f + (lane & 31);
        if constexpr (std::is_same<TX, Pair>::value)
          vx[s][f].load((const bf16_t*)a.x + ((k0 / 16 + s) * MF + f) * 512L + 8 * lane, a.plane, k1 - k, r < a.rows);
        else
          vx[s][f].load((const TX*)a.x + r * a.ldx, k, k1, r < a.rows, a.vx);
      }
    }
#pragma unroll
    for (int s = 0; s < U; ++s) {
      Frag<TW> w[M];
      Frag<TX> x;
#pragma unroll
      for (int m = 0; m < M; ++m) w[m].set(vw[s][m]);
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        x.set(vx[s][f]);
#pragma unroll
        for (int m = 0; m < M; ++m) acc[m][f] = times(w[m], x, acc[m][f]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) red[wave][m * MF + f][v][lane] = acc[m][f][v];
  __syncthreads();
  // a thread has columns n of pixel r: fragment value 4 (n / 8) + n % 4 of lane r % 32 +
  // 32 (n / 4 % 2), summed over the waves in order
  for (int e = threadIdx.x; e < 32 * 32 * MF; e += 64 * NW) {
    const int n = e & 31, r = e >> 5, f = r >> 5;
    if (r >= a.rows || n >= a.cw || j0 + n >= a.n) continue;
    const int v = 4 * (n >> 3) + (n & 3), l = (r & 31) + 32 * ((n >> 2) & 1);
    float s[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      s[m] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) s[m] += red[w][m * MF + f][v][l];
      if (a.b[m]) s[m] += a.b[m][j0 + n];
    }
    if constexpr (M == 2) {
      float act, slope;
      act_of<ACT, sizeof(TW) == 4>(s[0], &act, &slope);
      s[0] = act * s[1];
    }
    if constexpr (std::is_same<TY, Pair>::value) {
      const uint32_t top = f2bf(s[0]);
      const bool fine = (top & 0x7f80u) != 0x7f80u;   // an infinity or NaN has no rest
      const int c = j0 + n;
      bf16_t* to = (bf16_t*)a.y + ((c / 16 * MF + f) * 64L + (r & 31) + 32 * (c >> 3 & 1)) * 8 + (c & 7);
      to[0] = (bf16_t)top;
      to[a.plane] = (bf16_t)(fine ? f2bf(s[0] - bf2f(top)) : 0u);
    } else {
      Elt<TY>::st((TY*)a.y + r * a.ldy + j0 + n, s[0]);
    }
  }
}

// ------------------------------------------------- weights' gradients

// One matrix's gradient, a^T b over the pixels: m columns of a, n of b; partial sums
// of range q at part + q stride (rows of ldp floats), column sums of a at cols +
// q stride.  Of one range these are the gradients themselves (null: none), and are
// added to with `add`.
struct OuterJob {
  Segs<1> s;
  long lda, ldb;
  int m, n, ldp, tm, tn, blk0, vec;   // vec: rows at part lie at multiples of 16 bytes
  int sums;   // the pairs, a bit each, whose a's go into the column sums: every part once
  float *part, *cols;
};
struct OuterArgs {
  OuterJob j[3];
  int n, rows, per;    // jobs, pixels, pixels of a range (a multiple of the stage)
  int add;
  long stride;
};

template <typename PR>
__global__ __launch_bounds__(PR::T, PR::NW == 8 || PR::LDS <= 80 * 1024 ? 2 : 1) void gated_outer(OuterArgs a) {
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
    if (sums && lane < 32) {
      float* to = J.cols + q * a.stride + r;
      *to = a.add ? *to + ones[i][0] : ones[i][0];
    }
    if (!J.part) continue;
    float* to = J.part + q * a.stride + (long)r * J.ldp;
#pragma unroll
    for (int j = 0; j < PR::NT; ++j) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int at = j0 + (wave % PR::WN * PR::NT + j) * 32 + 8 * g + 4 * (lane >> 5);
        const f32x16_t& v = p.acc[0][i][j];
        if (J.vec) {
          if (at >= J.ldp) continue;
          float4 f = make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
          if (a.add) {
            const float4 o = *(const float4*)(to + at);
            f = make_float4(o.x + f.x, o.y + f.y, o.z + f.z, o.w + f.w);
          }
          *(float4*)(to + at) = f;
        } else {
#pragma unroll
          for (int z = 0; z < 4; ++z)
            if (at + z < J.n) to[at + z] = a.add ? to[at + z] + v[4 * g + z] : v[4 * g + z];
        }
      }
    }
  }
}

// Where a range's sums of a weight go: rows of ldp floats at part, its bias's at cols
// (null: not wanted), as an OuterJob's.
struct Sink {
  float *part, *cols;
  int ldp, n, vec;
};

struct SlimArgs {
  const bf16_t *x, *dy, *wg, *wu, *wd;
  long ldx, lddy, ldw, ldwd;
  int rows, per, cin, hidden, cout;
  const float *bg, *bu;
  Sink to[3];        // Wg, Wu, Wd
  long stride;
  int add;
  bf16_t* dx;
  long lddx;
  int vec;
};

// Everything of a backward pass through at most 64 channels, 256 hidden and 64 again,
// of bfloat16: a block takes `per` pixels, 64 at a time, and nothing of the hidden
// channels goes to memory.  A wave has 32 hidden channels; g, u and dh lie in its
// registers with a lane a hidden channel and pixels one after the other, which is how
// the weights' gradients' products over pixels take h, dg and du, with the rows of x and
// dy read from LDS in the order that those have (values j of a lane are pixels 4 (l / 32)
// + j and, from j = 4 on, 4 more).  The gradients' sums stay in registers to the end.
// For dx, dg and du go through LDS, 32 pixels at a time in their two parts, rows of hidden
// channels beside the weights' rows.
// What bounds it are the activations, the splitting in parts and the products, one after
// the other (147456 x 64, 256 hidden, GELU: 124 of a pass's 135 us, the rest the ranges'
// sums; a launch for h, dg and du, one for the weights and one for dx take three times as
// long).  The two halves of 64 pixels are a loop: unrolled, 39 registers spill (16 us).
template <int ACT, bool GRADS>
__global__ __launch_bounds__(512, 2) void gated_slim(SlimArgs a) {
  typedef Feed<64, 64, false, 2> F;   // (its layout: rows of 64 values)
  constexpr int TILE = 8192, WS = 32768;
  __shared__ __align__(1024) unsigned char lds[4 * WS + 4 * TILE];
  unsigned char *const wgs = lds, *const wus = lds + WS, *const dgs = lds + 2 * WS, *const dus = lds + 3 * WS,
                *const xs = lds + 4 * WS;   // [slot][x, dy]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int lo = blockIdx.x * a.per, hi = min(a.rows, lo + a.per);
  const unsigned base = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long)TGP_LDS(lds) + wave * 1024);
  auto desc = [&](const bf16_t* p) __attribute__((always_inline)) {
    const unsigned long at = (unsigned long)p;
    return u32x4{(unsigned)at, (unsigned)(at >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
  };
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ring_barrier();
  };
  // 64 pixels of x and dy, a KiB a wave each
  const int row = wave * 8 + lane / 8, q = (lane % 8) ^ F::swz(row);
  auto send = [&](int i0, int slot) __attribute__((always_inline)) {
    const int vx[1] = {row < hi - i0 && q * 8 < a.cin ? (int)(row * a.ldx * 2) + q * 16 : kOob};
    const int vy[1] = {row < hi - i0 && q * 8 < a.cout ? (int)(row * a.lddy * 2) + q * 16 : kOob};
    dma_n<1, 0>(desc(a.x + i0 * a.ldx), base + 4 * WS + slot * 2 * TILE, vx);
    dma_n<1, 0>(desc(a.dy + i0 * a.lddy), base + 4 * WS + slot * 2 * TILE + TILE, vy);
  };
  {
    int v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = (wave + 8 * u) * 8 + lane / 8, c = (lane % 8) ^ F::swz(r);
      v[u] = r < a.hidden && c * 8 < a.cin ? (int)(r * a.ldw * 2) + c * 16 : kOob;
    }
    dma_n<4, 8192>(desc(a.wg), base, v);
    dma_n<4, 8192>(desc(a.wu), base + WS, v);
  }
  send(lo, 0);
  const int hid = 32 * wave + (lane & 31);   // the lane's hidden channel
  const float bg = a.bg && hid < a.hidden ? a.bg[hid] : 0.f, bu = a.bu && hid < a.hidden ? a.bu[hid] : 0.f;
  u32x4 wd[4];   // a row of Wd^T
  {
    // (every lane loads, from inside the matrix: behind conditions the loads would wait for
    // one another)
    const bf16_t* const from = a.wd + min(hid, a.hidden - 1);
    unsigned e[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) e[k] = from[min(16 * (k / 8) + 8 * half + k % 8, a.cout - 1) * a.ldwd];
#pragma unroll
    for (int k = 0; k < 32; ++k)
      if (hid >= a.hidden || 16 * (k / 8) + 8 * half + k % 8 >= a.cout) e[k] = 0u;
#pragma unroll
    for (int k = 0; k < 16; ++k) wd[k / 4][k % 4] = e[2 * k] | e[2 * k + 1] << 16;
  }
  // reads by columns: rows r0 and r0 + 8 of sixteen, 8 bytes of this lane's part
  const int r0 = 4 * half + ((lane & 15) >> 2), q0 = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int at0 = r0 * 128 + ((q0 ^ F::swz(r0)) << 4) + 8 * (lane & 1);
  const int at8 = (r0 + 8) * 128 + ((q0 ^ F::swz(r0 + 8)) << 4) + 8 * (lane & 1);
  auto column = [&](const unsigned char* s, int f) __attribute__((always_inline)) {   // f: columns 32 f on
    const uint2 e = lds_tr16(s + (at0 ^ (64 * f))), g = lds_tr16(s + (at8 ^ (64 * f)));
    return u32x4{e.x, e.y, g.x, g.y};
  };
  f32x16_t sg[2], su[2], sd[2];
#pragma unroll
  for (int f = 0; f < 2; ++f) sg[f] = su[f] = sd[f] = f32x16_t{};
  float bsg = 0.f, bsu = 0.f, bsd = 0.f;
  int slot = 0;
  for (int i0 = lo; i0 < hi; i0 += 64, slot ^= 1) {
    wait_vmcnt<0>();
    meet();
    if (i0 + 64 < hi) send(i0 + 64, slot ^ 1);
    const unsigned char *const xt = xs + slot * 2 * TILE, *const yt = xt + TILE;
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      __builtin_amdgcn_sched_barrier(0);   // one fragment's values at a time: registers
      f32x16_t g{}, u{}, d{};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const u32x4 x = F::frag(xt, F::place(32 * i), h), y = F::frag(yt, F::place(32 * i), h);
        g = mfma32(as_bf16x8(x), as_bf16x8(F::frag(wgs, F::place(32 * wave), h)), g);
        u = mfma32(as_bf16x8(x), as_bf16x8(F::frag(wus, F::place(32 * wave), h)), u);
        d = mfma32(as_bf16x8(y), as_bf16x8(wd[h]), d);
        if (h & 1) __builtin_amdgcn_sched_barrier(0);
      }
      const int left = hi - i0 - 32 * i - 4 * half;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float act, slope;
        act_of<ACT, true>(g[v] + bg, &act, &slope);
        const float up = u[v] + bu, dh = d[v];
        const bool in = 8 * (v / 4) + v % 4 < left;   // (a bias may be infinite)
        g[v] = in ? dh * up * slope : 0.f;
        u[v] = in ? dh * act : 0.f;
        d[v] = in ? act * up : 0.f;
        bsg += g[v];
        bsu += u[v];
      }
      if (i && a.dx) meet();   // the first 32 pixels' sums are out of dgs
      // 16 pixels' parts of dg, du and h, and their products
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        const int s16 = (2 * i + k) * 2048;
        // of the 32 pixels' first parts chunks 0 .. 3, of their second 4 .. 7: pixels 8 (2 k) +
        // 4 half on, and 8 (2 k + 1) + 4 half on
        const int to = hid * 128 + 8 * half, sw = F::swz(hid), c = 2 * k;
#pragma unroll
        for (int m = 0; m < 3; ++m) {
          constexpr int Q = GRADS ? 3 : 2;
          u32x4 q[Q];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const f32x16_t& w = m == 0 ? g : m == 1 ? u : d;
            float e = w[8 * k + 2 * z], f = w[8 * k + 2 * z + 1];
#pragma unroll
            for (int n = 0; n < Q; ++n) {   // (an infinity leaves NaN)
              q[n][z] = pack_bf16(e, f);
              e -= __uint_as_float(q[n][z] << 16);
              f -= __uint_as_float(q[n][z] & 0xffff0000u);
            }
          }
          if (m < 2 && a.dx) {
            unsigned char* const ds = m ? dus : dgs;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              *(uint2*)(ds + to + (((c + 4 * n) ^ sw) << 4)) = make_uint2(q[n][0], q[n][1]);
              *(uint2*)(ds + to + (((c + 4 * n + 1) ^ sw) << 4)) = make_uint2(q[n][2], q[n][3]);
            }
          }
          if constexpr (GRADS)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
              const u32x4 x = column((m < 2 ? xt : yt) + s16, f);
#pragma unroll
              for (int w = Q - 1; w >= 0; --w) {
                const bf16x8_t e = as_bf16x8(q[w]);
                if (m == 0) sg[f] = mfma32(as_bf16x8(x), e, sg[f]);
                else if (m == 1) su[f] = mfma32(as_bf16x8(x), e, su[f]);
                else sd[f] = mfma32(e, as_bf16x8(x), sd[f]);
              }
            }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (!a.dx) continue;
      meet();
      // a fragment of dx a wave: of dg Wg (waves 0 to 3) or du Wu, of first or second parts
      const int part = wave >> 1 & 1, cf = wave & 1;
      const unsigned char *const ds = wave < 4 ? dgs : dus, *const ws = wave < 4 ? wgs : wus;
      f32x16_t o{};
#pragma unroll 2
      for (int h = 0; h < 16; ++h)
        o = mfma32(as_bf16x8(column(ws + h * 2048, cf)), as_bf16x8(column(ds + h * 2048, part)), o);
      meet();
      float* const rest = (float*)dgs + lane;   // [wave - 2][value][lane]
      if (wave >= 2)
#pragma unroll
        for (int v = 0; v < 16; ++v) rest[(wave - 2) * 1024 + v * 64] = o[v];
      meet();
      if (wave < 2) {
        // beside waves 0 and 1: the first parts of du, the second of dg and of du
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float* const q = rest + wave * 1024 + v * 64;
          o[v] = (o[v] + q[2 * 1024]) + (q[0] + q[4 * 1024]);
        }
        const float none[16] = {};
        const int r = i0 + 32 * i + (lane & 31);
        put_out<bf16_t>(o, none, a.dx + r * a.lddx, r < hi, 32 * cf, a.cin, a.vec);
      }
    }
    // column sums of dy: eight pixels a wave
    if constexpr (GRADS)
#pragma unroll
    for (int z = 0; z < 8; ++z) {
      const int r = 8 * wave + z;
      bsd += bf2f(*(const bf16_t*)(yt + r * 128 + (((lane >> 3) ^ F::swz(r)) << 4) + 2 * (lane & 7)));
    }
  }
  if constexpr (!GRADS) return;
  // The sums, a matrix at a time through LDS (64 KB): rows of hidden channels (of Wd's: of
  // cout), chunks of four columns XORed with the row.  (Straight from the registers the
  // stores are 16 KB of instructions, which one block after the other fetches.)
  const long off = blockIdx.x * a.stride;
  auto place = [&](int r, int chunk, int wide) __attribute__((always_inline)) {
    return (float4*)(dgs + (r * wide + (chunk ^ (r & 15))) * 16);
  };
  auto put = [&](const Sink& t, int rows, int wide) __attribute__((always_inline)) {
    meet();
#pragma unroll 1
    for (int e = threadIdx.x; e < 4096; e += 512) {
      const int r = e / wide, c = 4 * (e % wide);
      if (r >= rows || c >= t.n) continue;
      float4 v = *place(r, e % wide, wide);
      float* to = t.part + off + (long)r * t.ldp + c;
      if (t.vec) {
        if (a.add) {
          const float4 o = *(const float4*)to;
          v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
        }
        *(float4*)to = v;
      } else {
        const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int z = 0; z < 4; ++z)
          if (c + z < t.n) to[z] = a.add ? to[z] + w[z] : w[z];
      }
    }
  };
  auto put_col = [&](const Sink& t, int r, int n, float v) __attribute__((always_inline)) {
    if (!t.cols || r >= n) return;
    float* to = t.cols + off + r;
    *to = a.add ? *to + v : v;
  };
#pragma unroll
  for (int m = 0; m < 3; ++m) {
    if (!a.to[m].part) continue;
    meet();   // every wave is done with dgs and dus
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x16_t& w = m == 0 ? sg[f] : m == 1 ? su[f] : sd[f];
        float4* const to = m < 2 ? place(hid, 8 * f + 2 * g + half, 16)
                                 : place(32 * f + (lane & 31), 8 * wave + 2 * g + half, 64);
        *to = make_float4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
      }
    if (m < 2) put(a.to[m], a.hidden, 16);
    else put(a.to[m], a.cout, 64);
  }
  bsg += __shfl_xor(bsg, 32);
  bsu += __shfl_xor(bsu, 32);
  if (lane < 32) {
    put_col(a.to[0], hid, a.hidden, bsg);
    put_col(a.to[1], hid, a.hidden, bsu);
  }
  meet();   // every wave is done with dgs
  float* const cols = (float*)dgs;
  cols[wave * 64 + lane] = bsd;
  meet();
  if (wave) return;
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) t += cols[w * 64 + lane];
  put_col(a.to[2], lane, a.cout, t);
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
__global__ __launch_bounds__(256) void gated_sum(SumArgs a) {
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

__global__ void gated_zero(float* p, long n) {
  const long i = (long)blockIdx.x * kT + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

// ------------------------------------------------- plans

// Large and small tiles of each launch.  A CU takes 55 bytes a clock from DMA, so a stage
// of 128 x 128 tiles (64 values, 32 KB, 582 clocks) comes in slower than its 512 clocks of
// products: tiles of 256 rows where there are enough of them.  4096 pixels x 1024, 4096
// hidden: h 88 us (785 TFLOP/s), h, dg and du 174 (in two parts 156, and by two blocks of
// 128 x 64 a CU 163), the weights' gradients 317 (976; in two parts 215, and by tiles of
// 128 x 128 255), y 69 (988) and dx 136 (1011).  Stages of 32 pixels where both factors are read by columns: the
// fragments of one of 64 spill (787).  y and dx take a left factor's two parts in one
// stage, 48 KB of a 128 x 128 tile for twice the products (y part by part, the right
// factor read twice: 96 us).
typedef Product<2, 2, 4, 2, 64, 2, false, false, 2> HidL;
typedef Product<1, 1, 2, 2, 64, 3, false, false, 2> HidS;
typedef Product<2, 1, 2, 4, 64, 3, false, false, 2> BackL;
typedef Product<2, 1, 2, 4, 64, 3, false, true, 1> DhL;
typedef Product<1, 1, 2, 2, 64, 3, false, true, 1> DhS;
// BKS: the right factor's rows are the sum's; NA: the left factor's parts that are taken at once
template <bool BKS, int NA> struct Sums;
template <bool BKS> struct Sums<BKS, 1> {
  typedef Product<2, 2, 2, 2, 64, 4, false, BKS, 1> L;
  typedef Product<2, 2, 2, 2, 64, 2, false, BKS, 1> L2;
  typedef Product<1, 1, 2, 2, 64, 4, false, BKS, 1> S;
};
template <bool BKS> struct Sums<BKS, 2> {
  typedef Product<2, 2, 2, 2, 64, 3, false, BKS, 1, 2> L;
  typedef Product<2, 2, 4, 2, 64, 2, false, BKS, 1, 2> L2;
  typedef Product<1, 1, 2, 2, 64, 3, false, BKS, 1, 2> S;
};
typedef Product<2, 4, 4, 2, 32, 4, true, true, 1> OuterX;
typedef Product<2, 2, 2, 2, 32, 4, true, true, 1> OuterL;
typedef Product<1, 1, 2, 2, 64, 4, true, true, 1> OuterS;

constexpr long kFill = 256;   // tiles that fill the chip

// A call's workspace and how its pixels are taken.
struct Plan {
  int parts, hparts;     // of a factor; of h, dg and du
  long cinp, hidp, coutp;
  long chunk;            // pixels at a time
  bool slim;             // a backward pass in one launch
  int wide;              // the weights' gradients' tiles
  int ranges, per;       // of the pixels of a chunk, at most
  long stride;           // floats of a range's partial sums
  size_t x, dy, wg, wu, wd, h, dg, du, part, join, bytes;   // offsets
};

constexpr int kFewRows = 64;

// Whether one launch takes a forward pass whole: what its registers and LDS hold.
bool narrow(const tgp_gated_shape& s, long rows) {
  const int most = s.dtype == TGP_BF16 ? 256 : 128;
  return s.cin <= most && s.cout <= most && (rows > kFewRows || s.hidden <= 256);
}

// Whether two launches take it, whose weights go straight into registers.
bool few(const tgp_gated_shape& s, long rows) { return rows <= kFewRows && !narrow(s, rows); }
long few_pixels(long rows) { return rows <= 32 ? 32 : 64; }   // of its fragments

int ranges_of(long rows, int per) { return (int)((rows + per - 1) / per); }

// A long sum for few tiles of 64 x 64: ranges of `per` of its k values, four stages each
// at least, that the tiles' blocks fill the chip with; their partial sums are joined by a
// launch of its own (144 x 1024, k 4096: 20.6 us as 48 blocks, 7.5 and 4 as 240).
struct Split {
  int n, per;
};
Split split_of(long rows, long cols, int k, int pairs) {
  const long tiles = cdiv(rows, 64) * (long)cdiv(cols, 64), stages = (k + 63) / 64;
  const long want = std::min<long>(kFill / tiles, stages * pairs / 4);
  if (want < 2) return {1, k};
  const int per = (int)round_up((k + want - 1) / want, 64);
  return {(k + per - 1) / per, per};
}
size_t split_bytes(long rows, long cols, int k, int pairs) {
  const Split d = split_of(rows, cols, k, pairs);
  return d.n > 1 ? (size_t)4 * d.n * rows * round_up(cols, 4) : 0;
}

Plan plan_of(const tgp_gated_shape& s, long rows, bool backward) {
  Plan p{};
  p.parts = s.dtype == TGP_BF16 ? 1 : 3;
  p.hparts = s.dtype == TGP_BF16 && !backward ? 2 : 3;
  p.cinp = round_up(s.cin, 8);
  p.hidp = round_up(s.hidden, 8);
  p.coutp = round_up(s.cout, 8);
  const bool alone = !backward && narrow(s, rows);   // nothing lies between launches
  // so many pixels that what lies between launches stays in the caches, but that
  // a launch fills the chip
  const long a_row = 2 * (backward ? 3 * p.hparts * p.hidp + p.parts * (p.cinp + p.coutp)
                                   : (alone ? 0 : p.hparts * p.hidp) + p.parts * p.cinp);
  const long most = (long)(backward && p.parts == 1 ? 192 : 128) << 20;   // (of 256 MB)
  p.chunk = std::min(rows, std::max<long>(4096, most / a_row / 128 * 128));
  // (64 channels, 256 hidden, short runs of GELU: 1 pixel 21.9 us and in three launches 21.1,
  // 64 22.2 and 21.2, 1000 26.9 and 32.4, 12544 39.0 and 50.1, 147456 160 and 484; with few
  // hidden channels most waves of a block have none: 300 x 32, 64 hidden 24.6 and 21.2,
  // 12544 x 16, 32 hidden 30.5 and 26.8, 100000 x 16 93 and 114)
  p.slim = backward && s.dtype == TGP_BF16 && s.cin <= 64 && s.cout <= 64 && s.hidden > 64 && s.hidden <= 256;
  if (p.slim) p.chunk = std::min(rows, 1l << 22);   // (nothing lies between launches)
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += (n + 255) / 256 * 256;
    return here;
  };
  if (!backward && few(s, rows)) {   // reads all its operands where they are
    p.h = take((size_t)4 * few_pixels(rows) * round_up(s.hidden, 16));
    p.bytes = at;
    return p;
  }
  // copies of what does not lie in 16-byte pieces, which the query cannot see
  p.wg = take((size_t)2 * p.parts * s.hidden * p.cinp);
  p.wu = take((size_t)2 * p.parts * s.hidden * p.cinp);
  p.wd = take((size_t)2 * p.parts * s.cout * p.hidp);
  p.x = take((size_t)2 * p.parts * p.chunk * p.cinp);
  if (!backward) {
    p.h = take(alone ? 0 : (size_t)2 * p.hparts * p.chunk * p.hidp);
  } else {
    p.dy = take((size_t)2 * p.parts * p.chunk * p.coutp);
    const size_t plane = p.slim ? 0 : (size_t)2 * p.hparts * p.chunk * p.hidp;
    p.h = take(plane);
    p.dg = take(plane);
    p.du = take(plane);
    auto tiles = [&](long t) { return 2 * cdiv(s.hidden, t) * (long)cdiv(s.cin, t) + cdiv(s.cout, t) * (long)cdiv(s.hidden, t); };
    const long large = tiles(128);
    // as large as leave enough of them, with the ranges' help, and are not mostly padding
    const long x = tiles(256), runs = std::max<long>(1, p.chunk / 512);
    p.wide = 8 * 4 * x <= 9 * large && 4 * x * runs >= 3 * kFill ? 256 : large * runs >= kFill ? 128 : 64;
    const long n = tiles(p.wide), fill = p.wide == 256 ? kFill : 2 * kFill;
    // ranges of four stages at least, as many as fill the chip; one where the tiles do
    const long want = p.slim ? std::min<long>(kFill, cdiv(p.chunk, 64))
                      : 4 * n >= 3 * kFill ? 1 : std::max<long>(1, std::min<long>(fill / n, p.chunk / 256));
    p.per = (int)round_up((p.chunk + want - 1) / std::max<long>(want, 1), 64);
    p.ranges = ranges_of(p.chunk, p.per);
    p.stride = 2 * (long)s.hidden * round_up(s.cin, 4) + (long)s.cout * round_up(s.hidden, 4) +
               2 * round_up(s.hidden, 4) + round_up(s.cout, 4);
    p.part = take(p.ranges > 1 ? (size_t)4 * p.stride * p.ranges : 0);
  }
  const long rest = p.chunk ? rows % p.chunk : 0;
  auto room = [&](long r) {
    const int n = p.parts == 1 ? 1 : 6;   // pairs that add_sum makes
    return !r ? 0 : backward ? split_bytes(r, s.cin, s.hidden, 2 * n) : split_bytes(r, s.cout, s.hidden, n);
  };
  p.join = take(alone || p.slim ? 0 : std::max(room(p.chunk), room(rest)));
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
    if (g.s.dtype == TGP_BF16) TGP_LAUNCH(ps, gated_copy<bf16_t>, dim3((unsigned)copy_blocks), dim3(kT), 0, st, copies);
    else TGP_LAUNCH(ps, gated_copy<float>, dim3((unsigned)copy_blocks), dim3(kT), 0, st, copies);
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
    s->a[s->n][0] = a.part[i];
    s->b[s->n++][0] = b.part[j];
  });
}
// The same of a float32 network; of bfloat16 a's two parts as one pair with b.
template <typename T>
void add_sum(OutArgs* o, const Matrix& a, const Matrix& b) {
  Segs<1, 2>& s = o->s;
  if constexpr (sizeof(T) == 2) {
    s.a[s.n][0] = a.part[0];
    s.a[s.n][1] = a.part[1];
    s.b[s.n++][0] = b.part[0];
  } else {
    pairs(3, 3, [&](int i, int j) {
      s.a[s.n][0] = a.part[i];
      s.b[s.n++][0] = b.part[j];
    });
  }
}

bool fills(long rows, long cols) { return (long)cdiv(rows, 128) * cdiv(cols, 128) >= kFill; }

template <typename PR, typename T>
void launch_out(const char* name, OutArgs a, hipStream_t st) {
  a.tm = cdiv(a.rows, PR::BM);
  a.tn = cdiv(a.n, PR::BN);
  ProfScope ps(name, 2.0 * a.rows * a.k * a.n * a.s.n * PR::NA, 2.0 * a.rows * (a.k * PR::NA + a.n), st);
  TGP_LAUNCH(ps, (gated_out<PR, T, false>), dim3((unsigned)a.tm * a.tn), dim3(PR::T), 0, st, a);
}

// y or dx, by the number of tiles of 128 x 128: more than one a CU (bfloat16: 256 x 128 a
// block, 40000 x 304 of 600 58 us and by tiles of 128 x 128 62; float32: two shallow rings
// a CU), one, less, much less.
template <bool BKS, typename T>
void launch_sum(const char* name, const char* name_join, OutArgs a, void* join, hipStream_t st) {
  typedef Sums<BKS, sizeof(T) == 2 ? 2 : 1> PR;
  typedef typename PR::L2 PRL2;
  typedef typename PR::L PRL;
  typedef typename PR::S PRS;
  const long tiles = (long)cdiv(a.rows, 128) * cdiv(a.n, 128);
  if (tiles > kFill) return launch_out<PRL2, T>(name, a, st);
  if (tiles == kFill) return launch_out<PRL, T>(name, a, st);
  const Split d = split_of(a.rows, a.n, a.k, a.s.n);
  if (d.n == 1) return launch_out<PRS, T>(name, a, st);
  a.part = (float*)join;
  a.ldp = (int)round_up(a.n, 4);
  a.per = d.per;
  a.tm = cdiv(a.rows, PRS::BM);
  a.tn = cdiv(a.n, PRS::BN);
  {
    ProfScope ps(name, 2.0 * a.rows * a.k * a.n * a.s.n * PRS::NA, 2.0 * a.rows * a.k * PRS::NA + 4.0 * d.n * a.rows * a.n, st);
    TGP_LAUNCH(ps, (gated_out<PRS, T, true>), dim3((unsigned)a.tm * a.tn * d.n), dim3(PRS::T), 0, st, a);
  }
  ProfScope ps(name_join, 0, (4.0 * d.n + 2) * a.rows * a.n, st);
  TGP_LAUNCH(ps, gated_join<T>, dim3((unsigned)cdiv((long)a.rows * (a.ldp / 4), kT)), dim3(kT), 0, st, a, d.n);
}

HiddenArgs hidden_args(const Call& c, const Matrix& x, const Matrix& wg, const Matrix& wu, long rows) {
  const tgp_gated_shape& s = c.g.s;
  HiddenArgs a{};
  pairs(c.p.parts, c.p.parts, [&](int i, int j) {
    a.s.a[a.s.n][0] = x.part[i];
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

bool at16(const void* p, long ld, int size) { return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0; }

template <int P, int ACT, typename T>
void launch_narrow(const NarrowArgs& a, hipStream_t st) {
  ProfScope ps("gated_narrow", 2.0 * a.rows * a.hidden * (2 * a.cin + a.cout) * (P == 1 ? 1 : 6),
               2.0 * a.rows * (a.cin + a.cout), st);
  auto go = [&](auto ksx, auto nw, auto cg) {
    constexpr int KSX = decltype(ksx)::value, NW = decltype(nw)::value, CG = decltype(cg)::value;
    TGP_LAUNCH(ps, (gated_narrow<P, KSX, NW, CG, ACT, T>), dim3(cdiv(a.rows, 64)), dim3(64 * NW), 0, st, a);
  };
  typedef std::integral_constant<int, 2> two;
  typedef std::integral_constant<int, 4> four;
  typedef std::integral_constant<int, 8> eight;
  const int k = cdiv(a.cin, 64);
  // up to 128 channels four waves a block, of bfloat16 two blocks a CU: one's first loads
  // and activations beside the other's products (147456 x 64, 256 hidden channels: 51 us;
  // with h in one part 44, and so with eight waves 65)
  auto cols = [&](auto ksx) {
    if (a.cout <= 64) go(ksx, four(), two());
    else go(ksx, four(), four());
  };
  if constexpr (P == 1) {
    auto wide = [&](auto ksx) {
      if (a.cout <= 128) go(ksx, eight(), four());
      else go(ksx, eight(), eight());
    };
    if (k == 4) return wide(std::integral_constant<int, 4>());
    if (k == 3) return wide(std::integral_constant<int, 3>());
    if (a.cout > 128) return k == 1 ? go(std::integral_constant<int, 1>(), eight(), eight()) : go(two(), eight(), eight());
  }
  if (k == 1) cols(std::integral_constant<int, 1>());
  else cols(two());
}

template <typename T>
hipError_t forward_few(const Gated& g, const T* x, long ldx, T* y, long ldy, void* h, long ldh, hipStream_t st) {
  typedef std::conditional_t<sizeof(T) == 2, Pair, float> H;
  const tgp_gated_shape& s = g.s;
  const int rows = (int)g.rows, e = sizeof(T);
  const long plane = few_pixels(rows) * round_up(s.hidden, 16);
  auto width = [](int n) { return n >= 32 * 256 ? 32 : n >= 16 * 256 ? 16 : n >= 8 * 128 ? 8 : 4; };
  const FewArgs a{x, {g.w.gate, g.w.up}, {g.w.b_gate, g.w.b_up}, h, ldx, s.cin, ldh, rows, s.cin, s.hidden,
                  at16(x, ldx, e), at16(g.w.gate, s.cin, e) && at16(g.w.up, s.cin, e), width(s.hidden), plane};
  const FewArgs o{h, {g.w.down, nullptr}, {g.w.b_down, nullptr}, y, ldh, s.hidden, ldy, rows, s.hidden, s.cout,
                  at16(h, ldh, 4), at16(g.w.down, s.hidden, e), width(s.cout), plane};
  auto go = [&](auto mf) {
    constexpr int MF = decltype(mf)::value, NO = MF == 2 ? 8 : 16;   // (registers)
    with_act(s.act, [&](auto act) {
      ProfScope ps("gated_few_hidden", 4.0 * rows * s.cin * s.hidden, 2.0 * e * s.cin * s.hidden, st);
      TGP_LAUNCH(ps, (gated_few<T, T, H, 2, MF, 8, decltype(act)::value>), dim3(cdiv(s.hidden, a.cw)), dim3(512), 0, st, a);
    });
    ProfScope ps("gated_few_out", 2.0 * rows * s.cout * s.hidden, (double)e * s.cout * s.hidden, st);
    TGP_LAUNCH(ps, (gated_few<H, T, T, 1, MF, NO, 0>), dim3(cdiv(s.cout, o.cw)), dim3(64 * NO), 0, st, o);
  };
  if (few_pixels(rows) == 32) go(std::integral_constant<int, 1>());
  else go(std::integral_constant<int, 2>());
  return launch_status();
}

template <typename T>
hipError_t forward_t(const Gated& g, const T* x, long ldx, T* y, long ldy, void* ws, hipStream_t st) {
  constexpr int P = sizeof(T) == 2 ? 1 : 3, L = sizeof(T) == 2 ? 2 : 3;
  const tgp_gated_shape& s = g.s;
  Call c{g, plan_of(s, g.rows, false), (char*)ws, st};
  if (few(s, g.rows)) return forward_few<T>(g, x, ldx, y, ldy, (char*)ws + c.p.h, c.p.hidp, st);
  const Matrix wg = c.operand(g.w.gate, s.cin, s.hidden, s.cin, c.p.wg, s.hidden);
  const Matrix wu = c.operand(g.w.up, s.cin, s.hidden, s.cin, c.p.wu, s.hidden);
  const Matrix wd = c.operand(g.w.down, s.hidden, s.cout, s.hidden, c.p.wd, s.cout);
  const Matrix h = matrix_at(ws, c.p.h, L, c.p.chunk, c.p.hidp);
  for (long r0 = 0; r0 < g.rows; r0 += c.p.chunk) {
    const long rows = std::min(c.p.chunk, g.rows - r0);
    const Matrix xm = c.operand(x + r0 * ldx, ldx, rows, s.cin, c.p.x, c.p.chunk);
    if (hipError_t e = c.flush(); e != hipSuccess) return e;
    HiddenArgs a = hidden_args(c, xm, wg, wu, rows);
    if (narrow(s, g.rows)) {
      const NarrowArgs n{{xm.part[0], xm.part[1], xm.part[2]},
                         {{wg.part[0], wg.part[1], wg.part[2]}, {wu.part[0], wu.part[1], wu.part[2]}},
                         {wd.part[0], wd.part[1], wd.part[2]}, xm.ld, wg.ld, wd.ld, (int)rows, s.cin, s.hidden,
                         s.cout, a.bg, a.bu, g.w.b_down, y + r0 * ldy, ldy, at16(y + r0 * ldy, ldy, sizeof(T))};
      with_act(s.act, [&](auto act) { launch_narrow<P, decltype(act)::value, T>(n, st); });
      continue;
    }
    a.h = h;
    auto hidden = [&](auto pr, auto act) {
      typedef decltype(pr) PR;
      a.tm = cdiv(rows, PR::BM);
      a.tn = cdiv(s.hidden, PR::BN);
      ProfScope ps("gated_hidden", 4.0 * rows * s.cin * s.hidden * a.s.n, 2.0 * rows * (s.cin + L * s.hidden), st);
      TGP_LAUNCH(ps, (gated_hidden<PR, decltype(act)::value, L>), dim3((unsigned)a.tm * a.tn), dim3(PR::T), 0, st, a);
    };
    with_act(s.act, [&](auto act) {
      if (fills(rows, s.hidden)) hidden(HidL(), act);
      else hidden(HidS(), act);
    });
    OutArgs o{};
    add_sum<T>(&o, h, wd);
    o.lda = h.ld;
    o.ldb = wd.ld;
    o.rows = (int)rows;
    o.k = s.hidden;
    o.n = s.cout;
    o.bias = g.w.b_down;
    o.y = y + r0 * ldy;
    o.ldy = ldy;
    o.vec = at16(o.y, ldy, sizeof(T));
    launch_sum<false, T>("gated_out", "gated_out_join", o, (char*)ws + c.p.join, st);
  }
  return launch_status();
}

template <typename T>
hipError_t backward_t(const Gated& g, const T* dy, long lddy, const T* x, long ldx, T* dx, long lddx,
                      const tgp_gated_grads& gr, bool overwrite, void* ws, hipStream_t st) {
  constexpr int P = sizeof(T) == 2 ? 1 : 3, L = 3;
  const tgp_gated_shape& s = g.s;
  const bool grads = gr.gate || gr.up || gr.down || gr.b_gate || gr.b_up || gr.b_down;
  Call c{g, plan_of(s, g.rows, true), (char*)ws, st};
  const Plan& p = c.p;
  const Matrix wg = c.operand(g.w.gate, s.cin, s.hidden, s.cin, p.wg, s.hidden);
  const Matrix wu = c.operand(g.w.up, s.cin, s.hidden, s.cin, p.wu, s.hidden);
  const Matrix wd = c.operand(g.w.down, s.hidden, s.cout, s.hidden, p.wd, s.cout);
  const Matrix h = matrix_at(ws, p.h, L, p.chunk, p.hidp), dg = matrix_at(ws, p.dg, L, p.chunk, p.hidp),
               du = matrix_at(ws, p.du, L, p.chunk, p.hidp);
  auto add_up = [&](SumArgs& m) {
    const bool deep = m.ranges >= 8;
    int sb = 0;
    for (int k = 0; k < m.jobs; ++k) {
      m.j[k].blk0 = sb;
      sb += cdiv((long)m.j[k].rows * (m.j[k].ldp / 4), deep ? 64 : 256);
    }
    ProfScope ps("gated_sum", 0, 4.0 * m.ranges * p.stride, st);
    if (deep) TGP_LAUNCH(ps, gated_sum<4>, dim3((unsigned)sb), dim3(256), 0, st, m);
    else TGP_LAUNCH(ps, gated_sum<1>, dim3((unsigned)sb), dim3(256), 0, st, m);
  };
  for (long r0 = 0; r0 < g.rows; r0 += p.chunk) {
    const long rows = std::min(p.chunk, g.rows - r0);
    const Matrix xm = c.operand(x + r0 * ldx, ldx, rows, s.cin, p.x, p.chunk);
    const Matrix dym = c.operand(dy + r0 * lddy, lddy, rows, s.cout, p.dy, p.chunk);
    if (hipError_t e = c.flush(); e != hipSuccess) return e;
    if constexpr (sizeof(T) == 2) {
      if (p.slim) {
        SumArgs m{};
        m.ranges = ranges_of(rows, p.per);
        m.stride = p.stride;
        m.add = !overwrite || r0 > 0;
        const bool direct = p.ranges == 1;
        float* at = (float*)((char*)ws + p.part);
        auto sink = [&](int rows_w, int cols_w, float* w, float* b) {
          const int ldp = (int)round_up(cols_w, 4);
          const Sink t = direct ? Sink{w, b, cols_w, cols_w, at16(w, cols_w, 4)}
                                : Sink{w ? at : nullptr, b ? at + (long)rows_w * ldp : nullptr, ldp, cols_w, 1};
          if (w) m.j[m.jobs++] = {t.part, w, rows_w, cols_w, ldp, 0};
          if (b) m.j[m.jobs++] = {t.cols, b, 1, rows_w, (int)round_up(rows_w, 4), 0};
          at += (long)rows_w * ldp + round_up(rows_w, 4);
          return t;
        };
        SlimArgs a{xm.part[0], dym.part[0], wg.part[0], wu.part[0], wd.part[0], xm.ld, dym.ld, wg.ld, wd.ld, (int)rows,
                   p.per, s.cin, s.hidden, s.cout, g.w.b_gate, g.w.b_up, {}, p.stride, direct && m.add,
                   dx ? dx + r0 * lddx : nullptr, lddx, 0};
        a.vec = at16(a.dx, lddx, 2);
        a.to[0] = sink(s.hidden, s.cin, gr.gate, gr.b_gate);
        a.to[1] = sink(s.hidden, s.cin, gr.up, gr.b_up);
        a.to[2] = sink(s.cout, s.hidden, gr.down, gr.b_down);
        with_act(s.act, [&](auto act) {
          ProfScope ps("gated_slim", 2.0 * rows * (12 * s.cin + 4 * s.cout) * s.hidden,
                       2.0 * rows * (2 * s.cin + s.cout) + 4.0 * m.ranges * p.stride, st);
          constexpr int ACT = decltype(act)::value;
          if (grads) TGP_LAUNCH(ps, (gated_slim<ACT, true>), dim3((unsigned)m.ranges), dim3(512), 0, st, a);
          else TGP_LAUNCH(ps, (gated_slim<ACT, false>), dim3((unsigned)m.ranges), dim3(512), 0, st, a);
        });
        if (grads && !direct) add_up(m);
        continue;
      }
    }
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
      ProfScope ps("gated_back", 2.0 * rows * (2 * s.cin + s.cout) * s.hidden * a.s.n, 2.0 * rows * (s.cin + s.cout + 3 * L * s.hidden), st);
      constexpr bool ALL = decltype(all)::value;
      TGP_LAUNCH(ps, (gated_back<PR, decltype(pd), decltype(act)::value, ALL ? L : sizeof(T) == 2 ? 2 : 3, ALL>),
                 dim3((unsigned)a.tm * a.tn), dim3(PR::T), 0, st, a);
    };
    with_act(s.act, [&](auto act) {
      if (fills(rows, s.hidden)) {
        if (grads) back(BackL(), DhL(), act, std::true_type());
        else back(BackL(), DhL(), act, std::false_type());
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
      const bool direct = p.ranges == 1;
      o.add = direct && m.add;
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
          J.tm = cdiv(rows_w, p.wide);
          J.tn = w ? cdiv(cols_w, p.wide) : 1;   // the column sums alone: the first columns
          J.blk0 = blocks;
          int bit = 0;
          pairs(nu, nv, [&](int, int k) { J.sums |= (b && k == 0) << bit++; });
          J.part = at;
          J.cols = at + (long)rows_w * ldp;
          J.vec = 1;
          blocks += J.tm * J.tn * m.ranges;
          if (direct) {
            J.part = w;
            J.cols = b;
            J.ldp = cols_w;
            J.vec = at16(w, cols_w, 4);
            return;
          }
          if (w) m.j[m.jobs++] = {J.part, w, rows_w, cols_w, ldp, 0};
          if (b) m.j[m.jobs++] = {J.cols, b, 1, rows_w, (int)round_up(rows_w, 4), 0};
        }
        at += (long)rows_w * ldp + round_up(rows_w, 4);
      };
      job(dg, L, s.hidden, xm, P, s.cin, gr.gate, gr.b_gate);
      job(du, L, s.hidden, xm, P, s.cin, gr.up, gr.b_up);
      job(dym, P, s.cout, h, L, s.hidden, gr.down, gr.b_down);
      {
        ProfScope ps("gated_outer", 2.0 * rows * (2 * s.cin + s.cout) * s.hidden * o.j[0].s.n, 2.0 * rows * (s.cin + s.cout + 3 * L * s.hidden), st);
        if (p.wide == 64) TGP_LAUNCH(ps, gated_outer<OuterS>, dim3((unsigned)blocks), dim3(OuterS::T), 0, st, o);
        else if (p.wide == 128) TGP_LAUNCH(ps, gated_outer<OuterL>, dim3((unsigned)blocks), dim3(OuterL::T), 0, st, o);
        else TGP_LAUNCH(ps, gated_outer<OuterX>, dim3((unsigned)blocks), dim3(OuterX::T), 0, st, o);
      }
      if (!direct) add_up(m);
    }
    if (dx) {   // last: it may be written over x or dy
      OutArgs o{};
      add_sum<T>(&o, dg, wg);
      add_sum<T>(&o, du, wu);
      o.lda = p.hidp;
      o.ldb = wg.ld;
      o.rows = (int)rows;
      o.k = s.hidden;
      o.n = s.cin;
      o.y = dx + r0 * lddx;
      o.ldy = lddx;
      o.vec = at16(o.y, lddx, sizeof(T));
      launch_sum<true, T>("gated_dx", "gated_dx_join", o, (char*)ws + p.join, st);
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
      TGP_LAUNCH(ps, gated_zero, dim3((unsigned)((a.second + kT - 1) / kT)), dim3(kT), 0, st, a.first, a.second);
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
