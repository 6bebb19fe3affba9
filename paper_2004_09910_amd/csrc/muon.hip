// Orthogonalised updates of weight matrices: momentum, then Newton-Schulz
// products that bring the singular values of X near one.
//
// With m the shorter and n the longer side of a matrix, X is held m x n (a
// matrix of more rows than columns transposed), in float16 at a fixed scale,
// padded with zeros to multiples of 128.  All matrices lie in panels of 32
// columns, a panel's rows (64 bytes) one after the other: what a product's
// stage takes of an operand, 32 sum values of some rows or 32 sum rows of
// some panels, is then contiguous in pieces of 1 KiB and more.  One step is
//
//   A = X X^T          P = a I + b A + c A A          X' = P X
//
// launches over the tiles of all matrices, of A and P the upper ones only.  A
// and P are float16 with the rounding error of their diagonals beside them in
// float32: near convergence A is nearly a multiple of I, whose one rounding
// would shift every singular value alike and be multiplied by b / p(1) = 7.  A
// product of two such matrices (L + dL)(R + dR), dL and dR diagonal, is taken as
// L R + dL R + L dR.
//
// X itself is kept to 19 bits until two steps are left: what rounding it to
// float16 leaves out lies beside it (xl), in 8 bits a value.  Rounding X adds
// directions that U does not have at 2^-12 of it, and five steps multiply what is
// near zero by a^5 = 485: alone, float16 would leave an update of a rank-one U
// 0.14 of its norm off, of rank 8 0.035, of singular values that fall as 1 / k^2
// 0.02.  Those directions see P(0) = a I, so P X = P Xh + a xl is all the second
// part takes, one value at a time; in directions that U has, where P is less
// than a, this turns X's right side by about 2^-12 and is not multiplied.  With
// three steps left, when most singular values are near one and little
// multiplying is to come, P's own diagonal stands for it: nearly p I for a U of
// full rank, nearly a I for one of few directions.  Rounding A and P multiplies X
// by I + E from the left, which turns the update by |E| whatever the singular
// values.  Over spectra from flat to rank one, ranges of 2^14 and half of the
// singular values zero, 0.3 to 7e-3 of the update's norm is left beside its
// rounding to bfloat16, 1.7e-3.  xl costs two readings and two writings of a byte
// a value: 18 of 256 x 256 92 -> 95 us, 2048 x 18432 1113 -> 1167, a U-Net's 19
// matrices 544 -> 613 (with 16 bits a value 643).
//
// Two steps at once, for long matrices: X'' = P(A') P(A) X, and as P(A) and A
// commute, A' = X' X'^T = P A P.  That replaces the first step's product with X
// and the second's X X^T, 3 m^2 n operations, by four products of m x m
// matrices, 4 m^3.  (More than two at once would take fewer still, but A's
// eigenvalues span the square of X's range, which P^2 stretches 12-fold a
// step: three at once lose small singular values to float16's 11 bits, 8e-3
// of the update's norm where two leave 1.5e-3.)
//
// Five steps of one 2048 x 18432 take 1167 us, of a U-Net's 19 matrices of up
// to 1024 x 9216 613 us, of 18 of 256 x 256 95 us, of four of up to 16 x 144 15
// us: operations at 1256 TFLOP/s, what a large matrix product of float16
// reaches here, are 629, 182 and 5 us of that, the tensors' bytes 98, 81 and 2.
#include <algorithm>
#include <type_traits>

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
constexpr int kMaxMats = 20;       // matrices of one launch
constexpr int kFirstT = 768;       // threads of the first launch's blocks

struct Mat {
  const float* grad;
  float* mom;
  bf16_t* out;
  double* norm;        // partial sums of |U|^2
  f16 *x[2], *s[3];    // X (mp x np, ping-pong; then xl, bytes), A, P and their products (mp x mp)
  float* d[3];         // their diagonals' rounding errors
  float* part;         // partial tiles of A, of `split` ranges of its sum (1: none)
  int rows, cols, m, n, mp, np, norm_blocks, norm_per, split;
  int two;             // takes two steps at a time
  // one block's: no blocks of the other launches, and nothing but the addresses
  // and rows .. n set
  __host__ __device__ bool whole() const { return norm_blocks == 0; }
  __device__ unsigned char* xl() const { return (unsigned char*)(x[1] + (long)mp * np); }
};

// The matrices of a list and, for each kind of launch, the first block of each
// (and the number of blocks).  The first launch gets it as an argument and
// leaves it in the workspace for the others: arguments lie in host memory,
// which every block would have to reach for.
enum {
  L_MOMENTUM, L_NORMALIZE, L_GRAM, L_SUM, L_SYM, L_APPLY,   // every matrix
  L_GRAM1, L_SUM1, L_APPLY1,                                // those of one step at a time
  L_SYM2,                                                   // those of two
  LAUNCHES
};
struct Mats {
  int count;
  int blk0[LAUNCHES][kMaxMats + 1];
  Mat t[kMaxMats];
};
static_assert(sizeof(Mats) <= 3800, "kernel arguments");

// An argument of a launch: for matrices of one step at a time, and of two.
struct Each {
  int v[2];
};

// What a product P X does about xl, likewise: the factor of xl (0: X has none;
// P_DIAGONAL: P's diagonal), and whether X' gets one.
constexpr float P_DIAGONAL = -1.f;
struct EachLow {
  float factor[2];
  int out[2];
};
// An X with `left` steps to come, and its product of the next `take` of them.  The
// rounding of an X with two steps left is multiplied by a^2 at most: 1.7e-3.
__host__ __device__ __forceinline__ bool keeps_low(int left) { return left >= 3; }
__host__ __device__ __forceinline__ float low_factor(int left, int take) {
  return !keeps_low(left) ? 0.f : left == 3 ? P_DIAGONAL : take == 2 ? kA * kA : kA;
}

// Place of row i, column j of a matrix of mp rows.
__device__ __forceinline__ long at(int mp, int i, int j) { return ((long)(j >> 5) * mp + i) * 32 + (j & 31); }

// The matrix that block blk of a launch works on: the last to start at or
// before it.
__device__ __forceinline__ int find(const Mats* l, int launch, int blk) {
  const int lane = threadIdx.x & 63;
  const bool at_or_before = lane < l->count && l->blk0[launch][min(lane, kMaxMats)] <= blk;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(at_or_before)) - 1);
}

// A pointer read from the table, as one to global memory (else the compiler
// takes generic loads and stores).
template <typename T>
__device__ __forceinline__ T* gm(T* p) {
  return (T*)(__attribute__((address_space(1))) T*)(uintptr_t)p;
}

__device__ __forceinline__ float update_of(const Mat& t, long i, float mu, int nesterov) {
  const float g = gm(t.grad)[i];
  if (!gm(t.mom)) return g;
  return nesterov ? g + mu * gm(t.mom)[i] : gm(t.mom)[i];
}

// The update at N x 4 values, each four from a multiple of four on and inside
// (in[]), else zeros.  All loads at once, without a branch between them (where
// there is no momentum, the gradient's again): taken one by one they left
// 2048 x 18432 at 86 us.
template <int N>
__device__ __forceinline__ void update4(const Mat& t, const long (&at)[N], const bool (&in)[N], float mu, int nesterov,
                                        float4 (&u)[N]) {
  const float* gp = gm(t.grad);
  const bool mom = gm(t.mom) != nullptr;
  const float* mp = mom ? (const float*)gm(t.mom) : gp;
  float4 m[N];
#pragma unroll
  for (int z = 0; z < N; ++z) u[z] = *(const float4*)(gp + (in[z] ? at[z] : 0));
#pragma unroll
  for (int z = 0; z < N; ++z) m[z] = *(const float4*)(mp + (in[z] ? at[z] : 0));
  auto one = [&](bool in, float g, float m) {
    return !in ? 0.f : !mom ? g : nesterov ? g + mu * m : m;
  };
#pragma unroll
  for (int z = 0; z < N; ++z)
    u[z] = make_float4(one(in[z], u[z].x, m[z].x), one(in[z], u[z].y, m[z].y), one(in[z], u[z].z, m[z].z),
                       one(in[z], u[z].w, m[z].w));
}

// Sum over the first launch's threads (the same value in all of them).
__device__ __forceinline__ double first_sum(double s, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
#pragma unroll
  for (int w = 0; w < kFirstT / 64; ++w) s += sh[w];
  return s;
}

// Sum over the block's 256 threads (the same value in all of them).
__device__ __forceinline__ double block_sum(double s, double* sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// Leaves the argument in the workspace, by one block.
__device__ __forceinline__ void leave_table(const Mats& l, Mats* table) {
  for (int i = threadIdx.x; i < (int)(sizeof(Mats) / 4); i += kFirstT) ((int*)table)[i] = ((const int*)&l)[i];
}

// M = mu M + G, and partial sums of U^2 (in float64: squares of float32 values
// neither overflow nor vanish), block blk's of the launch.  Memory bounds it:
// 16-byte accesses, two of each tensor in flight a thread (2048 x 18432, 453 MB:
// 78 us, 5.8 TB/s).
__device__ __forceinline__ void momentum(const Mats& l, int blk, float mu, int nesterov, double* sh) {
  const int k = find(&l, L_MOMENTUM, blk);
  const Mat& t = l.t[k];
  const int b = blk - l.blk0[L_MOMENTUM][k];
  const long N = (long)t.rows * t.cols, N4 = N / 4, step = (long)t.norm_blocks * kFirstT;
  const float4* g4 = (const float4*)gm(t.grad);
  float4* m4 = (float4*)gm(t.mom);
  double s = 0;
  auto one = [&](float g, float& m) {
    float u = g;
    if (m4) {
      m = mu * m + g;
      u = nesterov ? g + mu * m : m;
    }
    s += (double)u * u;
  };
  for (long i = (long)b * kFirstT + threadIdx.x; i < N4; i += 2 * step) {
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
    float m = gm(t.mom) ? gm(t.mom)[e] : 0.f;
    one(gm(t.grad)[e], m);
    if (gm(t.mom)) gm(t.mom)[e] = m;
  }
  s = first_sum(s, sh);
  if (threadIdx.x == 0) gm(t.norm)[b] = s;
}

// The first launch of a list without matrices that one block does whole.
__global__ __launch_bounds__(kFirstT) void muon_momentum(Mats l, Mats* table, float mu, int nesterov) {
  __shared__ double sh[kFirstT / 64];
  if (blockIdx.x == 0) leave_table(l, table);
  momentum(l, blockIdx.x, mu, nesterov, sh);
}

// What rounding four values to float16s of X leaves out, as a word of xl.  A
// float32 has 13 bits of mantissa more than a float16: as integers the value and
// its float16 are at most 2^12 apart (but near zero, under 2^-25 of |U|, where as
// much as that is kept), of which the upper 8 bits of 13 are a byte.
__device__ __forceinline__ unsigned low4(const float* v) {
  unsigned w = 0;
#pragma unroll
  for (int z = 0; z < 4; ++z) {
    const int off = __float_as_int(v[z]) - __float_as_int((float)(f16)v[z]);
    w |= (unsigned)(min(max(off, -4096), 4095) + 4096) >> 5 << (8 * z);
  }
  return w;
}
// Value z of such a word beside the float16 h (the middle of what the byte
// stands for).
__device__ __forceinline__ float low_of(unsigned w, int z, float h) {
  return __int_as_float(__float_as_int(h) + (int)((w >> (8 * z) & 255u) << 5) + (16 - 4096)) - h;
}

// What U is multiplied by for X: kSX / norm, a factor that may pass float32's
// range, as a power of two, which is exact, and the rest.  A zero matrix stays
// zero.  The product is a float32, out of the compiler's sight: taken together
// with its rounding to float16 in one place and not in another, X and xl would
// differ by a whole unit where it lies halfway between two.
struct Scale {
  float rest;
  int two;
  __device__ __forceinline__ explicit Scale(double norm) {
    rest = (float)frexp(norm > 0 || norm != norm ? kSX / norm : 0.0, &two);
  }
  __device__ __forceinline__ float operator()(float u) const {
    float x = ldexpf(u, two) * rest;
    asm("" : "+v"(x));
    return x;
  }
};

// X = U / (|U| + eps) as float16, norm_per pieces of 4096 values a block, zeros
// in the padding: a piece is 64 rows x 64 columns through LDS where the matrix
// is transposed, else 32 rows x 128 columns.  Memory bounds it: U is read once
// more, as |U| is known only when all of it has been (2048 x 18432, 415 MB: 78 us,
// 5.3 TB/s).  keep: X gets its xl.
__global__ __launch_bounds__(256) void muon_normalize(const Mats* __restrict__ l, float mu, int nesterov, float eps,
                                                      int keep) {
  __shared__ double sh[4];
  __shared__ float tile[64][65];
  const int k = find(l, L_NORMALIZE, blockIdx.x);
  const Mat& t = l->t[k];
  const bool flip = t.rows > t.cols;
  double s = 0;
  for (int q = threadIdx.x; q < t.norm_blocks; q += 256) s += gm(t.norm)[q];
  // the sums' barriers come after the loads of the first piece
  Scale scale(0);
  auto set_scale = [&]() { scale = Scale(sqrt(block_sum(s, sh)) + eps); };
  auto put = [&](int i, int j, const float* f) {
    f16x8 h;
    float x[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      x[v] = scale(f[v]);
      h[v] = (f16)x[v];
    }
    *(f16x8*)(gm(t.x[0]) + at(t.mp, i, j)) = h;
    if (keep) *(uint2*)(gm(t.xl()) + at(t.mp, i, j)) = make_uint2(low4(x), low4(x + 4));
  };
  const int b0 = (blockIdx.x - l->blk0[L_NORMALIZE][k]) * t.norm_per;
  for (int b = b0; b < b0 + t.norm_per; ++b) {
    if (flip) {
      const int nt = t.np / 64, i0 = b / nt * 64, j0 = b % nt * 64;
      // four values of a row at once where their addresses allow it: 16 rows of
      // the matrix a turn, else 4 (9216 x 1024: 25 us, 40)
      if (t.cols % 4 == 0) {
        float4 u[4];
        const int c = i0 + threadIdx.x % 16 * 4;
        long src[4];
        bool in[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const int r = j0 + 16 * z + threadIdx.x / 16;
          src[z] = (long)r * t.cols + c;
          in[z] = r < t.rows && c < t.cols;
        }
        update4(t, src, in, mu, nesterov, u);
        if (b == b0) set_scale();
        __syncthreads();   // the previous piece has been read
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          float* to = &tile[16 * z + threadIdx.x / 16][threadIdx.x % 16 * 4];
          to[0] = u[z].x;
          to[1] = u[z].y;
          to[2] = u[z].z;
          to[3] = u[z].w;
        }
      } else {
        float u[16];
#pragma unroll
        for (int z = 0; z < 16; ++z) {
          const int r = j0 + z * 4 + (threadIdx.x >> 6), c = i0 + (threadIdx.x & 63);
          u[z] = r < t.rows && c < t.cols ? update_of(t, (long)r * t.cols + c, mu, nesterov) : 0.f;
        }
        if (b == b0) set_scale();
        __syncthreads();
#pragma unroll
        for (int z = 0; z < 16; ++z) tile[z * 4 + (threadIdx.x >> 6)][threadIdx.x & 63] = u[z];
      }
      __syncthreads();
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int i = threadIdx.x / 4, j = 32 * z + threadIdx.x % 4 * 8;
        float f[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) f[v] = tile[j + v][i];
        put(i0 + i, j0 + j, f);
      }
      continue;
    }
    const int nt = t.np / 128, i0 = b / nt * 32 + threadIdx.x / 16, j = b % nt * 128 + threadIdx.x % 16 * 8;
    float u[2][8];
    if (t.cols % 4 == 0) {
      float4 f[4];
      long src[4];
      bool in[4];
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const int i = i0 + z / 2 * 16, c = j + z % 2 * 4;
        src[z] = (long)i * t.cols + c;
        in[z] = i < t.rows && c < t.cols;
      }
      update4(t, src, in, mu, nesterov, f);
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        u[z / 2][z % 2 * 4] = f[z].x;
        u[z / 2][z % 2 * 4 + 1] = f[z].y;
        u[z / 2][z % 2 * 4 + 2] = f[z].z;
        u[z / 2][z % 2 * 4 + 3] = f[z].w;
      }
    } else {
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          const int i = i0 + 16 * z;
          u[z][v] = i < t.rows && j + v < t.cols ? update_of(t, (long)i * t.cols + j + v, mu, nesterov) : 0.f;
        }
    }
    if (b == b0) set_scale();
#pragma unroll
    for (int z = 0; z < 2; ++z) put(i0 + 16 * z, j, u[z]);
  }
}

// ------------------------------------------------- products

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b),
                                                c, 0, 0, 0);
}

// The tile product of a block: WM x WN waves, each MT x NT fragments of 32 x
// 32, over stages of U panels (32 sum values each) in a ring of NS LDS slots.
// L is BM rows from row i0 on, contiguous in the sum, R BN rows from j0 on
// likewise; with TR, R is the 32 sum rows of BN columns from j0 on, and its
// fragments are gathered by transpose loads.  A slot holds 64-byte rows, whose
// 16-byte chunks are XOR-swizzled.  With SWAP the accumulators hold the
// transposed tile: a lane has column (row with SWAP) l % 32 of a fragment and
// rows (columns) 8 (v / 4) + 4 (l / 32) + v % 4.
//
// A stage is visible to all waves one turn before it is multiplied, so that
// its fragments are read while the stage before it is (a step of 16 ahead, the
// 4 products of a 64 x 64 wave tile do not cover the reads: 8% of X X^T of 2048 x
// 18432).  With one fragment a wave a panel has
// two products, less than a turn's barrier and reads take: two panels a stage
// (18 of 256 x 256 100 -> 92 us, one of 1024 x 4096 210 -> 204).
template <int MT, int NT, int WM, int WN, int NS, int U, bool TR, bool SWAP>
struct Tile {
  static constexpr int NW = WM * WN, BM = 32 * MT * WM, BN = 32 * NT * WN;
  static constexpr int LCH = BM / 16, RCH = BN / 16;   // 1 KiB DMA chunks of a stage: 16 rows
  static constexpr int CH = LCH + RCH, SB = U * CH * 1024, PER = U * CH / NW;
  static_assert(LCH % NW == 0 && RCH % NW == 0 && NS * SB <= 160 * 1024, "whole DMA rounds, LDS ring");
  static_assert(NS >= 3, "a stage ahead");

  static constexpr int NL = LCH / NW, NR = RCH / NW;   // chunks of L and R a wave

  f32x16 acc[MT][NT];

  // Chunk q's slot in row `row`: sixteen rows read at one chunk, four each of
  // any remainder by 4, and (TR) half rows of four consecutive rows, hit
  // distinct banks (256 bytes).
  __device__ __forceinline__ static int kswz(int row, int q) { return q ^ ((row >> 2) & 3); }
  __device__ __forceinline__ static int rswz(int row, int q) { return q ^ (row & 2); }

  // L and R: matrices of lrows and rrows rows, R of rcols columns (what a TR
  // tile has beyond them reads as zeros); stages k0 .. k1 (one at least) of the
  // sum.
  __device__ __forceinline__ void run(unsigned char* ring, const f16* L, int lrows, int i0, const f16* R,
                                      int rrows, int rcols, int j0, int k0, int k1) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // what comes from a table in memory is the same in every lane
    k0 = __builtin_amdgcn_readfirstlane(k0);
    k1 = __builtin_amdgcn_readfirstlane(k1);
    const u32x4 rl = uniform(make_rsrc(L + (long)i0 * 32, 0x7fffffff));
    const u32x4 rr = uniform(TR ? make_rsrc(R + (long)j0 * rrows, (rcols - j0) * rrows * 2)
                                : make_rsrc(R + (long)j0 * 32, 0x7fffffff));
    // byte offsets of this lane in its chunks of a stage (rows of chunks NW
    // apart agree in their swizzle, NW being even), and of the next stage
    static_assert(NW % 2 == 0, "pairs of chunks");
    const int r16 = wave * 16 + (lane >> 2), rrow = (wave & 1) * 16 + (lane >> 2);
    int vl[3] = {}, vr[3] = {};
#pragma unroll
    for (int u = 0; u < NL; ++u) vl[u] = r16 * 64 + 16 * kswz(r16, lane & 3) + u * NW * 1024;
#pragma unroll
    for (int u = 0; u < NR; ++u)
      vr[u] = TR ? ((wave >> 1) + u * (NW / 2)) * rrows * 64 + rrow * 64 + 16 * rswz(rrow, lane & 3)
                 : r16 * 64 + 16 * kswz(r16, lane & 3) + u * NW * 1024;
    const int stl = __builtin_amdgcn_readfirstlane(lrows * 64);
    const int str = TR ? 2048 : __builtin_amdgcn_readfirstlane(rrows * 64);
    int sl = __builtin_amdgcn_readfirstlane(k0 * stl), sr = __builtin_amdgcn_readfirstlane(k0 * str);
    const unsigned dst = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long)TGP_LDS(ring) + wave * 1024);
    auto issue = [&](auto slot) __attribute__((always_inline)) {
      each<U>([&](auto u) {
        issue_panel<decltype(slot)::value * SB + decltype(u)::value * CH * 1024>(dst, vl, vr, rl, rr, sl, sr);
        sl += stl;
        sr += str;
      });
    };
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x16{};
    const int total = (k1 - k0) / U;
    // fragments of two stages in turn: those of the next are read while this
    // one's are multiplied
    u32x4 a[2][2 * U][MT], b[2][2 * U][NT];
    const int fr = lane & 31;                                   // row of a fragment
    const int kb = 8 * (lane >> 5) + ((lane & 15) >> 2);        // (TR) row of the transpose load
    const int cb = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);   // (TR) its chunk
    const int la = (wm * MT * 32 + fr) * 64 + kswz(fr, lane >> 5) * 16;
    const int lb = LCH * 1024 + (TR ? wn * NT * 2048 + kb * 64 + rswz(kb, cb) * 16 + 8 * (lane & 1)
                                    : (wn * NT * 32 + fr) * 64 + kswz(fr, lane >> 5) * 16);
    auto load = [&](auto slot, int z) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2 * U; ++h) {
        const unsigned char* s = ring + decltype(slot)::value * SB + h / 2 * CH * 1024;
#pragma unroll
        for (int i = 0; i < MT; ++i) a[z][h][i] = *(const u32x4*)(s + (la ^ (32 * (h & 1))) + i * 2048);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if constexpr (TR) b[z][h][j] = frag_tr(s + lb + j * 2048 + (h & 1) * 1024, 64);
          else b[z][h][j] = *(const u32x4*)(s + (lb ^ (32 * (h & 1))) + j * 2048);
        }
      }
    };
    each<NS - 1>([&](auto k) {
      if (decltype(k)::value < total) issue(k);
    });
    wait_stages<NS, PER>(min(NS - 2, total - 1));
    ring_barrier();
    load(std::integral_constant<int, 0>(), 0);
    // Stage idx (slot Z).  At its barrier stage idx + 1 has landed, for every
    // wave, and slot idx - 1 has been read.  A wave issues an instruction every
    // few clocks, so what surrounds the products is kept to a handful: slots
    // are constants, and addresses advance by two additions.  STEADY: the stage
    // to be issued exists.
    auto turn = [&](int idx, auto zc, auto steady) __attribute__((always_inline)) {
      constexpr int Z = decltype(zc)::value;
      constexpr bool STEADY = decltype(steady)::value;
      if constexpr (STEADY) wait_vmcnt<(NS - 3) * PER>();
      else wait_stages<NS - 1, PER>(min(NS - 3, total - 2 - idx));
      ring_barrier();
      if (STEADY || idx + NS - 1 < total) issue(std::integral_constant<int, (Z + NS - 1) % NS>());
      if (STEADY || idx + 1 < total) load(std::integral_constant<int, (Z + 1) % NS>(), (Z + 1) % 2);
#pragma unroll
      for (int h = 0; h < 2 * U; ++h)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            acc[i][j] = SWAP ? mfma(b[Z % 2][h][j], a[Z % 2][h][i], acc[i][j])
                             : mfma(a[Z % 2][h][i], b[Z % 2][h][j], acc[i][j]);
      // reads between the products
      if constexpr (STEADY) {
        constexpr int MF = 2 * U * MT * NT, RD = 2 * U * (MT + (TR ? 2 : 1) * NT), PM = (RD + MF - 1) / MF;
#pragma unroll
        for (int m = 0; m < MF; ++m) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);    // a product
          __builtin_amdgcn_sched_group_barrier(0x100, PM, 0);   // LDS reads
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(NS % 2 == 0, "fragment buffers in turn");
    int idx = 0;
    for (; idx + 2 * NS - 1 <= total; idx += NS)
      each<NS>([&](auto z) { turn(idx + decltype(z)::value, z, std::true_type()); });
    for (; idx < total; idx += NS)
      each<NS>([&](auto z) {
        if (idx + decltype(z)::value < total) turn(idx + decltype(z)::value, z, std::false_type());
      });
  }

 private:
  // The same in every lane, in scalar registers.
  __device__ __forceinline__ static u32x4 uniform(u32x4 v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __builtin_amdgcn_readfirstlane(v[k]);
    return v;
  }

  // f(0), f(1), .. f(N - 1), as constants
  template <int N, typename F>
  __device__ __forceinline__ static void each(F f) {
    if constexpr (N > 0) {
      each<N - 1>(f);
      f(std::integral_constant<int, N - 1>());
    }
  }

  // The wave's chunks of one stage, global to LDS at dst + AT, NW KiB apart:
  // L's at offsets vl + sl, then R's at vr + sr.  M0 holds the destination only
  // inside (as in dma16, one wait state between writing it and the load).
  template <int AT>
  __device__ __forceinline__ static void issue_panel(unsigned dst, const int (&vl)[3], const int (&vr)[3],
                                                     u32x4 rl, u32x4 rr, int sl, int sr) {
    unsigned saved;
#define TGP_FIRST "s_mov_b32 %0, m0\n\ts_add_u32 m0, %1, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 "
#define TGP_NEXT "s_add_u32 m0, m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 "
#define TGP_LAST "s_mov_b32 m0, %0"
#define TGP_OPS "=&s"(saved) : "s"(dst), "i"(AT), "i"(NW * 1024), "s"(rl), "s"(rr), "s"(sl), "s"(sr)
    if constexpr (NL == 1 && NR == 1)
      asm volatile(TGP_FIRST "%8, %4, %6 offen lds\n\t" TGP_NEXT "%9, %5, %7 offen lds\n\t" TGP_LAST
                   : TGP_OPS, "v"(vl[0]), "v"(vr[0]) : "memory", "scc");
    else if constexpr (NL == 2 && NR == 2)
      asm volatile(TGP_FIRST "%8, %4, %6 offen lds\n\t" TGP_NEXT "%9, %4, %6 offen lds\n\t"
                   TGP_NEXT "%10, %5, %7 offen lds\n\t" TGP_NEXT "%11, %5, %7 offen lds\n\t" TGP_LAST
                   : TGP_OPS, "v"(vl[0]), "v"(vl[1]), "v"(vr[0]), "v"(vr[1]) : "memory", "scc");
    else {
      static_assert(NL == 2 && NR == 3, "a tile of another shape");
      asm volatile(TGP_FIRST "%8, %4, %6 offen lds\n\t" TGP_NEXT "%9, %4, %6 offen lds\n\t"
                   TGP_NEXT "%10, %5, %7 offen lds\n\t" TGP_NEXT "%11, %5, %7 offen lds\n\t"
                   TGP_NEXT "%12, %5, %7 offen lds\n\t" TGP_LAST
                   : TGP_OPS, "v"(vl[0]), "v"(vl[1]), "v"(vr[0]), "v"(vr[1]), "v"(vr[2]) : "memory", "scc");
    }
#undef TGP_FIRST
#undef TGP_NEXT
#undef TGP_LAST
#undef TGP_OPS
  }
};

// The tile that block `blk` of n takes.  Workgroups are dealt round-robin over
// the 8 XCDs, each with its own L2: sixteen consecutive tiles, which share a
// panel of X, go to one XCD, and every 128 tiles are spread over all of them,
// since tiles of one launch differ in length (a contiguous eighth for each XCD
// leaves some with the long ones).  A U-Net's 19 matrices: X X^T 43 us and P X 62,
// 50 and 73 in the blocks' own order.
__device__ __forceinline__ int grouped(int blk, int n) {
  const int w = blk & ~127, r = blk & 127;
  return w + 128 <= n ? w + (r & 7) * 16 + (r >> 3) : blk;
}

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

typedef f16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned pack_f16(float a, float b) {
  const f16x2 v = {(f16)a, (f16)b};
  return __builtin_bit_cast(unsigned, v);
}

// Words of groups 0, 2, 1, 3 of 8 columns (4 of them in lane l, 4 in lane l + 32)
// to the words of 16 consecutive columns, 0 .. 15 in lane l and 16 .. 31 in lane
// l + 32, and back.
__device__ __forceinline__ u32x4 swap16(u32x4 v) {
  // (a word's upper half of the wave changes places with the lower half of the
  // word of the group two on)
  const auto a = __builtin_amdgcn_permlane32_swap(v[0], v[1], false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(v[2], v[3], false, false);
  return u32x4{a[0], a[1], b[0], b[1]};
}

__device__ __forceinline__ f32x4_t from_f16(const f16* p) {
  typedef f16 f16x4 __attribute__((ext_vector_type(4)));
  return __builtin_convertvector(*(const f16x4*)p, f32x4_t);
}

// Of a fragment on the diagonal (f[g][z]: row 8 g + 4 (l / 32) + z, column l %
// 32), this lane's diagonal element, if it has one (diagonal_here).
__device__ __forceinline__ bool diagonal_here() { return ((threadIdx.x >> 5) & 1) == ((threadIdx.x >> 2) & 1); }
__device__ __forceinline__ float diagonal(const f32x4_t (&f)[4]) {
  // selects of values (a select of array elements is one of addresses, which
  // puts the array in memory)
  auto pick = [](bool second, float a, float b) { return second ? b : a; };
  const int z = threadIdx.x & 3, g = (threadIdx.x >> 3) & 3;
  float c[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    c[k] = pick(g & 2, pick(g & 1, f[0][k], f[1][k]), pick(g & 1, f[2][k], f[3][k]));
  return pick(z & 2, pick(z & 1, c[0], c[1]), pick(z & 1, c[2], c[3]));
}
// What rounding v to a stored float16 leaves out.
__device__ __forceinline__ float lost(float v) { return v - (float)(f16)(v * kSM) * (1.f / kSM); }

// Stores one 32 x 32 fragment of a symmetric matrix of mp rows at rows i0,
// columns j0, and its mirror image: eight consecutive rows of a column are
// eight columns of the mirror's row as they are, and eight columns of a row come
// by way of `lds` (2 KiB of this wave's).  value(g, i, j) is what elements 4 g ..
// 4 g + 3 (rows i .. i + 3, column j) become.  What is stored is the upper half
// and its mirror image in every place: of a tile on the diagonal the fragments
// above it, and of a fragment on it the elements.  A product of two matrices
// that commute but for rounding is symmetric but for rounding, and both halves as
// computed cost half of the accuracy there (64 x 576 with 32 singular values
// of 1 and 32 of 1 / 20: 8.3e-3 of the update's norm, 4.5e-3 so).
template <typename F>
__device__ __forceinline__ void store_sym(f16* m, float* d, int mp, int i0, int j0, unsigned char* lds, F value) {
  if (i0 > j0) return;
  const int lane = threadIdx.x & 63, hi = lane >> 5, fr = lane & 31, j = j0 + fr;
  unsigned pk[8];
  f32x4_t f[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    f[g] = value(g, i0 + 8 * g + 4 * hi, j);
    pk[2 * g] = pack_f16(f[g][0] * kSM, f[g][1] * kSM);
    pk[2 * g + 1] = pack_f16(f[g][2] * kSM, f[g][3] * kSM);
    // rows of 64 bytes, chunks swizzled so that neither the writes nor the
    // transpose reads meet in a bank more than they must
    *(uint2*)(lds + fr * 64 + (g ^ ((fr >> 2) & 3)) * 16 + 8 * hi) = make_uint2(pk[2 * g], pk[2 * g + 1]);
  }
  if (i0 == j0 && diagonal_here()) d[j] = lost(diagonal(f));
  u32x4 down[2];   // columns 16 h + 8 hi .. of row j
  put8(pk, [&](int h, u32x4 c) { down[h] = c; });
  const int kb = 8 * hi + ((lane & 15) >> 2), cb = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint2 v[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int row = 16 * h + kb + 4 * z;
      v[z] = lds_tr16(lds + row * 64 + (cb ^ ((row >> 2) & 3)) * 16 + 8 * (lane & 1));
    }
    u32x4 across = {v[0].x, v[0].y, v[1].x, v[1].y};   // those of row i0 + fr
    if (i0 != j0) {
      *(u32x4*)(m + at(mp, j, i0 + 16 * h + 8 * hi)) = down[h];
    } else {
      // the same row: its columns from the diagonal on are above it as they are,
      // those before it as mirror images
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int c = 16 * h + 8 * hi + 2 * w;
        const unsigned above = (fr <= c ? 0xffffu : 0u) | (fr <= c + 1 ? 0xffff0000u : 0u);
        across[w] = (across[w] & above) | (down[h][w] & ~above);
      }
    }
    *(u32x4*)(m + at(mp, i0 + fr, j0 + 16 * h + 8 * hi)) = across;
  }
}

__device__ __forceinline__ f32x4_t part_of(const f32x16& a, int g) {
  return f32x4_t{a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]};
}

// Row and column of tile b of the upper triangle (row <= column) of nt x nt
// tiles: bands of four rows, in a band the triangle on the diagonal, then
// squares of 4 x 4, whose sixteen tiles share eight panels.
__device__ __forceinline__ void upper(int b, int nt, int& r, int& c) {
  int r0 = 0, h = min(4, nt);
  for (int n; b >= (n = h * (h + 1) / 2 + h * (nt - r0 - h)); h = min(4, nt - r0)) {
    b -= n;
    r0 += 4;
  }
  const int tri = h * (h + 1) / 2;
  if (b >= tri) {   // only a band of four rows has columns beyond its triangle
    b -= tri;
    r = r0 + (b & 3);
    c = r0 + 4 + (b >> 2);
    return;
  }
  int k = 0;
  while (b >= h - k) b -= h - k++;
  r = r0 + k;
  c = r + b;
}

enum { GRAM, POLY, MUL };

// Symmetric products, upper tiles only.  GRAM: s[0] = x[a] x[a]^T; where its
// sum is split, the ranges' partial tiles go to t.part as the accumulators lie,
// [range][tile][wave][fragment][g][lane].  POLY: s[c] = a I + b A + c A A of A =
// s[0].  MUL: s[c] = s[a] s[b], of matrices that commute.
//
// GRAM in tiles of 128 x 128: 2048 x 18432 88 us, 930 TFLOP/s of the upper tiles;
// 408 blocks of two a CU leave some CUs one, and the clock is at 2.0 GHz.  POLY
// and MUL in tiles of 64 x 64 (2048: 22 and 23 us, 390 TFLOP/s) wait two thirds of
// their waves' cycles for stages and barriers, with the matrix instructions and
// LDS at a sixth each; 528 tiles are two a CU and three on some.  Tiles of 128 x
// 128 would be 136 for 256 CUs: slower before the stage loop was as it is, and not
// measured since.  Under about 1024 a launch and the latencies of
// a tile's first and last stage are most of it (256: 5 to 6 us).
template <int MODE, int MT, int NT, int WM, int WN, int NS, int U>
__global__ __launch_bounds__(64 * WM * WN, 2) void muon_sym(const Mats* __restrict__ l, int launch, Each ea, int b, Each ec) {
  typedef Tile<MT, NT, WM, WN, NS, U, false, false> TL;
  static_assert(TL::BM == TL::BN, "square tiles");
  __shared__ __attribute__((aligned(16))) unsigned char ring[NS * TL::SB];
  const int blk = grouped(blockIdx.x, gridDim.x);
  const int k = find(l, launch, blk);
  const Mat& t = l->t[k];
  const int a = MODE == POLY ? 0 : pickg(ea.v, t.two), c = pickg(ec.v, t.two);
  const int nt = t.mp / TL::BM, tiles = nt * (nt + 1) / 2;
  const int q = blk - l->blk0[launch][k], sp = MODE == GRAM ? q / tiles : 0;
  int ti, tj;
  upper(q - sp * tiles, nt, ti, tj);
  const int i0 = ti * TL::BM, j0 = tj * TL::BN, nk = (MODE == GRAM ? t.np : t.mp) / 32;
  // ranges of whole pairs of panels
  const int k0 = MODE == GRAM ? (int)(nk / 2L * sp / t.split) * 2 : 0;
  const int k1 = MODE == GRAM ? (int)(nk / 2L * (sp + 1) / t.split) * 2 : nk;
  const f16* L = MODE == GRAM ? gm(t.x[a]) : gm(t.s[a]);
  const f16* R = MODE == MUL ? gm(t.s[b]) : L;
  const float* dl = gm(t.d[a]);
  const float* dr = MODE == MUL ? gm(t.d[b]) : dl;
  f16* out = gm(t.s[c]);
  float* dout = gm(t.d[c]);
  const int wave = threadIdx.x >> 6, wi = i0 + wave / WN * MT * 32, wj = j0 + wave % WN * NT * 32;
  // L's and R's own elements of this wave's fragment (read where symmetry has
  // them) and their diagonals' errors, on their way while the sum runs
  static_assert(MODE == GRAM || MT * NT == 1, "one fragment's elements in registers");
  const int lane = threadIdx.x & 63, col = wj + (lane & 31);
  f32x4_t lv[4], rv[4], dlr[4];
  float dlc = 0.f, drc = 0.f;
  if constexpr (MODE != GRAM) {
    dlc = dl[col];
    drc = dr[col];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int r = wi + 8 * g + 4 * (lane >> 5);
      lv[g] = from_f16(L + at(t.mp, col, r)) * (1.f / kSM);
      rv[g] = MODE == POLY ? lv[g] : from_f16(R + at(t.mp, col, r)) * (1.f / kSM);
      dlr[g] = *(const f32x4_t*)(dl + r);
    }
  }
  TL tl;
  tl.run(ring, L, t.mp, i0, R, t.mp, 0, j0, k0, k1);
  ring_barrier();   // the ring is free
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const f32x16& acc = tl.acc[i][j];
      if (MODE == GRAM && t.split > 1) {
        f32x4_t* part = (f32x4_t*)gm(t.part) +
                        ((((long)q * WM * WN + wave) * MT + i) * NT + j) * 256 + (threadIdx.x & 63);
#pragma unroll
        for (int g = 0; g < 4; ++g) part[64 * g] = part_of(acc, g);
        continue;
      }
      store_sym(out, dout, t.mp, wi + 32 * i, wj + 32 * j, ring + wave * 2048,
                [&](int g, int r, int c) {
        if constexpr (MODE == GRAM) {
          return part_of(acc, g) * (1.f / (kSX * kSX));
        } else {
          f32x4_t p = part_of(acc, g) * (1.f / (kSM * kSM)) + dlr[g] * rv[g] + lv[g] * drc;
          if constexpr (MODE == POLY) p = kC * p + kB * lv[g];
          if (wi == wj)
#pragma unroll
            for (int z = 0; z < 4; ++z)
              if (r + z == c) p[z] += MODE == POLY ? kA + (kB + kC * drc) * dlc : dlc * drc;
          return p;
        }
      });
    }
}

// s[0] from the ranges' partial tiles, added in order: a wave takes one
// fragment.  Three ranges of 2048 x 2048: 8.5 us, 27 MB from the caches.
template <int MT, int NT, int WM, int WN>
__global__ __launch_bounds__(256) void muon_gram_sum(const Mats* __restrict__ l, int launch) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * 2048];
  const int k = find(l, launch, blockIdx.x);
  const Mat& t = l->t[k];
  constexpr int BM = 32 * MT * WM, FR = WM * WN * MT * NT;
  const int nt = t.mp / BM, tiles = nt * (nt + 1) / 2;
  const int f = (blockIdx.x - l->blk0[launch][k]) * 4 + (threadIdx.x >> 6), tile = f / FR, q = f % FR;
  const int lane = threadIdx.x & 63, wave = q / (MT * NT), i = q / NT % MT, j = q % NT;
  int ti, tj;
  upper(tile, nt, ti, tj);
  const f32x4_t* in = (const f32x4_t*)gm(t.part) + ((long)tile * FR + q) * 256 + lane;
  const long step = (long)tiles * FR * 256;
  f32x4_t acc[4] = {};
  for (int s = 0; s < t.split; ++s)
#pragma unroll
    for (int g = 0; g < 4; ++g) acc[g] += in[s * step + 64 * g];
  store_sym(gm(t.s[0]), gm(t.d[0]), t.mp, ti * BM + (wave / WN * MT + i) * 32, tj * BM + (wave % WN * NT + j) * 32,
            lds + (threadIdx.x >> 6) * 2048,
            [&](int g, int, int) { return acc[g] * (1.f / (kSX * kSX)); });
}

// Stores values of row r of X, columns c0 .. c0 + 31 (as the accumulators of a
// transposed fragment lie), as the update.
__device__ __forceinline__ void store_update(const Mat& t, int r, int c0, const float (&y)[16]) {
  const int hi = (threadIdx.x & 63) >> 5;
  const bool flip = t.rows > t.cols;
  if (!flip && t.cols % 8 == 0) {
    unsigned pk[8];
#pragma unroll
    for (int g = 0; g < 8; ++g) pk[g] = f2bf(y[2 * g]) | (f2bf(y[2 * g + 1]) << 16);
    put8(pk, [&](int h, u32x4 c) {
      const int cc = c0 + 16 * h + 8 * hi;
      if (r < t.m && cc < t.n) *(u32x4*)(gm(t.out) + (long)r * t.cols + cc) = c;
    });
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int c = c0 + 8 * (v / 4) + 4 * hi + v % 4;
      if (r < t.m && c < t.n) gm(t.out)[flip ? (long)c * t.cols + r : (long)r * t.cols + c] = (bf16_t)f2bf(y[v]);
    }
  }
}

// X' = s[p] X, or (last) the update itself.  In tiles of 128 x 192 it is bound
// by the clock that the matrix instructions' power leaves, 1.7 GHz, 58% of whose
// cycles they are busy: 2048 x 18432 147 us, 1050 TFLOP/s (the library's product
// of 2048 x 2048 x 18432: 155 us), and 163 where it reads and writes xl.
template <int MT, int NT, int WM, int WN, int NS, int U>
__global__ __launch_bounds__(64 * WM * WN, 2) void muon_apply(const Mats* __restrict__ l, int launch, Each ep, Each efrom, int last,
                                                              EachLow elow) {
  typedef Tile<MT, NT, WM, WN, NS, U, true, true> TL;
  __shared__ __attribute__((aligned(16))) unsigned char ring[NS * TL::SB];
  const int blk = grouped(blockIdx.x, gridDim.x);
  const int k = find(l, launch, blk);
  const Mat& t = l->t[k];
  const int p = pickg(ep.v, t.two), from = pickg(efrom.v, t.two);
  const int b = blk - l->blk0[launch][k], nt = t.mp / TL::BM;
  const int i0 = b % nt * TL::BM, j0 = b / nt * TL::BN;
  const f16* x = gm(t.x[from]);
  const float* dp = gm(t.d[p]);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // X's own elements of a wave with one fragment, on their way while the sum
  // runs; with more there are the others' products to hide them
  constexpr bool EARLY = MT * NT == 1;
  const float factor = pickg(elow.factor, t.two);
  const bool keep = pickg(elow.out, t.two);
  unsigned char* xl = gm(t.xl());
  f32x4_t xe[4];
  if constexpr (EARLY) {
    const int r = i0 + wave / WN * 32 + (lane & 31), c0 = j0 + wave % WN * 32;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      xe[g] = c0 < t.np ? from_f16(x + at(t.mp, r, c0 + 8 * g + 4 * (lane >> 5))) : f32x4_t{};
  }
  // xl of 16 columns of the lane's rows likewise
  u32x4 le[MT][NT] = {};
  if (factor != 0)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int r = i0 + (wave / WN * MT + i) * 32 + (lane & 31), c0 = j0 + (wave % WN * NT + j) * 32;
        if (c0 < t.np) le[i][j] = *(const u32x4*)(xl + at(t.mp, r, c0 + 16 * (lane >> 5)));
      }
  TL tl;
  tl.run(ring, gm(t.s[p]), t.mp, i0, x, t.mp, t.np, j0, 0, t.mp / 32);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int r = i0 + (wave / WN * MT + i) * 32 + (lane & 31);
    const float d = dp[r] * (1.f / kSX);
    const float pl = (factor == P_DIAGONAL ? (float)gm(t.s[p])[at(t.mp, r, r)] * (1.f / kSM) + dp[r] : factor) * (1.f / kSX);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int c0 = j0 + (wave % WN * NT + j) * 32;
      if (c0 >= t.np) continue;
      const u32x4 lv = swap16(le[i][j]);   // as the accumulators lie: a word of group 0, 2, 1, 3 of 8 columns
      const f32x16& acc = tl.acc[i][j];
      unsigned pk[8];
      float y[16];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4_t xv = EARLY ? xe[g] : from_f16(x + at(t.mp, r, c0 + 8 * g + 4 * (lane >> 5)));
#pragma unroll
        for (int z = 0; z < 4; ++z)
          y[4 * g + z] = acc[4 * g + z] * (1.f / (kSM * kSX)) + d * xv[z];
        if (factor != 0)
#pragma unroll
          for (int z = 0; z < 4; ++z) y[4 * g + z] += pl * low_of(lv[g >> 1 | (g & 1) << 1], z, xv[z]);
      }
      if (!last) {
#pragma unroll
        for (int g = 0; g < 8; ++g) pk[g] = pack_f16(y[2 * g] * kSX, y[2 * g + 1] * kSX);
        f16* out = gm(t.x[from ^ 1]);
        put8(pk, [&](int h, u32x4 c) { *(u32x4*)(out + at(t.mp, r, c0 + 16 * h + 8 * (lane >> 5))) = c; });
        if (keep) {   // in place: what this wave has read
#pragma unroll
          for (int v = 0; v < 16; ++v) y[v] *= kSX;
          *(u32x4*)(xl + at(t.mp, r, c0 + 16 * (lane >> 5))) =
              swap16(u32x4{low4(y), low4(y + 8), low4(y + 4), low4(y + 12)});
        }
      } else {
        store_update(t, r, c0, y);
      }
    }
  }
}

// ------------------------------------------------- small matrices, whole

// A matrix whose X fits in LDS: the whole update by one block of twelve waves,
// X, A and P staying in LDS (panels of 32 columns, a row's 64 bytes 80 apart:
// eight rows read at one chunk hit distinct banks).  MS: m rounded up to 32 or
// 64.  What bounds it is one CU's rate of loading and the latencies between its
// barriers, three a step: five steps of 16 x 144 take 14.8 us, of 64 x 256 24
// (without xl 12.9 and 20; there eight waves 20.5, sixteen 22.5), where four
// launches a step take 70 to 90.  LDS could hold an X of 55296 values.  A list of
// 64 x 576 alone took 33 us so, and 89 as tiles; but among other matrices such a
// block runs on after the launch that it shares, for longer than tiles take for
// one matrix more (six matrices of all sorts, one of them 1144 x 9: 177 us so,
// 149 as tiles).
constexpr int kSmallX = 16384, kRow = 80;   // most values of X, bytes of a row
// chunks of 8 values of a thread, and those whose loads are in flight together
constexpr int kSmallChunks = (kSmallX / 8 + kFirstT - 1) / kFirstT, kFlight = 2;

struct SmallLds {
  unsigned char xs[kSmallX / 32 * kRow];               // X
  unsigned char as[2 * 64 * kRow], pms[2 * 64 * kRow];   // A, P
  float da[64], dp[64];                                // their diagonals' errors
  double sh[kFirstT / 64];
};

// xl is in registers, where each wave needs it.
template <int MS>
__device__ __forceinline__ void small_update(SmallLds& lds, const Mat& t, float mu, int nesterov, int steps,
                                             float eps) {
  constexpr int Q = MS / 32, F = Q * Q;   // fragments of A's side and of A
  unsigned char *xs = lds.xs, *as = lds.as, *pms = lds.pms;
  float *da = lds.da, *dp = lds.dp;
  const int ns = (t.n + 31) / 32 * 32, chunks = MS * ns / 8;
  const bool flip = t.rows > t.cols, vec = !flip && t.cols % 4 == 0;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // U in registers: chunk z of this thread is 8 columns from j of row i
  auto place = [&](int z, int& i, int& j) {
    const int c = z * kFirstT + tid;
    if (flip) {
      i = c % MS;
      j = c / MS * 8;
    } else {
      i = c / (ns / 8);
      j = c % (ns / 8) * 8;
    }
    return c < chunks;
  };
  float u[kSmallChunks][8];
  double sum = 0;
#pragma unroll
  for (int z0 = 0; z0 < kSmallChunks; z0 += kFlight) {
    if (z0 * kFirstT >= chunks) break;
    float m[kFlight][8];
#pragma unroll
    for (int z = z0; z < min(z0 + kFlight, kSmallChunks); ++z) {
      int i, j;
#pragma unroll
      for (int v = 0; v < 8; ++v) u[z][v] = m[z - z0][v] = 0.f;
      if (!place(z, i, j) || i >= t.m) continue;
      if (vec && j + 8 <= t.n) {
        const float4* g = (const float4*)(gm(t.grad) + i * t.cols + j);
        const float4 g0 = g[0], g1 = g[1];
        u[z][0] = g0.x; u[z][1] = g0.y; u[z][2] = g0.z; u[z][3] = g0.w;
        u[z][4] = g1.x; u[z][5] = g1.y; u[z][6] = g1.z; u[z][7] = g1.w;
        if (gm(t.mom)) {
          const float4* q = (const float4*)(gm(t.mom) + i * t.cols + j);
          const float4 m0 = q[0], m1 = q[1];
          float* to = m[z - z0];
          to[0] = m0.x; to[1] = m0.y; to[2] = m0.z; to[3] = m0.w;
          to[4] = m1.x; to[5] = m1.y; to[6] = m1.z; to[7] = m1.w;
        }
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if (j + v < t.n) {
            const int e = flip ? (j + v) * t.cols + i : i * t.cols + j + v;
            u[z][v] = gm(t.grad)[e];
            if (gm(t.mom)) m[z - z0][v] = gm(t.mom)[e];
          }
      }
    }
#pragma unroll
    for (int z = z0; z < min(z0 + kFlight, kSmallChunks); ++z) {
      int i, j;
      if (!place(z, i, j) || i >= t.m) continue;
      if (gm(t.mom)) {
        float* q = m[z - z0];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          q[v] = mu * q[v] + u[z][v];
          u[z][v] = nesterov ? u[z][v] + mu * q[v] : q[v];
        }
        if (vec && j + 8 <= t.n) {
          float4* to = (float4*)(gm(t.mom) + i * t.cols + j);
          to[0] = make_float4(q[0], q[1], q[2], q[3]);
          to[1] = make_float4(q[4], q[5], q[6], q[7]);
        } else {
#pragma unroll
          for (int v = 0; v < 8; ++v)
            if (j + v < t.n) gm(t.mom)[flip ? (j + v) * t.cols + i : i * t.cols + j + v] = q[v];
        }
      }
#pragma unroll
      for (int v = 0; v < 8; ++v) sum += (double)u[z][v] * u[z][v];
    }
  }
  const Scale scale(sqrt(first_sum(sum, lds.sh)) + eps);
  auto put_x = [&](auto part) {
#pragma unroll
    for (int z = 0; z < kSmallChunks; ++z) {
      int i, j;
      if (z * kFirstT >= chunks) break;
      if (!place(z, i, j)) continue;
      f16x8 h;
#pragma unroll
      for (int v = 0; v < 8; ++v) h[v] = (f16)part(scale(u[z][v]));
      *(f16x8*)(xs + ((j >> 5) * MS + i) * kRow + (j & 31) * 2) = h;
    }
    __syncthreads();
  };
  const int fr = lane & 31, hi = lane >> 5;
  // xl of this wave's panels (wave, wave + 12, ..), as the products' accumulators
  // lie: by way of X's place in LDS
  constexpr int kPanels = (kSmallX / MS / 32 + kFirstT / 64 - 1) / (kFirstT / 64);
  // (there as float16)
  constexpr float kSL = 2048.f;
  auto low = [](float v) { return (v - (float)(f16)v) * kSL; };
  unsigned xl[kPanels][Q][8];
  if (keeps_low(steps)) {
    put_x(low);
#pragma unroll
    for (int k = 0; k < kPanels; ++k)
#pragma unroll
      for (int i = 0; i < Q; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int pj = min(wave + k * (kFirstT / 64), ns / 32 - 1);
          const uint2 v = *(const uint2*)(xs + (pj * MS + 32 * i + fr) * kRow + 16 * g + 8 * hi);
          xl[k][i][2 * g] = v.x;
          xl[k][i][2 * g + 1] = v.y;
        }
    __syncthreads();
  }
  put_x([](float v) { return v; });

  const int kb = 8 * hi + ((lane & 15) >> 2), cb = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  // fragment of 32 rows from r0 on, sum values 16 kk .. of panel p
  auto rows_of = [&](const unsigned char* b, int p, int r0, int kk) {
    return *(const u32x4*)(b + (p * MS + r0 + fr) * kRow + (2 * kk + hi) * 16);
  };
  // place of four values of row r from column c on
  auto four = [&](unsigned char* b, int r, int c) { return b + ((c >> 5) * MS + r) * kRow + (c & 31) * 2; };
  // stores a fragment of a symmetric matrix (rows i0, columns j0) and its diagonal's errors
  auto store = [&](unsigned char* b, float* d, int i0, int j0, const f32x4_t (&f)[4]) {
    unsigned pk[8];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      pk[2 * g] = pack_f16(f[g][0] * kSM, f[g][1] * kSM);
      pk[2 * g + 1] = pack_f16(f[g][2] * kSM, f[g][3] * kSM);
    }
    if (i0 == j0 && diagonal_here()) d[j0 + fr] = lost(diagonal(f));
    put8(pk, [&](int h, u32x4 c) { *(u32x4*)four(b, j0 + fr, i0 + 16 * h + 8 * hi) = c; });
  };
  const int i0 = wave % F / Q * 32, j0 = wave % Q * 32;   // this wave's fragment of A and P
  for (int s = 0; s < steps; ++s) {
    // A = X X^T, the even and the odd panels' sums apart
    f32x4_t f[4];
    if (wave < F) {
      f32x16 acc = {}, odd = {};
      for (int p = 0; p < ns / 32; p += 2) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          acc = mfma(rows_of(xs, p, i0, kk), rows_of(xs, p, j0, kk), acc);
          if (p + 1 < ns / 32) odd = mfma(rows_of(xs, p + 1, i0, kk), rows_of(xs, p + 1, j0, kk), odd);
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) f[g] = (part_of(acc, g) + part_of(odd, g)) * (1.f / (kSX * kSX));
      store(as, da, i0, j0, f);
    }
    // one wave reads what its other lanes wrote: LDS keeps a wave's order, and
    // the compiler has to
    if constexpr (F > 1) __syncthreads();
    else asm volatile("" ::: "memory");
    // P = a I + b A + c A A
    if (wave < F) {
      const int c = j0 + fr;
      f32x16 acc = {};
#pragma unroll
      for (int p = 0; p < Q; ++p)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) acc = mfma(rows_of(as, p, i0, kk), rows_of(as, p, j0, kk), acc);
      const float dc = da[c], diag = i0 == j0 ? kA + (kB + kC * dc) * dc : 0.f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int r = i0 + 8 * g + 4 * hi;
        const f32x4_t a = from_f16((const f16*)four(as, c, r)) * (1.f / kSM);
        f[g] = kC * (part_of(acc, g) * (1.f / (kSM * kSM)) + a * (*(const f32x4_t*)(da + r) + dc)) + kB * a;
#pragma unroll
        for (int z = 0; z < 4; ++z) f[g][z] += r + z == c ? diag : 0.f;
      }
      store(pms, dp, i0, j0, f);
    }
    __syncthreads();
    // X = P X, a panel a wave and turn, in place
    const float factor = low_factor(steps - s, 1);
#pragma unroll
    for (int k = 0; k < kPanels; ++k) {
      const int pj = wave + k * (kFirstT / 64);
      if (pj >= ns / 32) break;
      f32x16 acc[Q] = {};
#pragma unroll
      for (int p = 0; p < Q; ++p)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const u32x4 b = frag_tr(xs + (pj * MS + 32 * p + 16 * kk + kb) * kRow + cb * 16 + 8 * (lane & 1), kRow);
#pragma unroll
          for (int i = 0; i < Q; ++i) acc[i] = mfma(b, rows_of(pms, p, 32 * i, kk), acc[i]);
        }
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const int r = 32 * i + fr;
        const float d = dp[r] * (1.f / kSX);
        float y[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4_t xv = from_f16((const f16*)four(xs, r, 32 * pj + 8 * g + 4 * hi));
#pragma unroll
          for (int z = 0; z < 4; ++z) y[4 * g + z] = acc[i][4 * g + z] * (1.f / (kSM * kSX)) + d * xv[z];
        }
        if (factor != 0) {
          const float p = factor == P_DIAGONAL ? (float)*(const f16*)four(pms, r, r) * (1.f / kSM) + dp[r] : factor;
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            const f16x2 v = __builtin_bit_cast(f16x2, xl[k][i][g]);
            y[2 * g] += p * (1.f / (kSX * kSL)) * (float)v[0];
            y[2 * g + 1] += p * (1.f / (kSX * kSL)) * (float)v[1];
            xl[k][i][g] = pack_f16(low(y[2 * g] * kSX), low(y[2 * g + 1] * kSX));
          }
        }
        if (s + 1 < steps) {
          unsigned pk[8];
#pragma unroll
          for (int g = 0; g < 8; ++g) pk[g] = pack_f16(y[2 * g] * kSX, y[2 * g + 1] * kSX);
          put8(pk, [&](int h, u32x4 c) { *(u32x4*)four(xs, r, 32 * pj + 16 * h + 8 * hi) = c; });
        } else {
          store_update(t, r, 32 * pj, y);
        }
      }
    }
    __syncthreads();
  }
}

// The first launch of a list with such matrices: a block each, while the other
// blocks take the others' momentum.
__global__ __launch_bounds__(kFirstT) void muon_whole(Mats l, Mats* table, int wholes, float mu, int nesterov, int steps,
                                                      float eps) {
  __shared__ __attribute__((aligned(16))) SmallLds lds;
  const int blk = blockIdx.x;
  if (blk >= wholes) {
    if (blk == wholes) leave_table(l, table);
    momentum(l, blk - wholes, mu, nesterov, lds.sh);
    return;
  }
  const Mat& t = l.t[l.count - wholes + blk];   // the last of the list
  if (t.m > 32) small_update<64>(lds, t, mu, nesterov, steps, eps);
  else small_update<32>(lds, t, mu, nesterov, steps, eps);
}

size_t al256(size_t x) { return (x + 255) & ~size_t(255); }
constexpr int kPad = 128;
constexpr int kBlocks = 512;   // two a CU
constexpr int kRange = 64;     // panels
int up(int x) { return (x + kPad - 1) / kPad * kPad; }
int uppers(int nt) { return nt * (nt + 1) / 2; }

// Whether two steps are taken at once.  The products with X that this saves
// run at about twice the rate of the m x m ones that replace them, on fewer
// tiles: from n = 4 m on (a 3 x 3 layer has 9 m and more).  1024 x 4096 224 us,
// 244 one step at a time; 2048 x 8192 740, 876.  At n = 2 m it depends on m: 1024 x
// 2048 174 and 165, 2048 x 4096 552 and 588.
bool pairs(const tgp_muon_tensor& d) {
  return std::max(d.rows, d.cols) >= 4 * (long)std::min(d.rows, d.cols);
}

// Whether one block does the whole update.
bool small(const tgp_muon_tensor& d) {
  const long m = std::min(d.rows, d.cols), n = std::max(d.rows, d.cols);
  return m <= 64 && (m <= 32 ? 32 : 64) * ((n + 31) / 32 * 32) <= kSmallX;
}
void describe(const tgp_muon_tensor& d, Mat& t) {
  t = Mat{};
  t.grad = d.grad;
  t.mom = d.momentum;
  t.out = (bf16_t*)d.update;
  t.rows = d.rows;
  t.cols = d.cols;
  t.m = std::min(t.rows, t.cols);
  t.n = std::max(t.rows, t.cols);
}

// Describes n (at most kMaxMats) matrices laid out in the workspace ws (NULL:
// only the size is asked for); returns its bytes.  The sum of A = X X^T is split
// where a matrix has too few tiles to fill the chip: into as many ranges as make
// at most kBlocks blocks (one more than run at once waits for all of them: 2048 x
// 18432 in 3 ranges 89 us and 8.6 to add them up, in 4 101 and 9.7, in 7 86 and
// 13.4), of kRange panels at least (writing and reading back a partial tile
// takes the time of 20; with 32 at least, before X had its xl, 2048 x 2048 took 398
// us and not 377, a U-Net's 19 matrices 635 and not 610, 1024 x 9216 318 and not
// 324).  The ranges depend on the matrix alone, so that its update does not
// depend on the others of the call.
size_t lay_out(int n, const tgp_muon_tensor* const* d, char* ws, Mats& l) {
  size_t pos = 0;
  auto take = [&](size_t bytes) {
    char* p = ws ? ws + pos : nullptr;
    pos += al256(bytes);
    return p;
  };
  l.count = n;
  take(sizeof(Mats));   // the launches' table, first
  for (int k = 0; k < n; ++k) {
    Mat& t = l.t[k];
    describe(*d[k], t);
    if (small(*d[k])) continue;
    t.two = pairs(*d[k]);
    t.mp = up(t.m);
    t.np = up(t.n);
    const long size = (long)t.rows * t.cols;
    t.norm_blocks = (int)std::min<long>(kNormBlocks, cdiv(size, 8 * kFirstT));
    t.norm_per = size >= 1 << 22 ? 4 : 1;   // where it is large, |U| is summed up by fewer blocks
    t.norm = (double*)take(kNormBlocks * sizeof(double));
    for (int z = 0; z < 2; ++z) t.x[z] = (f16*)take((size_t)t.mp * t.np * 2);
    take((size_t)t.mp * t.np);   // xl, after x[1] (whose size is a multiple of 256)
    for (int z = 0; z < 3; ++z) {
      t.s[z] = (f16*)take((size_t)t.mp * t.mp * 2);
      t.d[z] = (float*)take((size_t)t.mp * 4);
    }
    t.split = std::max(1, std::min(kBlocks / uppers(t.mp / 128), t.np / 32 / kRange));
    t.part = nullptr;
    if (t.split > 1) t.part = (float*)take((size_t)t.split * uppers(t.mp / 128) * 128 * 128 * sizeof(float));
  }
  return pos;
}

// Deals the matrices into lists of at most kMaxMats: the tiled ones, those of
// the longest sums first (stable), so that the short ones fill up a launch's
// end, and after them those that one block does whole.  Calls go(list of
// pointers, count).
template <typename F>
void each_list(int n, const tgp_muon_tensor* t, F go) {
  const tgp_muon_tensor* list[kMaxMats];
  int count = 0;
  auto flush = [&]() {
    std::stable_sort(list, list + count, [](const tgp_muon_tensor* a, const tgp_muon_tensor* b) {
      return small(*a) != small(*b) ? small(*b) : std::min(a->rows, a->cols) > std::min(b->rows, b->cols);
    });
    if (count) go(list, count);
    count = 0;
  };
  for (int kind = 0; kind < 2; ++kind)
    for (int k = 0; k < n; ++k) {
      if (small(t[k]) != (kind == 1)) continue;
      list[count++] = t + k;
      if (count == kMaxMats) flush();
    }
  flush();
}

// Fills blk0 of a launch with blocks(t) of each matrix; returns the grid.
template <typename F>
unsigned deal(Mats& l, int launch, F blocks) {
  int pos = 0;
  for (int k = 0; k < l.count; ++k) {
    l.blk0[launch][k] = pos;
    pos += blocks(l.t[k]);
  }
  l.blk0[launch][l.count] = pos;
  return (unsigned)pos;
}

hipError_t update_list(Mats& l, Mats* table, float mu, bool nesterov, int steps, float eps, hipStream_t st) {
  double n = 0, gram = 0, cube = 0, cells = 0;   // of the tiled matrices
  double wn = 0, wflops = 0;                     // of the others
  long t192 = 0, t128 = 0, g128 = 0;   // tiles of P X, of X X^T
  int wholes = 0;
  for (int k = 0; k < l.count; ++k) {
    const Mat& t = l.t[k];
    const double m = t.m, mn = m * t.n;
    if (t.whole()) {
      ++wholes;
      wn += mn;
      wflops += steps * (3 * m * mn + m * m * m);
      continue;
    }
    n += mn;
    gram += m * mn;
    cube += m * m * m;
    cells += m * m;
    t192 += (long)(t.mp / 128) * cdiv(t.np, 192);
    t128 += (long)(t.mp / 128) * (t.np / 128);
    g128 += (long)uppers(t.mp / 128) * t.split;
  }
  // Columns of a tile of P X and X X^T.  P X on tiles of 128 x 192 takes a
  // sixth less from the caches and LDS than on 128 x 128 (without xl 2048 x 18432:
  // 147 us, 160; 1024 x 9216, one and a half blocks a CU: 27.9, 29.5); it is taken
  // where its tiles make one block a CU.  (Where n is no multiple of 192 it
  // multiplies zeros, which this does not weigh: 20 of 512 x 640 285 us, and 267
  // in tiles of 128; 6 of 1024 x 1024 391 and 366.)  Where 128 x 128 leaves CUs
  // without one, 64 x 64.  The sums' order is the same in all of them.
  const int ba = t192 >= 256 ? 192 : t128 >= 256 ? 128 : 64, bg = g128 >= 256 ? 128 : 64;
  auto grams = [&](const Mat& t) { return uppers(t.mp / bg) * t.split; };
  auto sums = [&](const Mat& t) { return t.split > 1 ? uppers(t.mp / bg) * (bg / 64) * (bg / 64) : 0; };
  auto applies = [&](const Mat& t) { return (t.mp / std::min(ba, 128)) * cdiv(t.np, ba); };
  auto syms = [](const Mat& t) { return uppers(t.mp / 64); };
  unsigned grid[LAUNCHES];
  auto tiled = [&](int launch, auto blocks) {
    grid[launch] = deal(l, launch, [&](const Mat& t) { return t.whole() ? 0 : blocks(t); });
  };
  tiled(L_MOMENTUM, [](const Mat& t) { return t.norm_blocks; });
  tiled(L_NORMALIZE, [](const Mat& t) { return t.mp * (t.np / 128) / 32 / t.norm_per; });
  tiled(L_GRAM, grams);
  tiled(L_SUM, sums);
  tiled(L_SYM, syms);
  tiled(L_APPLY, applies);
  tiled(L_GRAM1, [&](const Mat& t) { return t.two ? 0 : grams(t); });
  tiled(L_SUM1, [&](const Mat& t) { return t.two ? 0 : sums(t); });
  tiled(L_APPLY1, [&](const Mat& t) { return t.two ? 0 : applies(t); });
  tiled(L_SYM2, [&](const Mat& t) { return t.two ? syms(t) : 0; });
  // The products of m x m matrices with up to two blocks a CU wait for their
  // stages: two panels each.  With more blocks one panel, whose ring takes half
  // the LDS, leaves room for more of them (2048 x 18432 without xl: 1122 us, 1160
  // with two).
  auto few = [&](int launch) { return grid[launch] <= kBlocks; };
  const Mats* tb = table;
  if (wholes) {
    ProfScope ps("muon_whole", wflops + 4 * n, 14 * wn + 12 * n, st);
    TGP_LAUNCH(ps, muon_whole, dim3(wholes + grid[L_MOMENTUM]), dim3(kFirstT), 0, st, l, table, wholes, mu,
               (int)nesterov, steps, eps);
    if (!grid[L_MOMENTUM]) return launch_status();
  } else {
    ProfScope ps("muon_momentum", 4 * n, 12 * n, st);
    TGP_LAUNCH(ps, muon_momentum, dim3(grid[L_MOMENTUM]), dim3(kFirstT), 0, st, l, table, mu, (int)nesterov);
  }
  {
    ProfScope ps("muon_normalize", 2 * n, 10 * n, st);
    TGP_LAUNCH(ps, muon_normalize, dim3(grid[L_NORMALIZE]), dim3(256), 0, st, tb, mu, (int)nesterov, eps,
               (int)keeps_low(steps));
  }
  // the launches, each over the matrices of its table that have blocks in it
  Each from{{0, 0}};   // which of its two buffers X is in
  auto gram_of = [&](int lg, int ls) {
    if (grid[lg]) {
      ProfScope ps("muon_gram", gram, 2 * n + 2 * cells, st);
      if (bg == 128)
        TGP_LAUNCH(ps, (muon_sym<GRAM, 2, 2, 2, 2, 4, 1>), dim3(grid[lg]), dim3(256), 0, st, tb, lg, from, 0, (Each{{0, 0}}));
      else
        TGP_LAUNCH(ps, (muon_sym<GRAM, 1, 1, 2, 2, 4, 2>), dim3(grid[lg]), dim3(256), 0, st, tb, lg, from, 0, (Each{{0, 0}}));
    }
    if (grid[ls]) {
      ProfScope ps("muon_gram_sum", 0, 0, st);
      if (bg == 128) TGP_LAUNCH(ps, (muon_gram_sum<2, 2, 2, 2>), dim3(grid[ls]), dim3(256), 0, st, tb, ls);
      else TGP_LAUNCH(ps, (muon_gram_sum<1, 1, 2, 2>), dim3(grid[ls]), dim3(256), 0, st, tb, ls);
    }
  };
  auto poly = [&](Each c) {
    ProfScope ps("muon_poly", cube, 4 * cells, st);
    if (few(L_SYM))
      TGP_LAUNCH(ps, (muon_sym<POLY, 1, 1, 2, 2, 4, 2>), dim3(grid[L_SYM]), dim3(256), 0, st, tb, (int)L_SYM,
                 (Each{{0, 0}}), 0, c);
    else
      TGP_LAUNCH(ps, (muon_sym<POLY, 1, 1, 2, 2, 4, 1>), dim3(grid[L_SYM]), dim3(256), 0, st, tb, (int)L_SYM,
                 (Each{{0, 0}}), 0, c);
  };
  auto mul = [&](int a, int b, int c) {
    if (!grid[L_SYM2]) return;
    ProfScope ps("muon_mul", cube, 6 * cells, st);
    if (few(L_SYM2))
      TGP_LAUNCH(ps, (muon_sym<MUL, 1, 1, 2, 2, 4, 2>), dim3(grid[L_SYM2]), dim3(256), 0, st, tb, (int)L_SYM2,
                 (Each{{a, a}}), b, (Each{{c, c}}));
    else
      TGP_LAUNCH(ps, (muon_sym<MUL, 1, 1, 2, 2, 4, 1>), dim3(grid[L_SYM2]), dim3(256), 0, st, tb, (int)L_SYM2,
                 (Each{{a, a}}), b, (Each{{c, c}}));
  };
  auto apply = [&](int la, Each p, int last, EachLow low) {
    if (!grid[la]) return;
    ProfScope ps("muon_apply", 2 * gram, 4 * n + 2 * cells, st);
    if (ba == 192)
      TGP_LAUNCH(ps, (muon_apply<2, 3, 2, 2, 4, 1>), dim3(grid[la]), dim3(256), 0, st, tb, la, p, from, last, low);
    else if (ba == 128)
      TGP_LAUNCH(ps, (muon_apply<2, 2, 2, 2, 4, 1>), dim3(grid[la]), dim3(256), 0, st, tb, la, p, from, last, low);
    else
      TGP_LAUNCH(ps, (muon_apply<1, 1, 2, 2, 4, 2>), dim3(grid[la]), dim3(256), 0, st, tb, la, p, from, last, low);
  };
  // Two steps a turn: what both kinds of matrices need is one launch for both,
  // and a list of one kind has no launches of the other.
  for (int s = 0; s < steps; s += 2) {
    const bool turn = s + 2 <= steps;
    gram_of(L_GRAM, L_SUM);
    poly(Each{{1, 1}});
    if (turn) {
      mul(1, 0, 2);                          // P A
      apply(L_APPLY1, Each{{1, 1}}, 0, EachLow{{low_factor(steps - s, 1), 0.f}, {keeps_low(steps - s - 1), 0}});
      if (grid[L_APPLY1]) from.v[0] ^= 1;
      mul(2, 1, 0);                          // A' = P A P
      gram_of(L_GRAM1, L_SUM1);
      poly(Each{{1, 2}});                    // P'
      mul(2, 1, 0);                          // P' P
    }
    const int end = std::min(s + 2, steps), keep = keeps_low(steps - end);
    apply(L_APPLY, Each{{1, turn ? 0 : 1}}, end == steps,
          EachLow{{low_factor(steps - end + 1, 1), low_factor(steps - s, end - s)}, {keep, keep}});
    from.v[0] ^= 1;
    from.v[1] ^= 1;
  }
  return launch_status();
}

}  // namespace

// The lists of one call run one after the other on its stream, and share the
// workspace.
size_t muon_bytes(int n, const tgp_muon_tensor* t) {
  size_t most = 0;
  Mats l;
  each_list(n, t, [&](const tgp_muon_tensor* const* d, int count) {
    most = std::max(most, lay_out(count, d, nullptr, l));
  });
  return most;
}

hipError_t muon_update(int n, const tgp_muon_tensor* t, float mu, bool nesterov, int steps,
                       float eps, void* ws, hipStream_t st) {
  hipError_t e = hipSuccess;
  each_list(n, t, [&](const tgp_muon_tensor* const* d, int count) {
    if (e != hipSuccess) return;
    Mats l;
    lay_out(count, d, (char*)ws, l);
    e = update_list(l, (Mats*)ws, mu, nesterov, steps, eps, st);
  });
  return e;
}

}  // namespace tgpk
