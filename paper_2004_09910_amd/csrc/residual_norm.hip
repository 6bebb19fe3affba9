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
#include <initializer_list>
#include <type_traits>

#include "common.h"
#include "prof.h"
#include "row_plan.h"
#include "row_regs.h"
#include "train_ops.h"

namespace tgpk {
namespace {

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

// Which pixels a block takes.  Ranges: `ranges` blocks for each of the groups of
// pixels that share a gate (one group of all pixels where none do), `per` pixels
// each.  Whole: whole groups by a wave (a block, where a row is a block's), side
// by side in parts of `part` lanes' rows (a power of two) where they are small.
struct BwdArgs {
  const void *dz, *dout, *out, *f, *gate;
  void *dr, *df, *dgate;
  long lddz, lddout, ldout, ldf, ldgate, lddr, lddf, lddgate, rows, group, per;
  Vectors w;
  const float4* stats;
  float* part;   // [block][4][C]: dz ohat, dz, S1, S2 (ranges of a shared gate: U1, U2)
  int C, G, ranges, slots;
  int shared;    // a gate for several pixels
};

// A row a block at a time, G of it in LDS; a column's sums belong to one thread of the
// block and lie in part, of whole groups with U1 and U2 of the present one behind them
// (six a block).  (32768 x 4104 bfloat16, a gate for 8192 pixels: 2.7 ms, by a block a
// gate 341.)
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kT) void res_bwd_any(BwdArgs a, int post) {
  extern __shared__ float row[];
  __shared__ float s4[4];
  const T *dz = (const T*)a.dz, *dout = (const T*)a.dout, *out = (const T*)a.out, *f = (const T*)a.f;
  const int C = a.C;
  const Vectors& w = a.w;
  float* mine = a.part + (long)blockIdx.x * (WHOLE ? 6 : 4) * C;
  float *P0 = mine, *P1 = P0 + C, *S1 = P1 + C, *S2 = S1 + C, *U1 = S2 + C, *U2 = U1 + C;
  for (int c = threadIdx.x; c < C; c += kT) P0[c] = P1[c] = S1[c] = S2[c] = 0.f;
  const float inv_c = 1.f / C;
  // pixel p with its gate at q; A1 and A2 take G fhat and G (times the gate, where it is the pixel's own)
  auto take = [&](long p, const T* q, float* A1, float* A2) {
    const float4 st = a.stats[p];
    float ms = 0.f, mp = 0.f;
    if (dz) {
      for (int c = threadIdx.x; c < C; c += kT) {
        const float d = Elt<T>::ld(dz + p * a.lddz + c), e = d * at_or(w.pre_gain, c, 1.f);
        const float o = (Elt<T>::ld(out + p * a.ldout + c) - st.z) * st.w;
        ms += e;
        mp += e * o;
        P0[c] += d * o;
        P1[c] += d;
      }
      ms = block_sum(ms, s4) * inv_c;
      mp = block_sum(mp, s4) * inv_c;
    }
    float ns = 0.f, np = 0.f;
    for (int c = threadIdx.x; c < C; c += kT) {
      float G = dout ? Elt<T>::ld(dout + p * a.lddout + c) : 0.f;
      if (dz) {
        const float e = Elt<T>::ld(dz + p * a.lddz + c) * at_or(w.pre_gain, c, 1.f);
        const float o = (Elt<T>::ld(out + p * a.ldout + c) - st.z) * st.w;
        G += st.w * (e - ms - o * mp);
      }
      row[c] = G;
      if (!post) continue;
      const float fh = (Elt<T>::ld(f + p * a.ldf + c) - st.x) * st.y;
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
      float fh = Elt<T>::ld(f + p * a.ldf + c), v = G * sc * g, n = fh;
      if (post) {
        const float pg = at_or(w.post_gain, c, 1.f);
        fh = (fh - st.x) * st.y;
        n = pg * fh + at_or(w.post_bias, c, 0.f);
        v = st.y * (v * pg - ns - fh * np);
      }
      const float h = a.shared ? G : g * G;
      A1[c] += h * fh;
      A2[c] += h;
      if (a.dgate && !a.shared) Elt<T>::st((T*)a.dgate + p * a.lddgate + c, sc * G * n);
      Elt<T>::st((T*)a.dr + p * a.lddr + c, G);
      Elt<T>::st((T*)a.df + p * a.lddf + c, v);
    }
  };
  if constexpr (!WHOLE) {
    const long g = blockIdx.x / (unsigned)a.ranges;
    const long lo = g * a.group + (blockIdx.x - g * a.ranges) * a.per, hi = min(lo + a.per, (g + 1) * a.group);
    for (long p = lo; p < hi; ++p) take(p, a.gate ? (const T*)a.gate + (a.shared ? g : p) * a.ldgate : nullptr, S1, S2);
  } else {
    for (long u = blockIdx.x; u * a.group < a.rows; u += gridDim.x) {
      const T* q = (const T*)a.gate + u * a.ldgate;
      for (int c = threadIdx.x; c < C; c += kT) U1[c] = U2[c] = 0.f;
      for (long p = u * a.group; p < (u + 1) * a.group; ++p) take(p, q, U1, U2);
      for (int c = threadIdx.x; c < C; c += kT) {
        const float g = Elt<T>::ld(q + c);
        S1[c] += g * U1[c];
        S2[c] += g * U2[c];
        if (a.dgate) {
          const float n = post ? at_or(w.post_gain, c, 1.f) * U1[c] + at_or(w.post_bias, c, 0.f) * U2[c] : U1[c];
          Elt<T>::st((T*)a.dgate + u * a.lddgate + c, at_or(w.scale, c, 1.f) * n);
        }
      }
    }
  }
}

// ------------------------------------------------- rows held in registers

// Row sums divided by C, of the values that the lane has.
template <typename SH, bool BLK, int NV, int V>
__device__ __forceinline__ float mean_of(const SH& sh, const float (&f)[NV][V], int C, float* s4) {
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) s += sh.has(k) ? f[k][v] : 0.f;
  return row_sum<BLK>(s, sh.G, s4) / C;
}

// f less its mean, and the row's mean and rstd: the differences' own mean is taken
// off them and added to the mean, as the layer norm does.
template <typename SH, bool BLK, int NV, int V>
__device__ __forceinline__ float2 centre(const SH& sh, float (&f)[NV][V], int C, float eps, float* s4) {
  float mean = mean_of<SH, BLK, NV, V>(sh, f, C, s4);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) f[k][v] -= mean;
  const float e = mean_of<SH, BLK, NV, V>(sh, f, C, s4);
  float q = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      f[k][v] -= e;
      if (sh.has(k)) q += f[k][v] * f[k][v];
    }
  return make_float2(mean + e, 1.f / sqrtf(row_sum<BLK>(q, sh.G, s4) / C + eps));
}

// One tensor's rows for a lane: those of a turn start at an address that is the same
// for the wave, from which the lane's row is `off` bytes away.  (64-bit addresses a
// lane and tensor cost registers, and the waves that hide memory's latency.)
template <typename T>
struct Lanes {
  char* p;
  long ld;        // bytes
  unsigned off;
  __device__ __forceinline__ Lanes(const void* t, long l, int row) : p((char*)t), ld(l * (long)sizeof(T)) {
    off = (unsigned)(row * ld);
  }
  __device__ __forceinline__ char* at(long row) const { return p + row * ld; }   // of the wave
};

// A lane's part of a row as it is in memory.  All loads of a row go out before the
// first value is looked at.
template <typename VT, int NV>
struct Raw {
  typename VT::raw r[NV];
  __device__ __forceinline__ void none() {
#pragma unroll
    for (int k = 0; k < NV; ++k) r[k] = typename VT::raw{};
  }
  __device__ __forceinline__ void load(const char* p, unsigned off, int k) { r[k] = *(const typename VT::mem*)(p + off); }
  template <int V>
  __device__ __forceinline__ void to(float (&f)[NV][V]) const {
#pragma unroll
    for (int k = 0; k < NV; ++k) VT::un(r[k], f[k]);
  }
};
// ov: byte offsets of the lane's vectors in a row.
template <typename VT, typename SH, typename T, int NV, int V>
__device__ __forceinline__ void store_row(const SH& sh, char* p, unsigned off, const unsigned (&ov)[NV],
                                          const float (&f)[NV][V]) {
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (sh.has(k)) {
      char* q = p + (off + ov[k]);
      if constexpr (sizeof(T) == 2 && V == 8)
        *(uint4*)q = make_uint4(pack_bf16(f[k][0], f[k][1]), pack_bf16(f[k][2], f[k][3]),
                                pack_bf16(f[k][4], f[k][5]), pack_bf16(f[k][6], f[k][7]));
      else if constexpr (sizeof(T) == 2 && V == 4)
        *(uint2*)q = make_uint2(pack_bf16(f[k][0], f[k][1]), pack_bf16(f[k][2], f[k][3]));
      else if constexpr (sizeof(T) == 2 && V == 2)
        *(uint32_t*)q = pack_bf16(f[k][0], f[k][1]);
      else
        *(typename VT::mem*)q = (typename VT::mem)VT::pk(f[k]);
    }
}

struct FwdArgs {
  const void *r, *f, *gate;
  void *out, *z;
  long ldr, ldf, ldgate, ldout, ldz, rows;
  unsigned group;
  Vectors w;
  float eps;
  float4* stats;
  int C, G;
};

// A row's values stay in registers from their loads to both results: G lanes of a wave a
// row, or a block.  Memory bounds it where there are many rows (147456 x 64 bfloat16 with
// z 17.7 us, 4.3 TB/s), the launch where there are few (144 x 1024 4.5 us).
template <typename T, int VB, int NV, bool BLK, bool POST>
__global__ __launch_bounds__(kT) void res_fwd(FwdArgs a) {
  typedef Vec<T, VB> VT;
  typedef Share<T, VB, NV, BLK> SH;
  constexpr int V = SH::V;
  __shared__ float s4[4];
  const SH sh(a.C, a.G, gridDim.x);
  // scale (post_gain fhat + post_bias) as one gain and one bias
  float pg[NV][V], pb[NV][V], ng[NV][V], nb[NV][V];
  sh.channels(a.w.scale, 1.f, pg);
  if constexpr (POST) {
    float t[NV][V];
    sh.channels(a.w.post_bias, 0.f, pb);
    sh.channels(a.w.post_gain, 1.f, t);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        pb[k][v] *= pg[k][v];
        pg[k][v] *= t[k][v];
      }
  }
  sh.channels(a.w.pre_gain, 1.f, ng);
  sh.channels(a.w.pre_bias, 0.f, nb);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rpw = BLK ? 1 : 64 / sh.G, rl = BLK ? 0 : (threadIdx.x & 63) / sh.G;   // rows of a wave, this lane's
  const Lanes<T> f(a.f, a.ldf, rl), rs(a.r, a.ldr, rl), out(a.out, a.ldout, rl), z(a.z, a.ldz, rl);
  unsigned ov[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) ov[k] = sh.vec(k) * VB;
  // the trip count is the same for every lane of the block (block_sum meets a barrier)
  for (long base = BLK ? blockIdx.x : (long)blockIdx.x * 4 * rpw; base < a.rows; base += sh.step) {
    const long p0 = base + (BLK ? 0 : wave * rpw), p = p0 + rl;   // the wave's first row, the lane's
    const bool in = p < a.rows;
    float x[NV][V], r[NV][V], q[NV][V];
    Raw<VT, NV> rx, rr, rq;
    rx.none();
    rr.none();
    rq.none();
    if (in) {
      const char *fp = f.at(p0), *rp = rs.at(p0);
      long g = p;
      if (a.group > 1) g = a.rows <= 0xffffffffl ? (long)((unsigned)p / a.group) : p / a.group;
      const char* gp = (const char*)a.gate + g * a.ldgate * (long)sizeof(T);
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (sh.has(k)) {
          rx.load(fp, f.off + ov[k], k);
          rr.load(rp, rs.off + ov[k], k);
          if (a.gate) rq.load(gp, ov[k], k);
        }
    }
    rx.to(x);
    rr.to(r);
    rq.to(q);
    float2 st = make_float2(0.f, 0.f), so = st;
    if constexpr (POST) st = centre<SH, BLK>(sh, x, a.C, a.eps, s4);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float n = POST ? x[k][v] * st.y * pg[k][v] + pb[k][v] : x[k][v] * pg[k][v];
        if (a.gate) n *= q[k][v];
        x[k][v] = r[k][v] + n;
      }
    if (in) store_row<VT, SH, T>(sh, out.at(p0), out.off, ov, x);
    if (a.z) {
      so = centre<SH, BLK>(sh, x, a.C, a.eps, s4);
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) x[k][v] = x[k][v] * so.y * ng[k][v] + nb[k][v];
      if (in) store_row<VT, SH, T>(sh, z.at(p0), z.off, ov, x);
    }
    if (in && a.stats && sh.l == 0) a.stats[p] = make_float4(st.x, st.y, so.x, so.y);
  }
}

// The four sums over rows stay in registers to a block's end, and the next row's loads
// are on their way while one is worked on (131072 x 128 bfloat16, rows 384 apart, with
// the sums' launches: 82.6 us with a row's loads one after the other and none ahead, 54
// so).  Memory bounds it (46 us on tensors that are new to the caches, 4.4 TB/s, 36.5 on
// ones that are not), and the sums' launches, 4 to 5 us each.
template <typename T, int VB, int NV, bool BLK, bool POST, bool WHOLE>
__global__ __launch_bounds__(kT) void res_bwd(BwdArgs a) {
  typedef Vec<T, VB> VT;
  typedef Share<T, VB, NV, BLK> SH;
  constexpr int V = SH::V;
  __shared__ float s8[2][4];
  const SH sh(a.C, a.G, gridDim.x);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rpw = BLK ? 1 : 64 / sh.G, rl = BLK ? 0 : lane / sh.G;   // rows of a wave, this lane's
  // (whole groups) rows of a part of the lanes, the lane's part and row in it
  const int side = WHOLE ? rpw / a.slots : rpw, slot = rl / side, first = rl - slot * side;
  const int lr = WHOLE ? (int)(slot * a.group) + first : rl;   // the lane's row from the wave's first
  const Lanes<T> tz(a.dz, a.lddz, lr), to_(a.out, a.ldout, lr), td(a.dout, a.lddout, lr), tf(a.f, a.ldf, lr),
      tg(a.gate, a.ldgate, lr), tr(a.dr, a.lddr, lr), tdf(a.df, a.lddf, lr), tdg(a.dgate, a.lddgate, lr);
  unsigned ov[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) ov[k] = sh.vec(k) * VB;
  // scale post_gain, scale post_bias, pre_gain; the first zero where the lane has no
  // channel, so that nothing of such a lane gets into a row's sums
  float pg[NV][V], pb[NV][V], ng[NV][V];
  sh.channels(a.w.scale, 1.f, pg);
  if constexpr (POST) {
    float t[NV][V];
    sh.channels(a.w.post_bias, 0.f, pb);
    sh.channels(a.w.post_gain, 1.f, t);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        pb[k][v] *= pg[k][v];
        pg[k][v] = sh.has(k) ? pg[k][v] * t[k][v] : 0.f;
      }
  }
  sh.channels(a.w.pre_gain, 1.f, ng);
  float sum[4][NV][V];
#pragma unroll
  for (int z = 0; z < 4; ++z)
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) sum[z][k][v] = 0.f;
  const float inv_c = 1.f / a.C;
  float q[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) q[k][v] = 1.f;

  // what a row's gradients need of memory; p: the wave's first row
  struct Row {
    float4 st;
    Raw<VT, NV> g, x, q, d, o;
  };
  auto fetch = [&](long p, bool in, Row& m) __attribute__((always_inline)) {
    m.st = make_float4(0.f, 0.f, 0.f, 0.f);
    m.g.none();
    m.x.none();
    m.q.none();
    m.d.none();
    m.o.none();
    if (!in) return;
    m.st = (a.stats + p)[lr];
    const char *pz = tz.at(p), *po = to_.at(p), *pd = td.at(p), *pf = tf.at(p), *pg = tg.at(p);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (sh.has(k)) {
        if (a.dz) {
          m.d.load(pz, tz.off + ov[k], k);
          m.o.load(po, to_.off + ov[k], k);
        }
        if (a.dout) m.g.load(pd, td.off + ov[k], k);
        m.x.load(pf, tf.off + ov[k], k);
        if (a.gate && !a.shared) m.q.load(pg, tg.off + ov[k], k);
      }
  };
  // one row's gradients; u1 and u2 take G fhat and G
  auto row = [&](long p, bool in, const Row& m, float (&u1)[NV][V], float (&u2)[NV][V]) __attribute__((always_inline)) {
    float G[NV][V], x[NV][V];
    const float4 st = m.st;
    m.g.to(G);
    m.x.to(x);
    if (a.gate && !a.shared) m.q.to(q);
    if (a.dz) {
      float d[NV][V], o[NV][V], s = 0.f, t = 0.f;
      m.d.to(d);
      m.o.to(o);
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          o[k][v] = (o[k][v] - st.z) * st.w;
          sum[0][k][v] += d[k][v] * o[k][v];
          sum[1][k][v] += d[k][v];
          d[k][v] *= ng[k][v];
          s += d[k][v];
          t += d[k][v] * o[k][v];
        }
      row_sums<BLK>(s, t, sh.G, s8);
      s *= inv_c;
      t *= inv_c;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float n = st.w * (d[k][v] - s - o[k][v] * t);
          G[k][v] += n;
        }
    }
    float b[NV][V], s = 0.f, t = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (POST) x[k][v] = (x[k][v] - st.x) * st.y;
        const float gq = G[k][v] * q[k][v], g = a.shared ? G[k][v] : gq;
        u1[k][v] += g * x[k][v];
        u2[k][v] += g;
        b[k][v] = gq * pg[k][v];
        if constexpr (POST) {
          s += b[k][v];
          t += b[k][v] * x[k][v];
        }
      }
    if constexpr (POST) {
      row_sums<BLK>(s, t, sh.G, s8);
      s *= inv_c;
      t *= inv_c;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) b[k][v] = st.y * (b[k][v] - s - x[k][v] * t);
    }
    if (!in) return;
    store_row<VT, SH, T>(sh, tr.at(p), tr.off, ov, G);
    store_row<VT, SH, T>(sh, tdf.at(p), tdf.off, ov, b);
    if (a.dgate && !a.shared) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) G[k][v] *= POST ? x[k][v] * pg[k][v] + pb[k][v] : x[k][v] * pg[k][v];
      store_row<VT, SH, T>(sh, tdg.at(p), tdg.off, ov, G);
    }
  };

  auto take_gate = [&](long g) __attribute__((always_inline)) {
    Raw<VT, NV> rq;
    rq.none();
    const char* gp = (const char*)a.gate + g * a.ldgate * (long)sizeof(T);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (sh.has(k)) rq.load(gp, ov[k], k);
    rq.to(q);
  };
  // trip counts are the same for every lane of a block whose rows are the block's
  if constexpr (!WHOLE) {
    const long g = blockIdx.x / (unsigned)a.ranges;
    const long lo = g * a.group + (blockIdx.x - g * a.ranges) * a.per, hi = min(lo + a.per, (g + 1) * a.group);
    if (a.shared) take_gate(g);
    const int turn = BLK ? 1 : 4 * rpw;
    // the next row's loads are on their way while a row is worked on
    const long p = lo + (BLK ? 0 : wave * rpw), mine = p + rl;
    Row m[2];
    fetch(p, mine < hi, m[0]);
    for (long t = 0; lo + t < hi; t += 2 * turn) {
      fetch(p + t + turn, mine + t + turn < hi, m[1]);
      row(p + t, mine + t < hi, m[0], sum[2], sum[3]);
      if (lo + t + turn >= hi) break;
      fetch(p + t + 2 * turn, mine + t + 2 * turn < hi, m[0]);
      row(p + t + turn, mine + t + turn < hi, m[1], sum[2], sum[3]);
    }
  } else {
    const long groups = a.rows / a.group, step = (long)gridDim.x * (BLK ? 1 : 4 * a.slots);
    for (long g0 = BLK ? blockIdx.x : ((long)blockIdx.x * 4 + wave) * a.slots; g0 < groups; g0 += step) {
      const long g = g0 + slot;
      const bool there = g < groups;
      float u1[NV][V], u2[NV][V];
      if (there) take_gate(g);
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) u1[k][v] = u2[k][v] = 0.f;
      for (long t = 0; t < a.group; t += side) {
        const bool in = there && t + first < a.group;
        Row m;
        fetch(g0 * a.group + t, in, m);
        row(g0 * a.group + t, in, m, u1, u2);
      }
      if constexpr (!BLK)
        for (int o = sh.G; o < sh.G * side; o <<= 1)
#pragma unroll
          for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) {
              u1[k][v] += __shfl_xor(u1[k][v], o);
              u2[k][v] += __shfl_xor(u2[k][v], o);
            }
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          // every lane of the group has the sums: the first row's takes them on
          sum[2][k][v] += first || !there ? 0.f : q[k][v] * u1[k][v];
          sum[3][k][v] += first || !there ? 0.f : q[k][v] * u2[k][v];
          u1[k][v] = POST ? pg[k][v] * u1[k][v] + pb[k][v] * u2[k][v] : pg[k][v] * u1[k][v];
        }
      if (a.dgate && there && first == 0)
        store_row<VT, SH, T>(sh, (char*)a.dgate + g * a.lddgate * (long)sizeof(T), 0u, ov, u1);
    }
  }
  if (!a.part) return;
  float* to = a.part + (long)blockIdx.x * 4 * a.C;
  if constexpr (BLK) {
#pragma unroll
    for (int z = 0; z < 4; ++z)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (sh.has(k))
#pragma unroll
          for (int v = 0; v < V; ++v) to[(long)z * a.C + sh.vec(k) * V + v] = sum[z][k][v];
  } else {
    // the wave's rows, then the four waves' sums in order
    __shared__ float ws[3][NV * V][64];
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      // (all values of a step together: one waits for LDS as long as twelve)
      for (int o = sh.G; o < 64; o <<= 1)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int v = 0; v < V; ++v) sum[z][k][v] += __shfl_xor(sum[z][k][v], o);
      if (z) __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (wave > 0) ws[wave - 1][k * V + v][lane] = sum[z][k][v];
      __syncthreads();
      if (wave == 0 && lane < sh.G)
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (sh.has(k))
#pragma unroll
            for (int v = 0; v < V; ++v) {
              const int e = k * V + v;
              to[(long)z * a.C + sh.vec(k) * V + v] = ((sum[z][k][v] + ws[0][e][lane]) + ws[1][e][lane]) + ws[2][e][lane];
            }
    }
  }
}

// Sums z0 and z0 + 1 over S of stride x C floats, columns c: 64 threads a column (k),
// summed in thread 0 of each.
__device__ __forceinline__ float2 tree_sums(const float* part, int S, int stride, int C, int c, int k, int l, int z0) {
  __shared__ float2 sh[64][17];
  float2 s = make_float2(0.f, 0.f);
  if (c < C)
#pragma unroll 8
    for (int b = k; b < S; b += 64) {
      const float* p = part + ((long)b * stride + z0) * C + c;
      s.x += p[0];
      s.y += p[C];
    }
  sh[k][l] = s;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
    if (k < o) {
      sh[k][l].x += sh[k + o][l].x;
      sh[k][l].y += sh[k + o][l].y;
    }
    __syncthreads();
  }
  return sh[0][l];
}

// The gates' gradients from the ranges' partial sums, and S1 and S2 of each gate in
// the place of U1 and U2 of its first range: the sums of dz (blockIdx.z = 0) or of G.
// MANY ranges: sixteen channels of a gate a block; else a thread a channel (35 gates of
// 2528 channels and five ranges: 33.9 us with 64 threads).
template <typename T, bool MANY>
__global__ __launch_bounds__(MANY ? 1024 : 256) void res_join(float* part, int ranges, const T* gate, long ldgate, Vectors w,
                                                 int post, T* dgate, long lddgate, int C) {
  float* of = part + (long)blockIdx.y * ranges * 4 * C;
  float2 s;
  int c;
  if constexpr (MANY) {
    const int l = threadIdx.x & 15, k = threadIdx.x >> 4;
    c = blockIdx.x * 16 + l;
    s = tree_sums(of, ranges, 4, C, c, k, l, 2 * blockIdx.z);
    if (k || c >= C) return;
  } else {
    c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    s = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int b = 0; b < ranges; ++b) {
      const float* p = of + (4L * b + 2 * blockIdx.z) * C + c;
      s.x += p[0];
      s.y += p[C];
    }
  }
  const float g = blockIdx.z ? Elt<T>::ld(gate + blockIdx.y * ldgate + c) : 1.f;
  of[2L * blockIdx.z * C + c] = g * s.x;
  of[(2L * blockIdx.z + 1) * C + c] = g * s.y;
  if (!dgate || !blockIdx.z) return;
  const float n = post ? at_or(w.post_gain, c, 1.f) * s.x + at_or(w.post_bias, c, 0.f) * s.y : s.x;
  Elt<T>::st(dgate + blockIdx.y * lddgate + c, at_or(w.scale, c, 1.f) * n);
}

// The vectors' gradients from the partial sums of S blocks, `stride` sums of C a
// block: sixteen columns a block, the pre norm's (blockIdx.y = 0) or the others.
__global__ __launch_bounds__(1024) void res_sums(const float* part, int S, int stride, Vectors w, int post,
                                                 tgp_residual_grads g, int overwrite, int C) {
  const int l = threadIdx.x & 15, k = threadIdx.x >> 4, c = blockIdx.x * 16 + l;
  const float2 s = tree_sums(part, S, stride, C, c, k, l, 2 * blockIdx.y);
  if (k || c >= C) return;
  auto put = [&](float* p, float v) {
    if (p) p[c] = overwrite ? v : p[c] + v;
  };
  if (blockIdx.y == 0) {
    put(g.pre_gain, s.x);
    put(g.pre_bias, s.y);
    return;
  }
  const float sc = at_or(w.scale, c, 1.f);
  put(g.post_gain, sc * s.x);
  put(g.post_bias, sc * s.y);
  put(g.scale, post ? at_or(w.post_gain, c, 1.f) * s.x + at_or(w.post_bias, c, 0.f) * s.y : s.x);
}

// ------------------------------------------------- plans

Vectors vectors(const tgp_residual_params& p) {
  return {p.scale, p.post_gain, p.post_bias, p.pre_gain, p.pre_bias};
}

constexpr int kFwdBlocks = 2048;   // most blocks of a forward launch
constexpr int kBlocks = 1024;      // most ranges of a backward one
constexpr int kAnyBlocks = 512;
static_assert(kRowThreads == kT, "lanes of a block");

bool any_sum(const tgp_residual_grads& g) {
  return g.scale || g.post_gain || g.post_bias || g.pre_gain || g.pre_bias;
}

// Calls f(VB, NV, BLK as constants); MOST: values a lane.  False: no kernel holds such a row.
template <int ESZ, int MOST, int WIDE, typename F>
bool with_plan(const RowPlan& p, F f) {
  bool done = false;
  auto nv = [&](auto vb, auto blk) {
    constexpr int TOP = MOST * ESZ / decltype(vb)::value;
    constexpr bool BLK = decltype(blk)::value;
    auto go = [&](auto n) {
      if constexpr (decltype(n)::value <= TOP && (BLK || decltype(n)::value <= 4)) {
        f(vb, n, blk);
        done = true;
      }
    };
    switch (p.nv) {
      case 1: return go(std::integral_constant<int, 1>());
      case 2: return go(std::integral_constant<int, 2>());
      case 3: return go(std::integral_constant<int, 3>());
      case 4: return go(std::integral_constant<int, 4>());
      case 8: return go(std::integral_constant<int, 8>());
      case kMostVectors: return go(std::integral_constant<int, kMostVectors>());
    }
  };
  auto vec = [&](auto blk) {
    if (p.vb == WIDE) nv(std::integral_constant<int, WIDE>(), blk);
    else if (p.vb == 4) nv(std::integral_constant<int, 4>(), blk);
    else if constexpr (ESZ == 2) nv(std::integral_constant<int, 2>(), blk);
  };
  if (p.g) vec(std::false_type());
  else vec(std::true_type());
  return done;
}

// f(whether there is a post norm, as a constant)
template <typename F>
void with_post(int post, F f) {
  if (post) f(std::true_type());
  else f(std::false_type());
}

// Whether a wave's rows of every tensor are within 32 bits of each other.
template <typename T>
bool near_rows(std::initializer_list<Rows> all) {
  for (const Rows& r : all)
    if (r.p && r.ld * (long)sizeof(T) * 64 >= 1l << 31) return false;
  return true;
}

// The bits of a tensor's address and row distance that the widest access has to divide.
template <typename T>
uintptr_t place(const Rows& r) { return r.p ? (uintptr_t)r.p | (uintptr_t)r.ld * sizeof(T) : 0; }

template <typename T>
hipError_t forward_t(const ResidualForward& a, hipStream_t st) {
  const double n = (double)a.s.rows * a.s.C;
  constexpr int WIDE = fwd_widest(sizeof(T));
  const RowPlan p = row_plan(sizeof(T), a.s.C, place<T>(a.r) | place<T>(a.f) | place<T>(a.gate) | place<T>(a.out) | place<T>(a.z),
                             kFwdValues, WIDE, near_rows<T>({a.r, a.f, a.out, a.z}));
  if (!p.vb || (a.gate.p && a.s.group > 0x7fffffff)) {
    ProfScope ps("residual_norm_fwd_any", 20 * n, 4 * n * sizeof(T), st);
    TGP_LAUNCH(ps, res_fwd_any<T>, dim3((unsigned)std::min<long>(a.s.rows, 2048)), dim3(kT),
               a.s.C * sizeof(float), st, (const T*)a.r.p, a.r.ld, (const T*)a.f.p, a.f.ld, (const T*)a.gate.p,
               a.gate.ld, (long)a.s.group, vectors(a.w), a.s.eps, a.s.post, (T*)a.out.p, a.out.ld, (T*)a.z.p, a.z.ld,
               (float4*)a.stats, (long)a.s.rows, a.s.C);
    return launch_status();
  }
  const FwdArgs k{a.r.p, a.f.p, a.gate.p, a.out.p, a.z.p, a.r.ld, a.f.ld, a.gate.ld, a.out.ld, a.z.ld, (long)a.s.rows,
                  (unsigned)a.s.group, vectors(a.w), a.s.eps, (float4*)a.stats, a.s.C, p.g};
  const unsigned grid = even_grid(a.s.rows, p.g == 0 ? 1 : 4 * (64 / p.g), kFwdBlocks);
  bool done = false;
  with_post(a.s.post, [&](auto post) {
    done = with_plan<sizeof(T), kFwdValues, WIDE>(p, [&](auto vb, auto nv, auto blk) {
      constexpr int VB = decltype(vb)::value, NV = decltype(nv)::value;
      constexpr bool BLK = decltype(blk)::value, POST = decltype(post)::value;
      ProfScope ps("residual_norm_fwd", 20 * n, (a.z.p ? 4 : 3) * n * sizeof(T), st);
      TGP_LAUNCH(ps, (res_fwd<T, VB, NV, BLK, POST>), dim3(grid), dim3(kT), 0, st, k);
    });
  });
  return done ? launch_status() : hipErrorNotSupported;
}

template <typename T>
hipError_t backward_t(const ResidualBackward& a, hipStream_t st) {
  constexpr int WIDE = bwd_widest(sizeof(T));
  const double n = (double)a.s.rows * a.s.C;
  const long rows = a.s.rows, group = a.gate.p ? (long)a.s.group : 1;
  const bool sums = any_sum(a.g), shared = group > 1;
  const RowPlan p = row_plan(sizeof(T), a.s.C,
                         place<T>(a.dz) | place<T>(a.dout) | (a.dz.p ? place<T>(a.out) : 0) | place<T>(a.f) | place<T>(a.gate) |
                             place<T>(a.dr) | place<T>(a.df) | place<T>(a.dgate),
                         kBwdValues, WIDE,
                         near_rows<T>({a.dz, a.dout, a.out, a.f, a.gate, a.dr, a.df, a.dgate}));
  auto add_up = [&](int S, int stride) {
    ProfScope ps("residual_norm_sums", 4.0 * S * a.s.C, 16.0 * S * a.s.C, st);
    TGP_LAUNCH(ps, res_sums, dim3(cdiv(a.s.C, 16), 2), dim3(1024), 0, st, a.part, S, stride, vectors(a.w), a.s.post, a.g,
               (int)a.overwrite, a.s.C);
  };
  BwdArgs k{a.dz.p, a.dout.p, a.out.p, a.f.p, a.gate.p, a.dr.p, a.df.p, a.dgate.p, a.dz.ld, a.dout.ld, a.out.ld, a.f.ld,
            a.gate.ld, a.dr.ld, a.df.ld, a.dgate.ld, rows, shared ? group : rows, 0, vectors(a.w), (const float4*)a.stats,
            nullptr, a.s.C, p.g, 1, 1, shared};
  const int rpw = p.g ? 64 / p.g : 1, turn = p.g ? 4 * rpw : 1;
  const long groups = rows / k.group;
  // blocks that fill the chip, of 24 rows where there are many (each leaves 16 bytes a
  // channel); of eight where a block takes a row at a time and waits for it
  const long most = std::min<long>(kBlocks, std::max<long>(256, rows / (p.g ? 24 : 8)));
  // whole groups where a wave (block) each fills the chip, or takes one in one turn
  const bool any = !p.vb, whole = shared && (groups >= (p.g ? 1024 : 512) || k.group <= rpw);
  unsigned grid;
  if (whole && any) {
    grid = (unsigned)std::min<long>(kAnyBlocks, groups);
  } else if (whole) {
    int part = 1;
    while (part < k.group && part < rpw) part <<= 1;
    k.slots = rpw / part;
    grid = even_grid(groups, p.g ? 4 * k.slots : 1, most);
  } else {
    const long want = std::max<long>(1, most / groups);
    k.per = (k.group + want - 1) / want;
    k.per = (k.per + turn - 1) / turn * turn;
    k.ranges = (int)((k.group + k.per - 1) / k.per);
    grid = (unsigned)(groups * k.ranges);
  }
  const bool join = shared && !whole && (sums || a.dgate.p);
  if (sums || join || any) k.part = a.part;
  if (any) {
    ProfScope ps("residual_norm_bwd_any", 40 * n, 6 * n * sizeof(T), st);
    if (whole) TGP_LAUNCH(ps, (res_bwd_any<T, true>), dim3(grid), dim3(kT), a.s.C * sizeof(float), st, k, a.s.post);
    else TGP_LAUNCH(ps, (res_bwd_any<T, false>), dim3(grid), dim3(kT), a.s.C * sizeof(float), st, k, a.s.post);
  }
  bool done = any;
  if (!any) with_post(a.s.post, [&](auto post) {
    done = with_plan<sizeof(T), kBwdValues, WIDE>(p, [&](auto vb, auto nv, auto blk) {
      constexpr int VB = decltype(vb)::value, NV = decltype(nv)::value;
      constexpr bool BLK = decltype(blk)::value, POST = decltype(post)::value;
      ProfScope ps("residual_norm_bwd", 40 * n, (3 + (a.dout.p ? 1 : 0) + (a.dz.p ? 2 : 0)) * n * sizeof(T), st);
      if (whole) TGP_LAUNCH(ps, (res_bwd<T, VB, NV, BLK, POST, true>), dim3(grid), dim3(kT), 0, st, k);
      else TGP_LAUNCH(ps, (res_bwd<T, VB, NV, BLK, POST, false>), dim3(grid), dim3(kT), 0, st, k);
    });
  });
  if (!done) return hipErrorNotSupported;
  if (join) {
    ProfScope ps("residual_norm_gates", 4.0 * grid * a.s.C, 16.0 * grid * a.s.C, st);
    auto go = [&](auto many) {
      constexpr bool MANY = decltype(many)::value;
      TGP_LAUNCH(ps, (res_join<T, MANY>), dim3(cdiv(a.s.C, MANY ? 16 : 256), (unsigned)groups, 2), dim3(MANY ? 1024 : 256),
                 0, st, a.part, k.ranges, (const T*)a.gate.p, a.gate.ld, vectors(a.w), a.s.post, (T*)a.dgate.p,
                 a.dgate.ld, a.s.C);
    };
    if (k.ranges > 16) go(std::true_type());
    else go(std::false_type());
  }
  if (sums && join) add_up((int)groups, 4 * k.ranges);
  else if (sums) add_up((int)grid, any && whole ? 6 : 4);
  return launch_status();
}

}  // namespace

hipError_t residual_norm_forward(const ResidualForward& a, hipStream_t st) {
  return a.s.dtype == TGP_BF16 ? forward_t<bf16_t>(a, st) : forward_t<float>(a, st);
}

size_t residual_norm_partial_floats(const tgp_residual_shape& s) {
  return (size_t)std::max<long>(6 * std::min<long>(kAnyBlocks, s.rows), 4 * std::min<long>(kBlocks, s.rows)) * s.C;
}

hipError_t residual_norm_backward(const ResidualBackward& a, hipStream_t st) {
  if (a.s.rows == 0) {
    if (!any_sum(a.g) || !a.overwrite) return hipSuccess;
    ProfScope ps("residual_norm_zero", 0, 20.0 * a.s.C, st);
    TGP_LAUNCH(ps, res_sums, dim3(cdiv(a.s.C, 16), 2), dim3(1024), 0, st, nullptr, 0, 4, Vectors{}, 0, a.g, 1, a.s.C);
    return launch_status();
  }
  return a.s.dtype == TGP_BF16 ? backward_t<bf16_t>(a, st) : backward_t<float>(a, st);
}

}  // namespace tgpk
