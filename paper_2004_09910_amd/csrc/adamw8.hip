// AdamW whose states are kept in 8 bits: m and root = sqrt(v) as E4M3 floats, a
// power of two for each 128 of them, rounded up or down by a hash so that the
// mean is the value itself.
//
// One pass over memory: 16 bytes a value and 2 more with the bfloat16 copy, eight
// values a thread, the 16 threads of a block of 128 agree on its exponents.  What
// decides a rounding is computed in float64: a value next to the border between
// two codes then goes the same way whatever the order of operations, and squares
// of float32 gradients neither overflow nor vanish.  Memory bounds it as long as those
// operations are few: codes from a float64's upper half, a root of one step (31.4 million
// values with the copy 114 us, 5.0 TB/s; with sqrt, scaled copies for the codes and
// tails that index registers 135 us).
#include <algorithm>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256, kMaxList = 48;
constexpr long kPer = 8 * kT;   // values of a block: eight a thread

struct List {
  int count;
  int blk0[kMaxList];        // first block of each tensor
  uint32_t key[kMaxList];    // of its random bits
  uint32_t first[kMaxList];  // its first value's block of kPer in the whole tensor
  tgp_adamw8_tensor t[kMaxList];
};
static_assert(sizeof(List) <= 3800, "kernel arguments");

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9e3779b1u;
  x ^= x >> 15;
  x *= 0xbb67ae85u;
  return x ^ (x >> 16);
}

// 2^k as a float64, -1023 < k < 1024.
__device__ __forceinline__ double pow2(int k) { return __longlong_as_double((long long)(k + 1023) << 52); }
// The upper half of |v|: its exponent + 1023 from bit 20 on, 20 bits of its fraction below.
__device__ __forceinline__ int upper(double v) { return (int)(__double_as_longlong(v) >> 32) & 0x7fffffff; }
constexpr int kInf = 0x7ff00000;   // of what is not finite, at least

// sqrt(v) to float64's precision, v 0 or more and a normal number: a start good to 2^-22,
// and the third-order step of 1 / sqrt(1 - d).  Not finite: NaN.
__device__ __forceinline__ double root_of(double v) {
  const double y = __builtin_amdgcn_rsq(v), r = v * y, d = fma(-r, y, 1.0);
  return v == 0 ? 0 : fma(r * d, fma(0.375, d, 0.5), r);
}

// Largest of the 16 lanes that share a block.
__device__ __forceinline__ int max16(int v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = max(v, __shfl_xor(v, o));
  return v;
}

// The codes of a block of exponent byte e.  A code's exponent and three bits of fraction
// lie on top of a float64's, and the next 17 bits of the upper half are how far a value
// lies between two codes: 16 random bits r and a half are added there, and what carries
// over rounds up.  The least normal code added to what lies below it has codes' equal
// steps there too.
struct Coder {
  double least;
  int top, off;
  __device__ __forceinline__ explicit Coder(int e) : least(pow2(e - 140)), top((e - 140 + 1023) << 20), off(8 * (e - 140 + 1022)) {}
  __device__ __forceinline__ uint32_t of(double v, uint32_t r) const {
    const bool low = upper(v) < top;
    const double s = fabs(v) + least;
    return (((uint32_t)(low ? upper(s) : upper(v)) + 2 * r + 1) >> 17) - (low ? off + 8 : off);
  }
};

struct AdamK {
  double beta1, beta2, gain1, gain2;   // gain: 1 - beta
  float rate, eps, keep, c1, rc2;
};

__global__ __launch_bounds__(kT) void adamw8_k(List l, AdamK a) {
  const int lane = threadIdx.x & 63;
  const bool before = lane < l.count && l.blk0[min(lane, kMaxList - 1)] <= (int)blockIdx.x;
  const int k = __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)) - 1);
  const tgp_adamw8_tensor t = l.t[k];
  const long i = ((long)(blockIdx.x - l.blk0[k]) * kT + threadIdx.x) * 8;
  const int n = (int)min(max(t.count - i, 0l), 8l);
  float w[8] = {}, g[8] = {};
  uint64_t m8 = 0, r8 = 0;
  uint32_t ex = 0;
  if (n > 0) ex = ((const uint16_t*)t.exps)[i / 128];
  if (n == 8) {
    *(float4*)g = *(const float4*)(t.grad + i);
    *(float4*)(g + 4) = *(const float4*)(t.grad + i + 4);
    m8 = *(const uint64_t*)(t.m + i);
    r8 = *(const uint64_t*)(t.root + i);
    *(float4*)w = *(const float4*)(t.w + i);
    *(float4*)(w + 4) = *(const float4*)(t.w + i + 4);
  } else {
#pragma unroll
    for (int z = 0; z < 8; ++z) {
      if (z >= n) continue;
      g[z] = t.grad[i + z];
      w[z] = t.w[i + z];
      m8 |= (uint64_t)t.m[i + z] << (8 * z);
      r8 |= (uint64_t)t.root[i + z] << (8 * z);
    }
  }
  // (squares of codes are exact in float32)
  const double sr = pow2((int)(ex >> 8) - 134);
  const double km = a.beta1 * pow2((int)(ex & 255) - 134), kr = a.beta2 * (sr * sr);
  double m[8], r[8];
  int em = 0, er = 0;
#pragma unroll
  for (int z = 0; z < 8; ++z) {
    const float mo = __builtin_amdgcn_cvt_f32_fp8((int)(m8 >> (8 * z)) & 255, 0);
    const float ro = __builtin_amdgcn_cvt_f32_fp8((int)(r8 >> (8 * z)) & 255, 0);
    const double gz = g[z];
    m[z] = fma((double)mo, km, a.gain1 * gz);
    r[z] = root_of(fma((double)(ro * ro), kr, a.gain2 * (gz * gz)));
    w[z] = w[z] * a.keep - a.rate * (((float)m[z] * a.c1) / ((float)r[z] * a.rc2 + a.eps));
    const int um = upper(m[z]), ur = upper(r[z]);
    em = max(em, um < kInf ? um : 0);
    er = max(er, ur < kInf ? ur : 0);
  }
  em = max16(em);
  er = max16(er);
  // 0: nothing but zeros
  em = em == 0 ? 0 : min(max((em >> 20) - 896, 1), 254);
  er = er == 0 ? 0 : min(max((er >> 20) - 896, 1), 254);
  const Coder cm8(em), cr8(er);
  const uint64_t at = (uint64_t)l.first[k] * kPer + i;
  const uint32_t key = l.key[k] + 0x9e3779b1u * (uint32_t)(at >> 32);
  uint64_t mn = 0, rn = 0;
#pragma unroll
  for (int z = 0; z < 8; ++z) {
    const uint32_t bits = mix((uint32_t)(at + z) ^ key);
    uint32_t cm = 0x7f, cr = 0x7f;
    if (upper(m[z]) < kInf) cm = cm8.of(m[z], bits & 0xffff) | ((uint32_t)(__double_as_longlong(m[z]) >> 56) & 0x80);
    if (upper(r[z]) < kInf) cr = upper(r[z]) > 0 ? max(cr8.of(r[z], bits >> 16), 1u) : 0;
    mn |= (uint64_t)cm << (8 * z);
    rn |= (uint64_t)cr << (8 * z);
  }
  if (n > 0 && i % 128 == 0) ((uint16_t*)t.exps)[i / 128] = (uint16_t)(em | er << 8);
  bf16_t* w16 = (bf16_t*)t.w16;
  if (n == 8) {
    *(uint64_t*)(t.m + i) = mn;
    *(uint64_t*)(t.root + i) = rn;
    *(float4*)(t.w + i) = *(float4*)w;
    *(float4*)(t.w + i + 4) = *(float4*)(w + 4);
    if (w16) {
      uint32_t d[4];
#pragma unroll
      for (int z = 0; z < 4; ++z) d[z] = pack_bf16(w[2 * z], w[2 * z + 1]);
      *(uint4*)(w16 + i) = make_uint4(d[0], d[1], d[2], d[3]);
    }
  } else {
#pragma unroll
    for (int z = 0; z < 8; ++z) {
      if (z >= n) continue;
      t.m[i + z] = (uint8_t)(mn >> (8 * z));
      t.root[i + z] = (uint8_t)(rn >> (8 * z));
      t.w[i + z] = w[z];
      if (w16) w16[i + z] = (bf16_t)f2bf(w[z]);
    }
  }
}

}  // namespace

hipError_t adamw8_step(int n, const tgp_adamw8_tensor* t, float rate, double beta1, double beta2,
                       float eps, float decay, float c1, float rc2, uint64_t seed, hipStream_t st) {
  constexpr int kMost = 1 << 20;   // blocks of a launch
  const AdamK a{beta1, beta2, 1 - beta1, 1 - beta2, rate, eps, 1.f - decay, c1, rc2};
  List l;
  l.count = 0;
  int blocks = 0;
  double bytes = 0;
  auto flush = [&]() -> hipError_t {
    if (l.count == 0) return hipSuccess;
    ProfScope ps("adamw8_step", 0, bytes, st);
    TGP_LAUNCH(ps, adamw8_k, dim3((unsigned)blocks), dim3(kT), 0, st, l, a);
    l.count = 0;
    blocks = 0;
    bytes = 0;
    return launch_status();
  };
  for (int k = 0; k < n; ++k) {
    const uint32_t key = mix((uint32_t)seed ^ mix((uint32_t)(seed >> 32) + mix((uint32_t)k + 1)));
    for (long i = 0; i < t[k].count;) {
      if (l.count == kMaxList || blocks >= kMost) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      const long len = std::min<long>(kMost * kPer, t[k].count - i);
      tgp_adamw8_tensor& d = l.t[l.count] = t[k];
      d.count = len;
      d.w += i;
      if (d.w16) d.w16 = (bf16_t*)d.w16 + i;
      d.grad += i;
      d.m += i;
      d.root += i;
      d.exps += i / TGP_ADAMW8_BLOCK * 2;
      l.key[l.count] = key;
      l.first[l.count] = (uint32_t)(i / kPer);
      l.blk0[l.count++] = blocks;
      blocks += (int)((len + kPer - 1) / kPer);
      bytes += (double)len * (16 + (d.w16 ? 2 : 0));
      i += len;
    }
  }
  return flush();
}

}  // namespace tgpk
