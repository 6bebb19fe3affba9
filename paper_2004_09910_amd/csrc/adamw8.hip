// AdamW whose states are kept in 8 bits: m and root = sqrt(v) as E4M3 floats, a
// power of two for each 128 of them, rounded up or down by a hash so that the
// mean is the value itself.
//
// One pass over memory: 16 bytes a value and 2 more with the bfloat16 copy, eight
// values a thread, the 16 threads of a block of 128 agree on its exponents.  What
// decides a rounding is computed in float64: a value next to the border between
// two codes then goes the same way whatever the order of operations, and squares
// of float32 gradients neither overflow nor vanish.
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
// floor(log2(v)) of a normal v > 0 (very small otherwise).
__device__ __forceinline__ int log2_of(double v) { return (int)((__double_as_longlong(v) >> 52) & 0x7ff) - 1023; }

// Largest of the 16 lanes that share a block.
__device__ __forceinline__ int max16(int v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = max(v, __shfl_xor(v, o));
  return v;
}

// The code of |v| for a block of exponent byte e; r: 16 random bits.
__device__ __forceinline__ uint32_t encode(double v, int e, uint32_t r) {
  const double t = fabs(v) * pow2(134 - e);
  const int k = max(log2_of(t), -6);
  return ((k + 6) << 3) + (uint32_t)(t * pow2(3 - k) + (r + 0.5) * 0x1p-16);
}

struct AdamK {
  double beta1, beta2;
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
    for (int z = 0; z < n; ++z) {
      g[z] = t.grad[i + z];
      w[z] = t.w[i + z];
      m8 |= (uint64_t)t.m[i + z] << (8 * z);
      r8 |= (uint64_t)t.root[i + z] << (8 * z);
    }
  }
  const double sm = pow2((int)(ex & 255) - 134), sr = pow2((int)(ex >> 8) - 134);
  double m[8], r[8];
  int em = -4096, er = -4096;
#pragma unroll
  for (int z = 0; z < 8; ++z) {
    const double mo = __builtin_amdgcn_cvt_f32_fp8((int)(m8 >> (8 * z)) & 255, 0) * sm;
    const double ro = __builtin_amdgcn_cvt_f32_fp8((int)(r8 >> (8 * z)) & 255, 0) * sr;
    const double gz = g[z];
    m[z] = a.beta1 * mo + (1 - a.beta1) * gz;
    r[z] = sqrt(a.beta2 * (ro * ro) + (1 - a.beta2) * (gz * gz));
    w[z] = w[z] * a.keep - a.rate * (((float)m[z] * a.c1) / ((float)r[z] * a.rc2 + a.eps));
    if (m[z] != 0 && isfinite(m[z])) em = max(em, log2_of(fabs(m[z])));
    if (r[z] != 0 && isfinite(r[z])) er = max(er, log2_of(r[z]));
  }
  em = max16(em);
  er = max16(er);
  // 0: nothing but zeros
  em = em == -4096 ? 0 : min(max(em + 127, 1), 254);
  er = er == -4096 ? 0 : min(max(er + 127, 1), 254);
  const uint64_t at = (uint64_t)l.first[k] * kPer + i;
  const uint32_t key = l.key[k] + 0x9e3779b1u * (uint32_t)(at >> 32);
  uint64_t mn = 0, rn = 0;
#pragma unroll
  for (int z = 0; z < 8; ++z) {
    const uint32_t bits = mix((uint32_t)(at + z) ^ key);
    uint32_t cm = 0x7f, cr = 0x7f;
    if (isfinite(m[z])) cm = encode(m[z], em, bits & 0xffff) | (signbit(m[z]) ? 0x80 : 0);
    if (isfinite(r[z])) cr = r[z] > 0 ? max(encode(r[z], er, bits >> 16), 1u) : 0;
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
      for (int z = 0; z < 4; ++z) d[z] = f2bf(w[2 * z]) | (f2bf(w[2 * z + 1]) << 16);
      *(uint4*)(w16 + i) = make_uint4(d[0], d[1], d[2], d[3]);
    }
  } else {
    for (int z = 0; z < n; ++z) {
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
  const AdamK a{beta1, beta2, rate, eps, 1.f - decay, c1, rc2};
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
