// The weights' step: w (1 - decay) - rate update for tensors with an
// orthogonalised update, AdamW for the others, and the bfloat16 copy of the
// weights in the same pass.  Purely a matter of memory: 16-byte accesses, eight
// values a thread, one launch over many tensors, whose addresses travel in the
// kernel's arguments.  31.4 million weights of 19 matrices with their bfloat16
// copies, 377 MB, and 5889 values by AdamW: 73 us, 5.2 TB/s.
#include <algorithm>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256, kMaxList = 48;
constexpr long kPer = 8 * kT;   // values of a block: eight a thread

template <typename D>
struct List {
  int count;
  int blk0[kMaxList];   // first block of each tensor
  D t[kMaxList];
};

// The tensor of this block: the last to start at or before it.
template <typename D>
__device__ __forceinline__ int find(const List<D>& l, int blk) {
  static_assert(kMaxList <= 64, "a lane each");
  const int lane = threadIdx.x & 63;
  const bool before = lane < l.count && l.blk0[min(lane, kMaxList - 1)] <= blk;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)) - 1);
}

// Eight values from i on (all of them inside the tensor), as floats.
__device__ __forceinline__ void load8(const float* p, long i, float (&f)[8]) {
  const float4 a = *(const float4*)(p + i), b = *(const float4*)(p + i + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t* p, long i, float (&f)[8]) {
  const uint4 v = *(const uint4*)(p + i);
  const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) { f[2 * k] = bf2f(d[k] & 0xffffu); f[2 * k + 1] = bf2f(d[k] >> 16); }
}
__device__ __forceinline__ void store8(float* p, long i, const float (&f)[8]) {
  *(float4*)(p + i) = make_float4(f[0], f[1], f[2], f[3]);
  *(float4*)(p + i + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(bf16_t* p, long i, const float (&f)[8]) {
  uint32_t d[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) d[k] = f2bf(f[2 * k]) | (f2bf(f[2 * k + 1]) << 16);
  *(uint4*)(p + i) = make_uint4(d[0], d[1], d[2], d[3]);
}
__device__ __forceinline__ void store_w(float* w, bf16_t* w16, long i, float v) {
  w[i] = v;
  if (w16) w16[i] = (bf16_t)f2bf(v);
}

__global__ __launch_bounds__(kT) void weight_step_k(List<tgp_step_tensor> l, float keep) {
  const int k = find(l, blockIdx.x);
  const tgp_step_tensor t = l.t[k];
  const long i = ((long)(blockIdx.x - l.blk0[k]) * kT + threadIdx.x) * 8;
  const bf16_t* u = (const bf16_t*)t.update;
  if (i + 8 <= t.count) {
    float w[8], o[8];
    load8(t.w, i, w);
    load8(u, i, o);
#pragma unroll
    for (int v = 0; v < 8; ++v) w[v] = w[v] * keep - t.rate * o[v];
    store8(t.w, i, w);
    if (t.w16) store8((bf16_t*)t.w16, i, w);
  } else {
    for (long e = i; e < t.count; ++e)
      store_w(t.w, (bf16_t*)t.w16, e, t.w[e] * keep - t.rate * bf2f(u[e]));
  }
}

struct AdamK {
  float rate, beta1, beta2, eps, keep, c1, c2;
  __device__ __forceinline__ void step(float& w, float g, float& m, float& v) const {
    m = beta1 * m + (1.f - beta1) * g;
    v = beta2 * v + (1.f - beta2) * (g * g);
    w = w * keep - rate * ((m * c1) / (sqrtf(v * c2) + eps));
  }
};

__global__ __launch_bounds__(kT) void adamw_k(List<tgp_adamw_tensor> l, AdamK a) {
  const int k = find(l, blockIdx.x);
  const tgp_adamw_tensor t = l.t[k];
  const long i = ((long)(blockIdx.x - l.blk0[k]) * kT + threadIdx.x) * 8;
  if (i + 8 <= t.count) {
    float w[8], g[8], m[8], v[8];
    load8(t.grad, i, g);
    load8(t.m, i, m);
    load8(t.v, i, v);
    load8(t.w, i, w);
#pragma unroll
    for (int z = 0; z < 8; ++z) a.step(w[z], g[z], m[z], v[z]);
    store8(t.m, i, m);
    store8(t.v, i, v);
    store8(t.w, i, w);
    if (t.w16) store8((bf16_t*)t.w16, i, w);
  } else {
    for (long e = i; e < t.count; ++e) {
      float w = t.w[e], m = t.m[e], v = t.v[e];
      a.step(w, t.grad[e], m, v);
      t.m[e] = m;
      t.v[e] = v;
      store_w(t.w, (bf16_t*)t.w16, e, w);
    }
  }
}

// A tensor's piece of `len` values from `at` on.
void cut(tgp_step_tensor& t, long at, long len) {
  t.count = len;
  t.w += at;
  if (t.w16) t.w16 = (bf16_t*)t.w16 + at;
  t.update = (const bf16_t*)t.update + at;
}
void cut(tgp_adamw_tensor& t, long at, long len) {
  t.count = len;
  t.w += at;
  if (t.w16) t.w16 = (bf16_t*)t.w16 + at;
  t.grad += at;
  t.m += at;
  t.v += at;
}

// go(list, blocks) for every kMaxList tensors that hold values; a tensor of
// more blocks than a grid should have goes in pieces.
template <typename D, typename F>
hipError_t each_list(int n, const D* t, F go) {
  constexpr int kMost = 1 << 20;   // blocks
  List<D> l;
  l.count = 0;
  int blocks = 0;
  auto flush = [&]() -> hipError_t {
    if (l.count == 0) return hipSuccess;
    go(l, (unsigned)blocks);
    l.count = 0;
    blocks = 0;
    return launch_status();
  };
  for (int k = 0; k < n; ++k)
    for (long i = 0; i < t[k].count;) {
      if (l.count == kMaxList || blocks >= kMost) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      const long len = std::min<long>(kMost * kPer, t[k].count - i);
      l.t[l.count] = t[k];
      cut(l.t[l.count], i, len);
      l.blk0[l.count++] = blocks;
      blocks += (int)((len + kPer - 1) / kPer);
      i += len;
    }
  return flush();
}

template <typename D>
double values(const List<D>& l, int extra, int each) {   // bytes: each per value, extra where w16 is set
  double b = 0;
  for (int k = 0; k < l.count; ++k) b += (double)l.t[k].count * (each + (l.t[k].w16 ? extra : 0));
  return b;
}

}  // namespace

hipError_t weight_step(int n, const tgp_step_tensor* t, float decay, hipStream_t st) {
  return each_list(n, t, [&](const List<tgp_step_tensor>& l, unsigned blocks) {
    ProfScope ps("weight_step", 0, values(l, 2, 10), st);
    TGP_LAUNCH(ps, weight_step_k, dim3(blocks), dim3(kT), 0, st, l, 1.f - decay);
  });
}

hipError_t adamw_step(int n, const tgp_adamw_tensor* t, float rate, float beta1, float beta2,
                      float eps, float decay, float c1, float c2, hipStream_t st) {
  const AdamK a{rate, beta1, beta2, eps, 1.f - decay, c1, c2};
  return each_list(n, t, [&](const List<tgp_adamw_tensor>& l, unsigned blocks) {
    ProfScope ps("adamw_step", 0, values(l, 2, 28), st);
    TGP_LAUNCH(ps, adamw_k, dim3(blocks), dim3(kT), 0, st, l, a);
  });
}

}  // namespace tgpk
