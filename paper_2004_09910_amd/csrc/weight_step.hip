// The weights' step: w (1 - decay) - rate update for tensors with an
// orthogonalised update, AdamW for the others, and the bfloat16 copy of the
// weights in the same pass.  Purely a matter of memory: one launch over many
// tensors, whose addresses travel in the kernel's arguments.
#include <algorithm>

#include "common.h"
#include "prof.h"
#include "train_ops.h"

namespace tgpk {
namespace {

constexpr int kT = 256, kMaxList = 48;
constexpr long kPer = 4 * kT;   // values of a block and pass

template <typename D>
struct List {
  int count;
  D t[kMaxList];
  long blk0[kMaxList + 1];   // first block of each tensor; [count] = all blocks
};

// Finds the tensor of this block (count <= kMaxList, uniform over the block).
template <typename D>
__device__ __forceinline__ int find(const List<D>& l, long blk) {
  int k = 0;
  while (k + 1 < l.count && blk >= l.blk0[k + 1]) ++k;
  return k;
}

__device__ __forceinline__ void store_w(float* w, bf16_t* w16, long i, float v) {
  w[i] = v;
  if (w16) w16[i] = (bf16_t)f2bf(v);
}

__global__ __launch_bounds__(kT) void weight_step_k(List<tgp_step_tensor> l, float keep) {
  const int k = find(l, blockIdx.x);
  const tgp_step_tensor t = l.t[k];
  const long i0 = ((long)blockIdx.x - l.blk0[k]) * kPer;
  const bf16_t* u = (const bf16_t*)t.update;
  for (long i = i0 + threadIdx.x; i < i0 + kPer && i < t.count; i += kT)
    store_w(t.w, (bf16_t*)t.w16, i, t.w[i] * keep - t.rate * bf2f(u[i]));
}

struct AdamK {
  float rate, beta1, beta2, eps, keep, c1, c2;
};

__global__ __launch_bounds__(kT) void adamw_k(List<tgp_adamw_tensor> l, AdamK a) {
  const int k = find(l, blockIdx.x);
  const tgp_adamw_tensor t = l.t[k];
  const long i0 = ((long)blockIdx.x - l.blk0[k]) * kPer;
  for (long i = i0 + threadIdx.x; i < i0 + kPer && i < t.count; i += kT) {
    const float g = t.grad[i];
    const float m = a.beta1 * t.m[i] + (1.f - a.beta1) * g;
    const float v = a.beta2 * t.v[i] + (1.f - a.beta2) * (g * g);
    t.m[i] = m;
    t.v[i] = v;
    store_w(t.w, (bf16_t*)t.w16, i,
            t.w[i] * a.keep - a.rate * ((m * a.c1) / (sqrtf(v * a.c2) + a.eps)));
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
  constexpr long kMost = kPer << 20;
  List<D> l;
  l.count = 0;
  long blocks = 0;
  auto flush = [&]() -> hipError_t {
    if (l.count == 0) return hipSuccess;
    l.blk0[l.count] = blocks;
    go(l, blocks);
    l.count = 0;
    blocks = 0;
    return launch_status();
  };
  for (int k = 0; k < n; ++k)
    for (long i = 0; i < t[k].count;) {
      if (l.count == kMaxList || blocks >= kMost / kPer) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      const long len = std::min<long>(kMost, t[k].count - i);
      l.t[l.count] = t[k];
      cut(l.t[l.count], i, len);
      l.blk0[l.count++] = blocks;
      blocks += (len + kPer - 1) / kPer;
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
  return each_list(n, t, [&](const List<tgp_step_tensor>& l, long blocks) {
    ProfScope ps("weight_step", 0, values(l, 2, 10), st);
    TGP_LAUNCH(ps, weight_step_k, dim3((unsigned)blocks), dim3(kT), 0, st, l, 1.f - decay);
  });
}

hipError_t adamw_step(int n, const tgp_adamw_tensor* t, float rate, float beta1, float beta2,
                      float eps, float decay, float c1, float c2, hipStream_t st) {
  const AdamK a{rate, beta1, beta2, eps, 1.f - decay, c1, c2};
  return each_list(n, t, [&](const List<tgp_adamw_tensor>& l, long blocks) {
    ProfScope ps("adamw_step", 0, values(l, 2, 28), st);
    TGP_LAUNCH(ps, adamw_k, dim3((unsigned)blocks), dim3(kT), 0, st, l, a);
  });
}

}  // namespace tgpk
