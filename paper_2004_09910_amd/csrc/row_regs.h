// Rows of a tensor held in registers: vectors of a row dealt over lanes, and sums
// over them.  Internal linkage.
#pragma once
#include <type_traits>

#include "common.h"

namespace tgpk {
namespace {

constexpr int kT = 256;   // threads of a block

// Sum over the block's kT threads, the same value in every thread: a wave's
// xor tree, then the waves' sums in order.
template <typename F>
__device__ __forceinline__ F block_sum(F v, F* s4) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (s4[0] + s4[1]) + (s4[2] + s4[3]);
  __syncthreads();
  return v;
}

// VB bytes of T as one access, and their values as floats.
template <typename T, int VB> struct Vec;
template <> struct Vec<bf16_t, 16> {
  typedef uint4 mem, raw;
  static __device__ __forceinline__ void un(raw v, float* f) {
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf2f(d[i] & 0xffffu); f[2 * i + 1] = bf2f(d[i] >> 16); }
  }
  static __device__ __forceinline__ raw pk(const float* f) {
    uint32_t d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = f2bf(f[2 * i]) | (f2bf(f[2 * i + 1]) << 16);
    return make_uint4(d[0], d[1], d[2], d[3]);
  }
};
template <> struct Vec<bf16_t, 8> {
  typedef uint2 mem, raw;
  static __device__ __forceinline__ void un(raw v, float* f) {
    f[0] = bf2f(v.x & 0xffffu); f[1] = bf2f(v.x >> 16); f[2] = bf2f(v.y & 0xffffu); f[3] = bf2f(v.y >> 16);
  }
  static __device__ __forceinline__ raw pk(const float* f) {
    return make_uint2(f2bf(f[0]) | (f2bf(f[1]) << 16), f2bf(f[2]) | (f2bf(f[3]) << 16));
  }
};
template <> struct Vec<bf16_t, 4> {
  typedef uint32_t mem, raw;
  static __device__ __forceinline__ void un(raw v, float* f) { f[0] = bf2f(v & 0xffffu); f[1] = bf2f(v >> 16); }
  static __device__ __forceinline__ raw pk(const float* f) { return f2bf(f[0]) | (f2bf(f[1]) << 16); }
};
template <> struct Vec<bf16_t, 2> {
  typedef uint16_t mem;
  typedef uint32_t raw;   // a register each: two loads into one's halves wait for each other
  static __device__ __forceinline__ void un(raw v, float* f) { f[0] = bf2f(v); }
  static __device__ __forceinline__ raw pk(const float* f) { return f2bf(f[0]); }
};
template <> struct Vec<float, 16> {
  typedef float4 mem, raw;
  static __device__ __forceinline__ void un(raw v, float* f) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
  static __device__ __forceinline__ raw pk(const float* f) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Vec<float, 4> {
  typedef float mem, raw;
  static __device__ __forceinline__ void un(raw v, float* f) { f[0] = v; }
  static __device__ __forceinline__ raw pk(const float* f) { return f[0]; }
};

// v of the lane that DPP control CTRL pairs with this one.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

// Sum over the lanes of one row: the G lanes of a group (G a power of two,
// the same for the whole launch), or the whole block.  Neighbours are added
// first; once the lanes of a half agree, mirroring reaches the other half.
template <bool BLK>
__device__ __forceinline__ float row_sum(float v, int G, float* s4) {
  if constexpr (BLK) {
    return block_sum(v, s4);
  } else {
    if (G >= 2) v += dpp<0xB1>(v);     // lanes 1 0 3 2
    if (G >= 4) v += dpp<0x4E>(v);     // lanes 2 3 0 1
    if (G >= 8) v += dpp<0x141>(v);    // mirror of 8
    if (G >= 16) v += dpp<0x140>(v);   // mirror of 16
    if (G >= 32) v += __shfl_xor(v, 16);
    if (G >= 64) v += __shfl_xor(v, 32);
    return v;
  }
}

// Two such sums side by side.
template <bool BLK>
__device__ __forceinline__ void row_sums(float& s, float& t, int G, float (*s8)[4]) {
  if constexpr (BLK) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      s += __shfl_xor(s, o);
      t += __shfl_xor(t, o);
    }
    if ((threadIdx.x & 63) == 0) {
      s8[0][threadIdx.x >> 6] = s;
      s8[1][threadIdx.x >> 6] = t;
    }
    __syncthreads();
    s = (s8[0][0] + s8[0][1]) + (s8[0][2] + s8[0][3]);
    t = (s8[1][0] + s8[1][1]) + (s8[1][2] + s8[1][3]);
    __syncthreads();
  } else {
    auto step = [&](auto c) __attribute__((always_inline)) {
      s += dpp<decltype(c)::value>(s);
      t += dpp<decltype(c)::value>(t);
    };
    typedef std::integral_constant<int, 0xB1> s1;
    typedef std::integral_constant<int, 0x4E> s2;
    typedef std::integral_constant<int, 0x141> s4;
    typedef std::integral_constant<int, 0x140> s8th;
    if (G >= 16) {
      step(s1());
      step(s2());
      step(s4());
      step(s8th());
      if (G >= 32) {
        s += __shfl_xor(s, 16);
        t += __shfl_xor(t, 16);
        if (G >= 64) {
          s += __shfl_xor(s, 32);
          t += __shfl_xor(t, 32);
        }
      }
    } else if (G == 8) {
      step(s1());
      step(s2());
      step(s4());
    } else if (G >= 2) {
      step(s1());
      if (G == 4) step(s2());
    }
  }
}

// How the lanes of a block share rows.  A row's nvec vectors of VB bytes lie
// on G lanes of a wave (64 / G rows side by side), or (BLK) on the block's
// 256 lanes, NV a lane: vector k of lane l is number l + G k.
template <typename T, int VB, int NV, bool BLK>
struct Share {
  static constexpr int V = VB / (int)sizeof(T);
  int l, G, nvec;
  long row0, step;   // first row of this lane, rows from one turn to the next
  // blocks: those of the launch that take rows
  __device__ __forceinline__ Share(int C, int g, int blocks) : G(BLK ? kT : g), nvec(C / V) {
    const int per = BLK ? 1 : 64 / G, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    l = BLK ? threadIdx.x : lane & (G - 1);
    row0 = BLK ? blockIdx.x : ((long)blockIdx.x * 4 + wave) * per + lane / G;
    step = (long)blocks * (BLK ? 1 : 4 * per);
  }
  // first row of the block's first turn
  __device__ __forceinline__ long first() const { return BLK ? row0 : (long)blockIdx.x * 4 * (64 / G); }
  __device__ __forceinline__ bool has(int k) const { return l + G * k < nvec; }
  __device__ __forceinline__ int vec(int k) const { return l + G * k; }
  // the lane's channels of a float32 vector over channels (NULL: `none`)
  __device__ __forceinline__ void channels(const float* p, float none, float (&f)[NV][V]) const {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));   // p is at a multiple of 4 only
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int v = 0; v < V; ++v) f[k][v] = none;
      if (!p || !has(k)) continue;
      const float* q = p + (long)vec(k) * V;
      if constexpr (V % 4 == 0) {
#pragma unroll
        for (int v = 0; v < V; v += 4) {
          const f4 t = *(const f4*)(q + v);
          f[k][v] = t.x; f[k][v + 1] = t.y; f[k][v + 2] = t.z; f[k][v + 3] = t.w;
        }
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) f[k][v] = q[v];
      }
    }
  }
};

// At most `most` blocks, each with as many turns over its rows as the others.
unsigned even_grid(long rows, long per_block, long most) {
  const long blocks = (rows + per_block - 1) / per_block, turns = (blocks + most - 1) / most;
  return (unsigned)((blocks + turns - 1) / turns);
}

}  // namespace
}  // namespace tgpk
