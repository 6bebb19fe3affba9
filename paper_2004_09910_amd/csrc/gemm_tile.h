// Tile products of bfloat16 matrices for gfx950: operands fed to a ring of LDS
// slots by DMA, fragments read from there, sums in registers.  Internal linkage.
//
// A stage is BK values of the sum.  An operand is a matrix whose rows are those of
// the tile, contiguous in the sum, or (KS) whose rows are the sum's, contiguous
// in the tile.  In LDS a stage of the first kind is rows of BK values, of the
// second BK rows of the tile's width; fragments of the second are gathered by
// transpose loads.  16-byte chunks are XOR-swizzled so that what a fragment's
// load takes at once lies in distinct banks: sixteen rows at one chunk, or 64
// bytes of four rows of the sum.
//
// Whatever lies outside a matrix (rows, columns, the end of the sum) is a buffer
// read out of range, zeros: 0 x 0, so that no infinity of a neighbour gets in.
// Rows' starts are at multiples of 16 bytes and lengths multiples of 8 values.
#pragma once
#include <type_traits>

#include "common.h"
#include "mfma_util.h"

namespace tgpk {
namespace {

// f(0), f(1), .. f(N - 1), as constants
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>());
  }
}

// N x 16 bytes a lane from a buffer to LDS at dst, dst + STEP, .. (lane l at
// + 16 l), as dma16.
template <int N, int STEP>
__device__ __forceinline__ void dma_n(u32x4 rsrc, unsigned dst, const int (&vo)[N]) {
  unsigned saved;
#define TGP_HEAD "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %2, 0 offen lds\n\t"
#define TGP_MORE(v) "s_add_u32 m0, m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 " v ", %2, 0 offen lds\n\t"
#define TGP_TAIL "s_mov_b32 m0, %0"
#define TGP_OPS "=&s"(saved) : "s"(dst), "s"(rsrc), "i"(STEP)
  if constexpr (N == 1)
    asm volatile(TGP_HEAD TGP_TAIL : TGP_OPS, "v"(vo[0]) : "memory", "scc");
  else if constexpr (N == 2)
    asm volatile(TGP_HEAD TGP_MORE("%5") TGP_TAIL : TGP_OPS, "v"(vo[0]), "v"(vo[1]) : "memory", "scc");
  else if constexpr (N == 3)
    asm volatile(TGP_HEAD TGP_MORE("%5") TGP_MORE("%6") TGP_TAIL
                 : TGP_OPS, "v"(vo[0]), "v"(vo[1]), "v"(vo[2]) : "memory", "scc");
  else {
    static_assert(N == 4, "loads of a stage");
    asm volatile(TGP_HEAD TGP_MORE("%5") TGP_MORE("%6") TGP_MORE("%7") TGP_TAIL
                 : TGP_OPS, "v"(vo[0]), "v"(vo[1]), "v"(vo[2]), "v"(vo[3]) : "memory", "scc");
  }
#undef TGP_HEAD
#undef TGP_MORE
#undef TGP_TAIL
#undef TGP_OPS
}

// One operand of a block's tile: R rows (columns) of it, NW waves.
template <int R, int BK, bool KS, int NW>
struct Feed {
  static constexpr int CPR = KS ? R / 8 : BK / 8;   // chunks of an LDS row
  static constexpr int BYTES = R * BK * 2, LOADS = BYTES / 1024 / NW;
  static_assert(BYTES % (1024 * NW) == 0 && LOADS >= 1 && NW % 2 == 0, "whole rounds of DMA");

  int vo[LOADS];      // byte offsets of the lane's chunks
  int kq;             // first value of the sum in them (not KS)
  long ldb;           // bytes from one row to the next
  unsigned long at;   // address of the stage's first value

  // Chunk q of LDS row `row` lies at chunk q ^ swz(row).
  __device__ __forceinline__ static int swz(int row) {
    if constexpr (!KS) return BK == 64 ? (row & 2) << 1 | (row >> 2 & 3) : (row >> 2) & 3;
    else if constexpr (R >= 128) return (row & 3) << 2;
    else if constexpr (R == 64) return ((row >> 1) & 1) << 2;
    else return 0;
  }

  // ld: of the matrix; have: rows (KS: columns) of it from the tile's first on.
  __device__ __forceinline__ void init(long ld, int have) {
    static_assert(BK == 32 || BK == 64, "stage");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ldb = ld * 2;
    kq = 0;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int row = (wave + u * NW) * (64 / CPR) + lane / CPR, q = (lane % CPR) ^ swz(row);
      const bool in = KS ? q * 8 < have : row < have;
      vo[u] = in ? (int)(row * ldb) + q * 16 : kOob;
      if (!KS && u == 0) kq = q * 8;   // the same in all: swz sees the wave's parity alone
    }
  }

  // The sum starts at value k of the matrix whose tile starts at row (column) i0.
  __device__ __forceinline__ void seek(const bf16_t* p, long i0, long k) {
    const unsigned long a = (unsigned long)p + (KS ? k * ldb + i0 * 2 : i0 * ldb + k * 2);
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a);   // (it returns an int)
    const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
    at = (unsigned long)hi << 32 | lo;
  }

  // The next stage: left, values of the sum from its first on.  Its loads u = 0 .. LOADS - 1
  // go to LDS from dst on (of the wave: + 1024 wave).
  u32x4 rsrc;
  bool in;     // the lane's chunks are inside the sum (not KS)
  __device__ __forceinline__ void next(int left) {
    rsrc = u32x4{(unsigned)at, (unsigned)(at >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
    if constexpr (KS) {
      if (left < BK) rsrc[2] = (unsigned)(left * (int)ldb);
      rsrc[2] = __builtin_amdgcn_readfirstlane(rsrc[2]);
      at += (unsigned long)(BK * ldb);
    } else {
      in = kq < left;
      at += BK * 2;
    }
  }
  template <int U>
  __device__ __forceinline__ void load(unsigned dst) const {
    const int v[1] = {KS || in ? vo[U] : kOob};
    dma_n<1, 0>(rsrc, dst + U * NW * 1024, v);
  }

  // Byte offset of this lane's part of the fragment of rows f .. f + 31, and (KS) of
  // its column part: the fragment of step h (16 values) of a stage is read by frag.
  __device__ __forceinline__ static int place(int f) {
    const int lane = threadIdx.x & 63;
    if constexpr (!KS) {
      const int row = f + (lane & 31);
      return row * BK * 2 + (((lane >> 5) ^ swz(row)) << 4);
    } else {
      const int k = 8 * (lane >> 5) + ((lane & 15) >> 2);
      const int q = f / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      return k * R * 2 + ((q ^ swz(k)) << 4) + 8 * (lane & 1);
    }
  }
  __device__ __forceinline__ static u32x4 frag(const unsigned char* s, int place, int h) {
    if constexpr (!KS) return *(const u32x4*)(s + (place ^ (32 * h)));
    else return frag_tr(s + place + h * 16 * R * 2, R * 2);
  }
};

// What one launch's tile products run over: `segs` pairs of matrices of the same
// shape one after the other (parts of a sum whose factors are split).
constexpr int kMaxSegs = 12;
template <int NB, int NA = 1>
struct Segs {
  const bf16_t* a[kMaxSegs][NA];
  const bf16_t* b[kMaxSegs][NB];
  int n;
};

// WM x WN waves of MT x NT fragments of 32 x 32, for each of NB right factors that
// share the left one, whose NA parts are summed; NS slots.  Lane l of a wave holds row l % 32 of a fragment and
// its columns 8 (v / 4) + 4 (l / 32) + v % 4.
template <int MT_, int NT_, int WM_, int WN_, int BK_, int NS_, bool AKS, bool BKS, int NB_, int NA_ = 1>
struct Product {
  static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, BK = BK_, NS = NS_, NB = NB_, NA = NA_;
  static constexpr int NW = WM * WN, T = 64 * NW, BM = 32 * MT * WM, BN = 32 * NT * WN;
  typedef Feed<BM, BK, AKS, NW> FA;
  typedef Feed<BN, BK, BKS, NW> FB;
  static constexpr int SLOT = NA * FA::BYTES + NB * FB::BYTES, LPS = NA * FA::LOADS + NB * FB::LOADS;
  static constexpr int LDS = NS * SLOT;
  static_assert(LDS <= 160 * 1024 && NS >= 2, "LDS ring");

  f32x16_t acc[NB][MT][NT];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[b][i][j] = f32x16_t{};
  }

  // The sums over values k0 .. k1 (k0 a multiple of BK) of every pair of `s`: rows
  // i0 .. of A (m in all), columns j0 .. of B (n).  extra(a, i, p): more products of a
  // left fragment (u32x4, fragment row i) of pair p.
  template <int SA, typename X>
  __device__ __forceinline__ void run(unsigned char* ring, const Segs<NB, SA>& s, long lda, long ldb, int m, int n, int i0,
                                      int j0, int k0, int k1, X extra) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    static_assert(SA >= NA, "parts");
    FA fa[NA];
    FB fb[NB];
#pragma unroll
    for (int q = 0; q < NA; ++q) fa[q].init(lda, m - i0);
#pragma unroll
    for (int b = 0; b < NB; ++b) fb[b].init(ldb, n - j0);
    const int per = (k1 - k0 + BK - 1) / BK, total = per * s.n;
    const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(unsigned long)TGP_LDS(ring) + wave * 1024);
    int seg = 0, left = k1 - k0;   // of the next stage to be sent for
    auto seek = [&]() {
#pragma unroll
      for (int q = 0; q < NA; ++q) fa[q].seek(s.a[seg][q], i0, k0);
#pragma unroll
      for (int b = 0; b < NB; ++b) fb[b].seek(s.b[seg][b], j0, k0);
    };
    seek();
    auto next = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < NA; ++q) fa[q].next(left);
#pragma unroll
      for (int b = 0; b < NB; ++b) fb[b].next(left);
      left -= BK;
      if (left <= 0 && ++seg < s.n) {
        left = k1 - k0;
        seek();
      }
    };
    auto load = [&](auto uc, int slot) __attribute__((always_inline)) {   // load u of its LPS
      constexpr int u = decltype(uc)::value;
      const unsigned d = lds + slot * SLOT;
      if constexpr (u < NA * FA::LOADS) {
        constexpr int q = u / FA::LOADS;
        fa[q].template load<u % FA::LOADS>(d + q * FA::BYTES);
      } else {
        constexpr int v = u - NA * FA::LOADS, b = v / FB::LOADS;
        fb[b].template load<v % FB::LOADS>(d + NA * FA::BYTES + b * FB::BYTES);
      }
    };
    int pa[MT], pb[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) pa[i] = FA::place((wm * MT + i) * 32);
#pragma unroll
    for (int j = 0; j < NT; ++j) pb[j] = NA * FA::BYTES + FB::place((wn * NT + j) * 32);
#pragma unroll
    for (int k = 0; k < NS; ++k)
      if (k < total) {
        next();
        each<LPS>([&](auto u) { load(u, k); });
      }
    // the fragments of the stage to be multiplied
    constexpr int H = BK / 16;
    u32x4 a[H][NA][MT], b[H][NB][NT];
    auto read = [&](int h, const unsigned char* st) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < NA; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i) a[h][q][i] = FA::frag(st + q * FA::BYTES, pa[i], h);
#pragma unroll
      for (int q = 0; q < NB; ++q)
#pragma unroll
        for (int j = 0; j < NT; ++j) b[h][q][j] = FB::frag(st + q * FB::BYTES, pb[j], h);
    };
    wait_stages<NS + 1, LPS>(min(NS - 1, total - 1));
    ring_barrier();
#pragma unroll
    for (int h = 0; h < H; ++h) read(h, ring);
    int slot = 0, pair = 0, more = per;
    // A turn multiplies a stage and, between its products, reads the next one's fragments
    // in their place and sends the loads of the stage NS ahead: at its barrier the next
    // stage has landed, and every wave has this one's fragments, so that its slot is free.
    // (Reads and loads before the products: a wave waits for LDS, and for its loads to be
    // taken, a KiB in 19 clocks; 12544 x 256 through 1024 hidden channels 58 us and 33.)
    for (int idx = 0; idx < total; ++idx) {
      wait_stages<NS, LPS>(max(0, min(NS - 2, total - 2 - idx)));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      ring_barrier();
      const int nslot = slot + 1 == NS ? 0 : slot + 1;
      const bool send = idx + NS < total;
      if (send) next();
      each<H>([&](auto hc) {
        constexpr int h = decltype(hc)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < NB; ++q)
#pragma unroll
          for (int r = NA - 1; r >= 0; --r)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
              for (int j = 0; j < NT; ++j)
                acc[q][i][j] = mfma32(as_bf16x8(b[h][q][j]), as_bf16x8(a[h][r][i]), acc[q][i][j]);
#pragma unroll
        for (int i = 0; i < MT; ++i) extra(a[h][0][i], i, pair);
        read(h, ring + nslot * SLOT);
        if (send) each<(h + 1) * LPS / H - h * LPS / H>([&](auto u) {
          load(std::integral_constant<int, h * LPS / H + decltype(u)::value>(), slot);
        });
      });
      __builtin_amdgcn_sched_barrier(0);
      if (--more == 0) {
        more = per;
        ++pair;
      }
      slot = nslot;
    }
  }
};

// The rows and columns of tile t of tm x tn: groups of eight rows of tiles, column
// by column, so that the tiles in flight on one XCD share their operands.
__device__ __forceinline__ void tile_of(int t, int tm, int tn, int* i, int* j) {
  const int per = 8 * tn, g = t / per, rows = min(8, tm - 8 * g), r = t - g * per;
  *i = 8 * g + r % rows;
  *j = r / rows;
}

// Eight consecutive columns of a fragment's lane as one 16-byte chunk: lanes l
// and l + 32 hold columns 8 g + 0..3 and 8 g + 4..7; swapping the halves of groups
// 2 h and 2 h + 1 leaves each lane one whole group, 2 h + l / 32.  Calls put(h,
// chunk) for h = 0, 1; the chunk starts at column 16 h + 8 (l / 32).
template <typename F>
__device__ __forceinline__ void put8(const unsigned (&pk)[8], F put) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto s0 = __builtin_amdgcn_permlane32_swap(pk[4 * h], pk[4 * h + 2], false, false);
    const auto s1 = __builtin_amdgcn_permlane32_swap(pk[4 * h + 1], pk[4 * h + 3], false, false);
    put(h, u32x4{s0[0], s1[0], s0[1], s1[1]});
  }
}

}  // namespace
}  // namespace tgpk
