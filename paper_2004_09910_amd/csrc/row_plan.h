// How a launch of the residual norms holds a row in registers.  Host code alone,
// so that a test can go through every width.
#pragma once
#include <algorithm>
#include <cstdint>

namespace tgpk {

constexpr int kRowThreads = 256;                   // lanes of a row that is a block's
constexpr int kFwdValues = 32, kBwdValues = 16;    // of a row, a lane, at most
// Accesses of a lane, at most: kernels are there for 1, 2, 3, 4, 8 and 16.  (Forward, rows
// of more than 4096 channels read a value at a time go through LDS for it.)
constexpr int kMostVectors = 16;
constexpr int fwd_widest(int) { return 16; }       // bytes of the widest access
constexpr int bwd_widest(int esz) { return 4 * esz; }

// vb bytes an access, nv of them a lane, g lanes a row (0: the block); vb = 0: not in
// registers at all.
struct RowPlan {
  int vb, nv, g;
};

// The widest accesses that every row's start and length allow, at most `most` values a
// lane; then the lanes that leave fewest idle, more lanes where two leave the same.
// near: a wave's rows are within 32 bits of each other; else it takes one at a time.
inline RowPlan row_plan(int esz, int C, uintptr_t bits, int most, int widest, bool near) {
  bits |= (uintptr_t)C * esz;
  const int vb = bits % widest == 0 ? widest : bits % 4 == 0 ? 4 : 2, nvec = C * esz / vb, top = most * esz / vb;
  RowPlan best{vb, 0, 64};
  int room = 1 << 30;
  for (int g = 64; g >= (near ? 1 : 64); g >>= 1) {
    const int nv = (nvec + g - 1) / g;
    if (nv > std::min(4, top)) break;
    if (nv * g < room) room = nv * g, best = {vb, nv, g};
  }
  if (best.nv) return best;
  const int nv = (nvec + kRowThreads - 1) / kRowThreads;
  if (nv > std::min(kMostVectors, top)) return {0, 0, 0};
  return {vb, nv <= 4 ? nv : nv <= 8 ? 8 : 16, 0};
}

}  // namespace tgpk
