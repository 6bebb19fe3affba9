// Every width of the residual norms against the plan of its registers: with each
// type, direction and alignment, near and far rows.  A plan's vectors have to hold
// the whole row, and a kernel of their number has to exist.  Prints the widths that
// none does and exits 1 if there are any.
#include <cstdio>

#include "row_plan.h"

int main() {
  long bad = 0, held = 0;
  for (int esz : {2, 4})
    for (bool fwd : {true, false})
      for (uintptr_t bits : {(uintptr_t)2, (uintptr_t)4, (uintptr_t)8, (uintptr_t)16})
        for (bool near : {true, false})
          for (int C = 1; C <= 32768; ++C) {
            if (bits < (uintptr_t)esz) continue;   // elements lie at multiples of their size
            const int most = fwd ? tgpk::kFwdValues : tgpk::kBwdValues;
            const int wide = fwd ? tgpk::fwd_widest(esz) : tgpk::bwd_widest(esz);
            const tgpk::RowPlan p = tgpk::row_plan(esz, C, bits, most, wide, near);
            if (p.vb == 0) continue;   // the kernel that keeps a row in LDS
            ++held;
            const int lanes = p.g ? p.g : tgpk::kRowThreads, v = p.vb / esz;
            const bool kernel = p.nv == 1 || p.nv == 2 || p.nv == 3 || p.nv == 4 || (!p.g && (p.nv == 8 || p.nv == 16));
            const bool access = p.vb == wide || p.vb == 4 || (esz == 2 && p.vb == 2);
            const bool at = p.vb % esz == 0 && bits % p.vb == 0 && (long)C * esz % p.vb == 0;
            if (kernel && access && at && (near || !p.g || p.g == 64) && p.nv * v <= most && (long)p.nv * lanes * v >= C) continue;
            if (bad++ < 10)
              std::printf("esz %d %s, bits %d, near %d, C %d: %d bytes, %d of them, %d lanes\n", esz, fwd ? "forward" : "backward",
                          (int)bits, near, C, p.vb, p.nv, lanes);
          }
  std::printf("%ld plans, %ld bad\n", held, bad);
  return bad || held == 0;
}
