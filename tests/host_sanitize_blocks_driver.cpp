// Host-side driver of the gated block, the residual norms and AdamW with 8-bit
// states for an AddressSanitizer / UBSan build: workspace sizes and refusals, and
// the launchers' own host code (plans, parts of pixels, lists) with every launch
// skipped by tgp_debug_fail_launch(1), so that it runs without a GPU.  Exits 0
// when every expectation holds; the sanitizers abort on their own findings.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "tgp.h"

static int failures = 0;
#define EXPECT(cond)                                                                  \
  do {                                                                                \
    if (!(cond)) {                                                                    \
      std::fprintf(stderr, "%s:%d: expectation failed: %s (%s)\n", __FILE__, __LINE__, #cond, \
                   tgp_last_error());                                                 \
      ++failures;                                                                     \
    }                                                                                 \
  } while (0)

// Places far from each other, never dereferenced.
static char* fake(int k, int off = 0) { return (char*)((uintptr_t)(k + 1) << 42) + off; }

int main() {
  std::mt19937 rng(1);
  const int widths[] = {1, 7, 8, 64, 100, 256, 264, 1000, 2056};
  // ---- gated blocks: every width against every other, few and many pixels, at
  // 16-byte places and others, with and without each result
  for (int dt : {TGP_BF16, TGP_FP32})
    for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)64, (int64_t)65, (int64_t)300, (int64_t)20000, (int64_t)3000001})
      for (int ci : widths)
        for (int hi : widths)
          for (int pick = 0; pick < 3; ++pick) {
            const int co = pick ? widths[rng() % 9] : ci, e = dt == TGP_BF16 ? 2 : 4;
            const tgp_gated_shape s{ci, hi, co, dt, (int)(rng() % 2)};
            const int off = pick == 2 ? e : 0;
            const int64_t ldx = ci + (rng() % 2 ? 0 : 8), ldy = co + rng() % 3;
            size_t fw = 0, bw = 0;
            EXPECT(tgp_gated_workspace(&s, rows, 0, &fw) == TGP_OK);
            EXPECT(tgp_gated_workspace(&s, rows, 1, &bw) == TGP_OK);
            const tgp_gated_weights w{fake(0, off), fake(1), fake(2), rng() & 1 ? (float*)fake(3) : nullptr, nullptr, (float*)fake(4)};
            tgp_debug_fail_launch(1);
            const tgp_status f = tgp_gated_forward(&s, rows, &w, fake(5, off), ldx, fake(6), ldy, fake(7), fw, nullptr);
            tgp_debug_fail_launch(0);
            EXPECT(f == (rows ? TGP_EHIP : TGP_OK));
            float* g[6];
            for (int k = 0; k < 6; ++k) g[k] = rng() % 4 ? (float*)fake(8 + k, 4 * (int)(rng() % 2)) : nullptr;
            const tgp_gated_grads gr{g[0], g[1], g[2], g[3], g[4], g[5]};
            const bool any = g[0] || g[1] || g[2] || g[3] || g[4] || g[5];
            const int over = rng() % 2;
            void* dx = rng() % 3 ? fake(14) : nullptr;
            const bool take = rng() % 5;
            tgp_debug_fail_launch(1);
            const tgp_status b = tgp_gated_backward(&s, rows, &w, fake(6), ldy, fake(5, off), ldx, dx, ldx,
                                                    take ? &gr : nullptr, over, fake(7), bw, nullptr);
            tgp_debug_fail_launch(0);
            if (!dx && !(take && any)) EXPECT(b == TGP_EINVAL);
            else if (rows) EXPECT(b == TGP_EHIP);
            else EXPECT(b == TGP_EHIP || b == TGP_OK);
            if (rows && any && bw)
              EXPECT(tgp_gated_backward(&s, rows, &w, fake(6), ldy, fake(5, off), ldx, dx, ldx, &gr, over, fake(7),
                                        bw - 1, nullptr) == TGP_ENOSPACE);
          }
  // ---- residual norms: every plan, and gates of every kind
  for (int dt : {TGP_BF16, TGP_FP32})
    for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)60, (int64_t)6000, (int64_t)2999988})
      for (int C : {1, 2, 7, 12, 64, 100, 513, 1024, 2049, 4100, 9000, 32768})
        for (int64_t group : {(int64_t)0, (int64_t)1, (int64_t)6, rows})
          for (int post : {0, 1}) {
            if (group == 0 && rows == 0) continue;
            const bool gate = group > 0;
            const int64_t ld = C + rng() % 9;
            const tgp_residual_shape s{rows, gate ? (rows % group ? 1 : group) : 0, C, dt, post, 1e-5f};
            const tgp_residual_params p{(float*)fake(0), post ? (float*)fake(1) : nullptr, nullptr, (float*)fake(2), (float*)fake(3)};
            size_t bytes = 0;
            EXPECT(tgp_residual_norm_backward_workspace(&s, &bytes) == TGP_OK);
            tgp_debug_fail_launch(1);
            const tgp_status f = tgp_residual_norm_forward(&s, &p, fake(4), ld, fake(5), ld, gate ? fake(6) : nullptr, ld,
                                                           fake(7), ld, rng() % 2 ? fake(8) : nullptr, ld, (float*)fake(9), nullptr);
            tgp_debug_fail_launch(1);
            const tgp_residual_grads g{(float*)fake(10), nullptr, rng() % 2 && post ? (float*)fake(11) : nullptr, (float*)fake(12), nullptr};
            const tgp_status b = tgp_residual_norm_backward(
                &s, &p, fake(13), ld, rng() % 2 ? fake(14) : nullptr, ld, fake(7), ld, fake(5), ld, gate ? fake(6) : nullptr, ld,
                (float*)fake(9), fake(15), ld, fake(16), ld, gate && rng() % 2 ? fake(17) : nullptr, ld, &g, (int)(rng() % 2),
                fake(18), bytes, nullptr);
            tgp_debug_fail_launch(0);
            EXPECT(f == (rows ? TGP_EHIP : TGP_OK));
            EXPECT(b == TGP_EHIP || (rows == 0 && b == TGP_OK));
          }
  // ---- 8-bit states: more tensors than a launch takes, empty ones, one beyond a launch's blocks
  for (int count : {0, 1, 47, 48, 49, 200}) {
    std::vector<tgp_adamw8_tensor> t((size_t)count);
    int64_t all = 0;
    for (auto& d : t) {
      const int64_t n = rng() % 40 == 0 ? (int64_t)5 << 30 : rng() % 3 ? (int64_t)(rng() % 100000) : 0;
      all += n;
      d = {n, (float*)fake(0), rng() & 1 ? fake(1) : nullptr, (const float*)fake(2), (uint8_t*)fake(3), (uint8_t*)fake(4), (uint8_t*)fake(5)};
    }
    tgp_debug_fail_launch(1);
    const tgp_status g = tgp_adamw8_step(count, t.data(), 1e-3f, 0.9, 0.99, 1e-8f, 0.f, 1, 7, nullptr);
    tgp_debug_fail_launch(0);
    EXPECT(g == (all ? TGP_EHIP : TGP_OK));
  }
  if (failures) return 1;
  std::printf("host operators: ok\n");
  return 0;
}
