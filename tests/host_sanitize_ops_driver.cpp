// Host-side driver of the training operators for an AddressSanitizer / UBSan
// build: workspace sizes and refusals, and the launchers' own host code (lists
// of matrices dealt over launches, workspaces laid out) with every launch
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

static void* const FAKE = (void*)(uintptr_t)(1u << 20);   // never dereferenced

int main() {
  std::mt19937 rng(1);
  auto upto = [&](int most) { return 1 + (int)(rng() % (unsigned)most); };
  // ---- lists of every length, of matrices that one block takes whole, of
  // those in tiles, of one and two steps at a time, and mixed
  for (int count : {0, 1, 2, 19, 20, 21, 40, 41, 100}) {
    for (int kind = 0; kind < 5; ++kind) {
      std::vector<tgp_muon_tensor> t((size_t)count);
      for (auto& m : t) {
        const int k = kind == 4 ? (int)(rng() % 4) : kind;
        m.rows = k == 0 ? upto(64) : k == 1 ? 65 + upto(900) : k == 2 ? upto(256) : upto(3);
        m.cols = k == 0 ? upto(256) : k == 1 ? 65 + upto(900) : k == 2 ? 1024 + upto(8000) : 20000 + upto(9);
        if (rng() & 1) std::swap(m.rows, m.cols);
        m.grad = (const float*)FAKE;
        m.momentum = rng() & 1 ? (float*)FAKE : nullptr;
        m.update = FAKE;
      }
      size_t bytes = 0;
      EXPECT(tgp_muon_workspace(count, t.data(), &bytes) == TGP_OK);
      EXPECT((count == 0) == (bytes == 0));
      for (int steps : {1, 2, 5}) {
        tgp_debug_fail_launch(1);
        const tgp_status got = tgp_muon_update(count, t.data(), 0.95f, 1, steps, 1e-7f, FAKE, bytes, nullptr);
        tgp_debug_fail_launch(0);
        EXPECT(got == (count ? TGP_EHIP : TGP_OK));
      }
      if (bytes) EXPECT(tgp_muon_update(count, t.data(), 0.95f, 1, 5, 1e-7f, FAKE, bytes - 1, nullptr) == TGP_ENOSPACE);
      if (count) {
        t[(size_t)count / 2].rows = 1 << 20;
        t[(size_t)count / 2].cols = 1 << 20;
        EXPECT(tgp_muon_workspace(count, t.data(), &bytes) == TGP_EUNSUPPORTED);
        t[(size_t)count / 2].cols = 0;
        EXPECT(tgp_muon_workspace(count, t.data(), &bytes) == TGP_EINVAL);
      }
    }
  }
  // ---- layer norm: plans of every width, alignment and number of rows
  for (int dt : {TGP_BF16, TGP_FP32})
    for (int64_t rows : {0, 1, 63, 1024, 1025, 300000})
      for (int C : {1, 2, 7, 64, 100, 513, 1024, 2049, 4100, 9000, 1 << 20})
        for (int more : {0, 1, 8}) {
          size_t bytes = 0;
          EXPECT(tgp_layer_norm_backward_workspace(rows, C, dt, &bytes) == TGP_OK);
          tgp_debug_fail_launch(1);
          const tgp_status f = tgp_layer_norm_forward(rows, C, dt, FAKE, C + more, (const float*)FAKE, nullptr, 1e-5f,
                                                      FAKE, C + more, (float*)FAKE, nullptr);
          tgp_debug_fail_launch(1);
          const tgp_status b = tgp_layer_norm_backward(rows, C, dt, FAKE, C + more, FAKE, C + more, nullptr,
                                                       (const float*)FAKE, FAKE, C + more, (float*)FAKE, (float*)FAKE,
                                                       1, FAKE, bytes, nullptr);
          tgp_debug_fail_launch(0);
          EXPECT(f == (rows ? TGP_EHIP : TGP_OK));
          EXPECT(b == TGP_EHIP);
        }
  // ---- weight steps: more tensors than a launch takes, empty ones among them
  for (int count : {0, 1, 47, 48, 49, 200}) {
    std::vector<tgp_step_tensor> s((size_t)count);
    std::vector<tgp_adamw_tensor> a((size_t)count);
    int64_t all = 0;
    for (int k = 0; k < count; ++k) {
      const int64_t n = rng() % 3 ? (int64_t)(rng() % 100000) : 0;
      all += n;
      s[k] = {n, (float*)FAKE, rng() & 1 ? FAKE : nullptr, FAKE, 0.1f};
      a[k] = {n, (float*)FAKE, rng() & 1 ? FAKE : nullptr, (const float*)FAKE, (float*)FAKE, (float*)FAKE};
    }
    tgp_debug_fail_launch(1);
    const tgp_status g = tgp_weight_step(count, s.data(), 0.1f, nullptr);
    tgp_debug_fail_launch(1);
    const tgp_status h = tgp_adamw_step(count, a.data(), 1e-3f, 0.9f, 0.99f, 1e-8f, 0.f, 1, nullptr);
    tgp_debug_fail_launch(0);
    EXPECT(g == (all ? TGP_EHIP : TGP_OK) && h == (all ? TGP_EHIP : TGP_OK));
  }
  if (failures) return 1;
  std::printf("host operators: ok\n");
  return 0;
}
