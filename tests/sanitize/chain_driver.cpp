// CPU driver of the composition of segment maps (csrc/wm_chain.h): the bits of
// a run's map do not depend on which fans' maps are there when it is composed,
// and the map is that of the steps.  Exit status 0 when every expectation holds.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>

#include "../../paper_2205_01435_amd/csrc/wm_chain.h"

using wm::kFan;
using wm::Map;

static int g_failures = 0;

static void expect(bool ok, const char* what, double mean, int s, int s1) {
  if (ok) return;
  if (++g_failures <= 5) std::fprintf(stderr, "%s: gates around %g, segments %d to %d\n", what, mean, s, s1);
}

struct Chain {
  std::vector<Map> seg, fan;
  // steps of 128 a segment; in 64 bits too
  std::vector<double> A, U;
  Chain(int segs, double mean, std::mt19937& rng) {
    std::normal_distribution<double> normal;
    for (int k = 0; k < segs; ++k) {
      Map m{1.0f, 0.0f};
      double A1 = 1.0, U1 = 0.0;
      for (int t = 0; t < 128; ++t) {
        const float g = (float)(mean + normal(rng)), x = (float)normal(rng);
        const float a = (float)(1.0 / (1.0 + std::exp(-(double)g))), b = (float)(1.0 / (1.0 + std::exp((double)g)));
        m = wm::then(m, {a, b * x});
        A1 *= a;
        U1 = a * U1 + (double)b * x;
      }
      seg.push_back(m);
      A.push_back(A1);
      U.push_back(U1);
    }
    // as a segment that ends a fan publishes it: the seven before it composed, then its own
    for (int k = 0; k + kFan <= segs; k += kFan)
      fan.push_back(wm::then(run(k, k + kFan - 1, [](int) { return false; }), seg[k + kFan - 1]));
  }
  template <typename There>
  Map run(int s, int s1, There there) const {
    return wm::compose(
        s, s1,
        [&](int i, Map& f) {
          if (!there(i / kFan)) return false;
          f = fan[i / kFan];
          return true;
        },
        [&](int i, int e, auto take) {
          for (; i < e; ++i) take(seg[i]);
        });
  }
};

static bool same(Map a, Map b) { return std::memcmp(&a, &b, sizeof a) == 0; }

int main() {
  std::mt19937 rng(1);
  for (double mean : {-8.0, 0.0, 2.0, 5.0, 7.0, 9.0})
    for (int n = 0; n < 40; ++n) {
      const Chain c(66, mean, rng);
      for (int s = 0; s < 66; s += kFan)
        for (int s1 : {s + 1, s + 7, s + 8, s + 17, s + 24, 65}) {
          if (s1 > 65 || s1 <= s) continue;
          const Map all = c.run(s, s1, [](int) { return true; }), none = c.run(s, s1, [](int) { return false; });
          expect(same(all, none), "all fans there or none", mean, s, s1);
          for (int k = 0; k < 4; ++k)
            expect(same(all, c.run(s, s1, [&](int) { return rng() % 2 == 0; })), "some fans there", mean, s, s1);
          double A = 1.0, U = 0.0;
          for (int i = s; i < s1; ++i) {
            A *= c.A[i];
            U = c.A[i] * U + c.U[i];
          }
          // each of a segment's steps and each composition adds at most 3 roundings of magnitudes below 5
          const double u = std::ldexp(1.0, -24), ops = 3.0 * (128 + 1) * (s1 - s);
          expect(std::fabs(all.A - A) <= ops * u * A + std::ldexp(1.0, -126), "A", mean, s, s1);
          expect(std::fabs(all.U - U) <= ops * u * 5.0, "U", mean, s, s1);
        }
    }
  std::printf("chain driver: %d failures\n", g_failures);
  return g_failures ? 1 : 0;
}
