// Host-side driver of the attending-core entry points for sanitizer builds:
// every call here fails validation or takes a documented no-op path, the size
// queries run over grids of sizes up to the largest, and the rotation's table is
// a host function, so no call reaches the GPU.  Fake device pointers are never
// dereferenced: validation rejects the call first.  Exit status 0 when every
// expectation holds.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>

#include "wm.h"

static int g_failures = 0;

#define EXPECT(cond)                                                               \
  do {                                                                             \
    if (!(cond)) {                                                                 \
      std::fprintf(stderr, "%s:%d: expectation failed: %s\n", __FILE__, __LINE__, #cond); \
      ++g_failures;                                                                \
    }                                                                              \
  } while (0)

template <typename T>
static T* fake(uintptr_t a) { return reinterpret_cast<T*>(a); }

static void* const P = fake<void>(4096);
static float* const F = fake<float>(4096);
static int32_t* const I = fake<int32_t>(4096);
static uint8_t* const U = fake<uint8_t>(4096);
static uint64_t* const TB = fake<uint64_t>(4096);
static const int64_t kBig = (int64_t)1 << 60;

static void sizes() {
  const int64_t ns[] = {-1, 0, 1, 63, 4097, 200000, INT32_MAX, (int64_t)1 << 32, kBig};
  const int32_t hs[] = {-1, 0, 1, 3, 16, 1024, 1025, INT32_MAX};
  const int32_t ds[] = {-3, 0, 1, 2, 37, 64, 128, 129, 256, 257, 65536, 65537, INT32_MAX};
  for (int64_t n : ns)
    for (int32_t hq : hs)
      for (int32_t hk : hs)
        for (int32_t D : ds) {
          const size_t b = wm_qk_norm_grad_workspace_bytes(n, hq, hk, D);
          const bool ok = n >= 0 && hq > 0 && hq <= 1024 && hk >= 0 && hk <= 1024 && D > 0 && D <= 256 &&
                          n <= INT32_MAX / (hq + hk);
          EXPECT(ok ? b >= (size_t)D * 8 : b == 0);
        }
  const int32_t ts[] = {-1, 0, 1, 63, 64, 65, 255, 256, 257, 32768, 1000003, INT32_MAX};
  const int32_t bs[] = {-1, 0, 1, 7, 512, 4096, INT32_MAX};
  for (int32_t T : ts)
    for (int32_t B : bs)
      for (int32_t N : hs)
        for (int32_t K : ds)
          for (int32_t V : ds) {
            const size_t f = wm_linattn_workspace_bytes(T, B, N, K, V), g = wm_linattn_states_bytes(T, B, N, K, V);
            const bool in = T >= 0 && B >= 0 && N > 0 && K > 0 && K <= 128 && V > 0 && V <= 128;
            const __int128 most = INT32_MAX, w = K > V ? K : V;
            const bool ok = in && (__int128)B * N <= 1 << 22 && (__int128)T * B <= most && (__int128)B * N * K * V <= most && (__int128)T * B * N * w <= most;
            if (!ok) EXPECT(f == 0 && g == 0);
            if (ok && T < 128) EXPECT(f == 0);
            EXPECT(f <= (size_t)1 << 40 && g <= (size_t)1 << 40);
          }
  for (int64_t n : ns)
    for (int32_t D : ds)
      for (int32_t G : ds)
        for (int dt = -1; dt < 3; ++dt) {
          const size_t b = wm_glu_grad_workspace_bytes(dt, n, D, G);
          const bool ok = (dt == 0 || dt == 1) && n >= 0 && n <= 1 << 30 && D > 0 && D <= 65536 && G > 0 && G <= 65536 &&
                          n <= ((int64_t)1 << 35) / (D > G ? D : G);
          const size_t v = wm_glu_saved_bytes(dt, n, D, G);
          EXPECT(ok ? b >= (size_t)n * 2 * G * (dt == 0 ? 4 : 2) : b == 0);
          EXPECT(ok ? v >= (size_t)n * 2 * G * (dt == 0 ? 4 : 3) : v == 0);
        }
}

static void table() {
  std::vector<uint64_t> t(128);
  EXPECT(wm_rotary_table(256, 10000.0, t.data()) == WM_OK);
  // 1 / (2 pi) of a turn, and falling
  EXPECT(std::fabs((double)t[0] / 18446744073709551616.0 - 0.15915494309189535) < 1e-16);
  for (int i = 1; i < 128; ++i) EXPECT(t[i] < t[i - 1]);
  EXPECT(wm_rotary_table(0, 10000.0, nullptr) == WM_OK);
  EXPECT(wm_rotary_table(8, 1.0, t.data()) == WM_OK && t[3] == t[0]);
  EXPECT(wm_rotary_table(8, 1e300, t.data()) == WM_OK);
  EXPECT(wm_rotary_table(8, 10000.0, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_rotary_table(7, 10000.0, t.data()) == WM_ERR_INVALID_ARG);
  EXPECT(wm_rotary_table(-2, 10000.0, t.data()) == WM_ERR_INVALID_ARG);
  EXPECT(wm_rotary_table(258, 10000.0, t.data()) == WM_ERR_INVALID_ARG);
  EXPECT(wm_rotary_table(8, 0.5, t.data()) == WM_ERR_INVALID_ARG);
  EXPECT(wm_rotary_table(8, NAN, t.data()) == WM_ERR_INVALID_ARG);
  EXPECT(wm_rotary_table(8, INFINITY, t.data()) == WM_ERR_INVALID_ARG);
}

static void qk() {
  struct A {
    int dt = WM_FP32;
    int64_t rows = 4;
    int Hq = 2, Hk = 1, D = 8, R = 8, nb = 0;
    const void *q = P, *k = P;
    int64_t ql = 16, kl = 8;
    float eps = 1e-6f;
    const int32_t* pos = I;
    const uint64_t* tab = TB;
    void *qo = P, *ko = P;
    int64_t qol = 16, kol = 8;
    wm_status operator()() const {
      return wm_qk_norm(dt, rows, Hq, Hk, D, R, nb, q, ql, k, kl, F, F, eps, pos, tab, qo, qol, ko, kol, nullptr);
    }
  };
  auto bad = [](auto set, wm_status want) {
    A a;
    set(a);
    EXPECT(a() == want);
  };
  bad([](A& a) { a.dt = 2; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.rows = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.Hq = 0; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.Hk = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.Hq = 1025; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.D = 257; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.rows = kBig; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.R = 9; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.R = 10; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.R = -2; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.nb = 2; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.eps = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.eps = NAN; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.ql = 15; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.kl = 7; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.qol = 15; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.kol = 7; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.ql = kBig; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.q = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.k = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.pos = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.tab = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.qo = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.q = fake<void>(4098); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.dt = WM_BF16, a.ko = fake<void>(4097); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.tab = fake<uint64_t>(4100); }, WM_ERR_INVALID_ARG);
  EXPECT(std::strlen(wm_last_error()) > 0);
  bad([](A& a) { a.rows = 0, a.q = a.k = nullptr, a.pos = nullptr; }, WM_OK);
  EXPECT(std::strlen(wm_last_error()) == 0);
  auto grad = [](const void* q, const void* dq, int64_t ld, void* out, void* ws, size_t b) {
    return wm_qk_norm_grad(WM_BF16, 40, 2, 1, 8, 8, 1, q, 16, P, 8, F, F, 1e-6f, I, TB, dq, ld, P, 8, out, 16, P, 8, F, F, ws, b,
                           nullptr);
  };
  const size_t need = wm_qk_norm_grad_workspace_bytes(40, 2, 1, 8);
  EXPECT(grad(P, P, 16, P, P, need - 1) == WM_ERR_WORKSPACE);
  EXPECT(grad(P, P, 16, P, nullptr, need) == WM_ERR_WORKSPACE);
  EXPECT(grad(P, P, 16, P, fake<void>(4100), need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(nullptr, P, 16, P, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, nullptr, 16, P, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, P, 15, P, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, P, 16, fake<void>(4097), P, need) == WM_ERR_INVALID_ARG);
}

static void attn() {
  struct A {
    int dt = WM_FP32, T = 600, B = 2, N = 2, K = 8, V = 4;
    const void *q = P, *k = P, *v = P;
    int64_t qt = 32, qb = 16, vt = 16, vb = 8, ot = 32, ob = 16;
    const float* decay = F;
    float scale = 1.0f;
    const float* h0 = F;
    const int32_t* len = I;
    void* y = P;
    float* hT = F;
    void *ws = P, *st = P;
    size_t less = 0, sless = 0;
    wm_status fwd() const {
      const size_t b = wm_linattn_workspace_bytes(T, B, N, K, V);
      return wm_linattn(dt, T, B, N, K, V, q, qt, qb, k, 32, 16, v, vt, vb, decay, scale, h0, U, len, y, hT, st, wm_linattn_states_bytes(T, B, N, K, V) - sless, ws,
                        b - less, nullptr);
    }
    wm_status grad() const {
      const size_t b = wm_linattn_workspace_bytes(T, B, N, K, V);
      return wm_linattn_grad(dt, T, B, N, K, V, q, qt, qb, k, 32, 16, v, vt, vb, decay, scale, h0, U, len, P, 16, 8, hT, st,
                             wm_linattn_states_bytes(T, B, N, K, V) - sless, y, ot, ob, P, 32, 16, P, 16, 8, F, ws, b - less, nullptr);
    }
  };
  EXPECT(wm_linattn_workspace_bytes(600, 2, 2, 8, 4) > 0);
  auto bad = [](auto set, wm_status want, bool both = true) {
    A a;
    set(a);
    EXPECT(a.fwd() == want);
    if (both) EXPECT(a.grad() == want);
  };
  bad([](A& a) { a.dt = 5; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.T = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.B = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.N = 0; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.K = 129; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.V = 129; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.T = INT32_MAX; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.q = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.v = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.y = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.decay = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.q = fake<void>(4098); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.qt = -32; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.vt = kBig; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.scale = NAN; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.h0 = fake<float>(4098); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.hT = fake<float>(4097); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.len = fake<int32_t>(4098); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.ws = nullptr; }, WM_ERR_WORKSPACE);
  bad([](A& a) { a.less = 1; }, WM_ERR_WORKSPACE);
  bad([](A& a) { a.ws = fake<void>(4100); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.sless = 1; }, WM_ERR_WORKSPACE);
  bad([](A& a) { a.st = fake<void>(4100); }, WM_ERR_INVALID_ARG);
  A none;
  none.st = nullptr;
  EXPECT(none.grad() == WM_ERR_WORKSPACE);
  bad([](A& a) { a.B = 0; }, WM_OK);
  A overlap;
  overlap.ot = 31;
  EXPECT(overlap.grad() == WM_ERR_INVALID_ARG);
  overlap.ot = 32, overlap.ob = 15;
  EXPECT(overlap.grad() == WM_ERR_INVALID_ARG);
}

static void glu() {
  struct A {
    int dt = WM_FP32;
    int64_t rows = 4;
    int D = 8, G = 6, act = WM_ACT_SILU;
    const void *x = P, *W = P;
    int64_t xl = 8, hl = 6;
    void* h = P;
    void *ws = P, *saved = P;
    size_t less = 0, sless = 0;
    wm_status fwd() const {
      return wm_glu(dt, rows, D, G, act, x, xl, W, h, hl, saved, wm_glu_saved_bytes(dt, rows, D, G) - sless, nullptr);
    }
    wm_status grad() const {
      const size_t b = wm_glu_grad_workspace_bytes(dt, rows, D, G);
      return wm_glu_grad(dt, rows, D, G, act, x, xl, W, saved, wm_glu_saved_bytes(dt, rows, D, G) - sless, h, hl, P, 8, P, ws,
                         b - less, nullptr);
    }
  };
  auto bad = [](auto set, wm_status want) {
    A a;
    set(a);
    EXPECT(a.fwd() == want);
    EXPECT(a.grad() == want);
  };
  bad([](A& a) { a.dt = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.rows = -1; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.D = 0; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.G = 0; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.act = 2; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.D = 65537, a.xl = 65537; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.G = 65537, a.hl = 65537; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.rows = kBig; }, WM_ERR_UNSUPPORTED);
  bad([](A& a) { a.xl = 7; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.hl = 5; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.x = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.W = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.h = nullptr; }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.x = fake<void>(4098); }, WM_ERR_INVALID_ARG);
  bad([](A& a) { a.dt = WM_BF16, a.W = fake<void>(4097); }, WM_ERR_INVALID_ARG);
  A a;
  a.saved = nullptr;
  EXPECT(a.grad() == WM_ERR_WORKSPACE);
  a.saved = P, a.sless = 1;
  EXPECT(a.fwd() == WM_ERR_WORKSPACE && a.grad() == WM_ERR_WORKSPACE);
  a.sless = 0, a.saved = fake<void>(4100);
  EXPECT(a.fwd() == WM_ERR_INVALID_ARG && a.grad() == WM_ERR_INVALID_ARG);
  a.saved = P, a.less = 1;
  EXPECT(a.grad() == WM_ERR_WORKSPACE);
  a.less = 0, a.ws = fake<void>(4100);
  EXPECT(a.grad() == WM_ERR_INVALID_ARG);
  a.rows = 0, a.x = a.W = nullptr, a.h = nullptr;
  EXPECT(a.fwd() == WM_OK);
}

int main() {
  sizes();
  table();
  qk();
  attn();
  glu();
  std::printf("attending-core driver: %d failures\n", g_failures);
  return g_failures ? 1 : 0;
}
