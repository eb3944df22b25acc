// Host-side driver of the sequence-core entry points for sanitizer builds:
// every call here fails validation or takes a documented no-op path, and the
// size queries run over grids of sizes up to the largest, so no call reaches
// the GPU.  Fake device pointers are never dereferenced: validation rejects the
// call first.  Exit status 0 when every expectation holds.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

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
static const int64_t kBig = (int64_t)1 << 60;

static void sizes() {
  const int64_t ns[] = {-1, 0, 1, 63, 4096, 4097, 100000, (int64_t)1 << 30, ((int64_t)1 << 30) + 1, kBig};
  const int32_t vs[] = {-1, 0, 1, 7, 255, 256, 57600, 70001, INT32_MAX};
  const int32_t hs[] = {-3, 0, 1, 3, 8, 367, 1024, 8192, 8193, 65536, 65537, INT32_MAX};
  for (int64_t n : ns)
    for (int32_t V : vs)
      for (int32_t H : hs) {
        const size_t b = wm_embed_grad_workspace_bytes(n, V, H);
        const bool ok = n >= 0 && n <= (int64_t)1 << 30 && V > 0 && H > 0 && H <= 65536;
        EXPECT(ok ? b >= (size_t)n * 16 : b == 0);
      }
  for (int64_t n : ns)
    for (int32_t H : hs) {
      const size_t b = wm_layer_norm_grad_workspace_bytes(n, H);
      const bool ok = n >= 0 && n <= (int64_t)1 << 32 && H > 0 && H <= 8192;
      EXPECT(ok ? b >= (size_t)H * 8 : b == 0);
    }
  const int32_t ts[] = {-1, 0, 1, 2, 16, 17, 128, 129, 1000, 32768, 131072, 131073, 10000000, INT32_MAX};
  const int32_t bs[] = {-1, 0, 1, 7, 4096, INT32_MAX};
  for (int32_t T : ts)
    for (int32_t B : bs)
      for (int32_t H : hs) {
        const size_t s = wm_linrec_states_bytes(T, B, H), w = wm_linrec_workspace_bytes(T, B, H);
        const bool ok = T >= 0 && B >= 0 && H > 0 && (int64_t)T * B <= INT32_MAX && (int64_t)B * H <= INT32_MAX;
        if (!ok) EXPECT(s == 0 && w == 0);
        if (ok && T <= 128) EXPECT(w == 0);
        if (ok && T > 0) EXPECT(s >= (size_t)B * H * 4 * ((size_t)T / 16));
      }
  // a workspace for many positions serves few
  size_t last = 0;
  for (int64_t n = 1; n < 600000; n += n < 5000 ? 1 : 997) {
    const size_t b = wm_embed_grad_workspace_bytes(n, 300, 700);
    EXPECT(b >= last);
    last = b;
  }
}

static void embed() {
  auto fwd = [](int dt, int64_t n, int V, int H, const int32_t* tok, const void* tab, void* out, int64_t ld) {
    return wm_embed(dt, n, V, H, tok, tab, 1.0f, out, ld, nullptr);
  };
  EXPECT(fwd(2, 4, 5, 8, I, P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(-1, 4, 5, 8, I, P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, -1, 5, 8, I, P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 0, 8, I, P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 0, I, P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 65537, I, P, P, 65537) == WM_ERR_UNSUPPORTED);
  EXPECT(fwd(WM_FP32, kBig, 5, 8, I, P, P, 8) == WM_ERR_UNSUPPORTED);
  EXPECT(fwd(WM_FP32, 4, 5, 8, I, P, P, 7) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 8, I, P, P, kBig) == WM_ERR_UNSUPPORTED);
  EXPECT(fwd(WM_FP32, 4, 5, 8, nullptr, P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 8, I, nullptr, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 8, I, P, nullptr, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 8, I, fake<void>(4098), P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_BF16, 4, 5, 8, I, P, fake<void>(4097), 8) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 5, 8, fake<int32_t>(4098), P, P, 8) == WM_ERR_INVALID_ARG);
  EXPECT(std::strlen(wm_last_error()) > 0);
  EXPECT(fwd(WM_FP32, 0, 5, 8, nullptr, nullptr, nullptr, 8) == WM_OK);
  EXPECT(std::strlen(wm_last_error()) == 0);
  auto grad = [](int dt, int64_t n, const int32_t* tok, const void* d, int64_t ld, float* g, void* ws, size_t b) {
    return wm_embed_grad(dt, n, 5, 8, tok, d, ld, 1.0f, g, ws, b, nullptr);
  };
  const size_t need = wm_embed_grad_workspace_bytes(100, 5, 8);
  EXPECT(grad(WM_FP32, 100, I, P, 8, F, P, need - 1) == WM_ERR_WORKSPACE);
  EXPECT(grad(WM_FP32, 100, I, P, 8, F, nullptr, need) == WM_ERR_WORKSPACE);
  EXPECT(grad(WM_FP32, 100, I, P, 8, F, fake<void>(4100), need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(WM_FP32, 100, nullptr, P, 8, F, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(WM_FP32, 100, I, P, 8, nullptr, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(WM_BF16, 100, I, fake<void>(4097), 8, F, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(WM_FP32, 100, I, P, 4, F, P, need) == WM_ERR_INVALID_ARG);
}

static void norm() {
  auto fwd = [](int dt, int64_t rows, int H, const void* x, int64_t xl, float eps, void* y, int64_t yl, float* m, float* r) {
    return wm_layer_norm(dt, rows, H, x, xl, F, F, eps, y, yl, m, r, nullptr);
  };
  EXPECT(fwd(7, 4, 8, P, 8, 1e-5f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, -4, 8, P, 8, 1e-5f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 0, P, 8, 1e-5f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8193, P, 8193, 1e-5f, P, 8193, F, F) == WM_ERR_UNSUPPORTED);
  EXPECT(fwd(WM_FP32, kBig, 8, P, 8, 1e-5f, P, 8, F, F) == WM_ERR_UNSUPPORTED);
  EXPECT(fwd(WM_FP32, 4, 8, P, 7, 1e-5f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, P, 8, 1e-5f, P, 7, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, P, 8, -1.0f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, P, 8, NAN, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, P, 8, INFINITY, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, P, 8, 1e-5f, P, 8, F, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, nullptr, 8, 1e-5f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, P, 8, 1e-5f, nullptr, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 4, 8, fake<void>(4097), 8, 1e-5f, P, 8, F, F) == WM_ERR_INVALID_ARG);
  EXPECT(fwd(WM_FP32, 0, 8, nullptr, 8, 1e-5f, nullptr, 8, nullptr, nullptr) == WM_OK);
  auto grad = [](const void* x, const void* dy, const float* m, void* dx, int64_t dl, void* ws, size_t b) {
    return wm_layer_norm_grad(WM_BF16, 40, 9, x, 9, dy, 9, F, m, F, dx, dl, F, F, ws, b, nullptr);
  };
  const size_t need = wm_layer_norm_grad_workspace_bytes(40, 9);
  EXPECT(grad(P, P, F, P, 9, P, need - 1) == WM_ERR_WORKSPACE);
  EXPECT(grad(P, P, F, P, 9, nullptr, need) == WM_ERR_WORKSPACE);
  EXPECT(grad(nullptr, P, F, P, 9, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, nullptr, F, P, 9, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, P, nullptr, P, 9, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, P, F, nullptr, 9, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, P, F, P, 8, P, need) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, P, F, P, 9, fake<void>(4104), need) == WM_ERR_INVALID_ARG);
}

static void linrec() {
  struct Call {
    int dt = WM_FP32, T = 300, B = 4, H = 6;
    const void *x = P, *g = P;
    int64_t xt = 24, xb = 6, gt = 24, gb = 6;
    const float* h0 = F;
    void* y = P;
    float* hT = F;
    void* st = P;
    size_t stb = (size_t)1 << 40;
    void* ws = P;
    size_t wsb = (size_t)1 << 40;
    wm_status run() const {
      return wm_linrec(dt, T, B, H, x, xt, xb, g, gt, gb, h0, U, I, y, hT, st, stb, ws, wsb, nullptr);
    }
  };
  auto bad = [](wm_status want, auto change) {
    Call c;
    change(c);
    EXPECT(c.run() == want);
  };
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.dt = 3; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.T = -1; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.B = -1; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.H = 0; });
  bad(WM_ERR_UNSUPPORTED, [](Call& c) { c.T = c.B = 1 << 16; });
  bad(WM_ERR_UNSUPPORTED, [](Call& c) { c.H = 1 << 30; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.x = nullptr; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.g = nullptr; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.y = nullptr; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.x = fake<void>(4098); });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.dt = WM_BF16, c.g = fake<void>(4097); });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.xt = -1; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.gb = -1; });
  bad(WM_ERR_UNSUPPORTED, [](Call& c) { c.xt = kBig; });
  bad(WM_ERR_UNSUPPORTED, [](Call& c) { c.gb = kBig; });
  bad(WM_ERR_UNSUPPORTED, [](Call& c) { c.xb = (int64_t)1 << 40; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.h0 = fake<float>(4097); });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.hT = fake<float>(4098); });
  bad(WM_ERR_WORKSPACE, [](Call& c) { c.stb = wm_linrec_states_bytes(c.T, c.B, c.H) - 1; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.st = fake<void>(4100); });
  bad(WM_ERR_WORKSPACE, [](Call& c) { c.wsb = wm_linrec_workspace_bytes(c.T, c.B, c.H) - 1; });
  bad(WM_ERR_WORKSPACE, [](Call& c) { c.ws = nullptr; });
  bad(WM_ERR_INVALID_ARG, [](Call& c) { c.ws = fake<void>(4128); });
  bad(WM_OK, [](Call& c) { c.B = 0, c.x = c.g = nullptr, c.y = nullptr, c.ws = nullptr; });
  // the gradient: output rows that overlap
  auto grad = [](void* dx, int64_t dt, int64_t db, const void* st, size_t stb, float* dh0 = nullptr) {
    return wm_linrec_grad(WM_FP32, 5, 4, 6, P, 24, 6, P, 24, 6, nullptr, nullptr, P, 0, 0, nullptr, st, stb, dx, dt, db, P,
                          24, 6, dh0, nullptr, 0, nullptr);
  };
  const size_t stb = wm_linrec_states_bytes(5, 4, 6);
  EXPECT(grad(nullptr, 24, 6, P, stb) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, 23, 6, P, stb) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, 24, 5, P, stb) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, 6, 29, P, stb) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, 0, 6, P, stb) == WM_ERR_INVALID_ARG);
  EXPECT(grad(P, 24, 6, nullptr, stb) == WM_ERR_WORKSPACE);
  EXPECT(grad(P, 24, 6, P, stb - 1) == WM_ERR_WORKSPACE);
  EXPECT(grad(P, 6, 30, P, stb - 1) == WM_ERR_WORKSPACE);  // (batch-major rows pass the check before)
  EXPECT(grad(P, 24, 6, P, stb, fake<float>(4098)) == WM_ERR_INVALID_ARG);
}

static void clip() {
  wm_grad_tensor t[3] = {{P, P, 100, WM_FP32}, {nullptr, nullptr, 0, WM_BF16}, {P, P, 7, WM_BF16}};
  const size_t need = wm_clip_grads_workspace_bytes(3, t);
  EXPECT(need > 0);
  EXPECT(wm_clip_grads_workspace_bytes(-1, t) == 0 && wm_clip_grads_workspace_bytes(3, nullptr) == 0);
  EXPECT(wm_clip_grads_workspace_bytes(0, nullptr) == 0);
  EXPECT(wm_clip_grads(-1, t, 1.0f, F, P, need, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_clip_grads(3, nullptr, 1.0f, F, P, need, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_clip_grads(3, t, -1.0f, F, P, need, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_clip_grads(3, t, NAN, F, P, need, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_clip_grads(3, t, INFINITY, F, P, need, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_clip_grads(3, t, 1.0f, nullptr, P, need, nullptr) == WM_ERR_INVALID_ARG);
  EXPECT(wm_clip_grads(3, t, 1.0f, F, P, need - 1, nullptr) == WM_ERR_WORKSPACE);
  EXPECT(wm_clip_grads(3, t, 1.0f, F, fake<void>(4104), need, nullptr) == WM_ERR_INVALID_ARG);
  for (int k = 0; k < 5; ++k) {
    wm_grad_tensor b[3] = {t[0], t[1], t[2]};
    if (k == 0) b[2].grad = nullptr;
    if (k == 1) b[2].out = nullptr;
    if (k == 2) b[0].grad = fake<void>(4098);
    if (k == 3) b[1].n = -1;
    if (k == 4) b[0].dtype = 9;
    EXPECT(wm_clip_grads(3, b, 1.0f, F, P, need, nullptr) == WM_ERR_INVALID_ARG);
  }
  t[0].n = (int64_t)1 << 43;
  EXPECT(wm_clip_grads(3, t, 1.0f, F, P, need, nullptr) == WM_ERR_UNSUPPORTED);
  // hundreds of tensors, the largest lists
  static wm_grad_tensor many[1000];
  for (int i = 0; i < 1000; ++i) many[i] = {P, P, i % 7 ? i * 1000003L : 0, i % 2};
  EXPECT(wm_clip_grads_workspace_bytes(1000, many) > 0);
  for (int i = 0; i < 1000; ++i) many[i].n = (int64_t)1 << 32;
  EXPECT(wm_clip_grads_workspace_bytes(1000, many) > 0);
  for (int i = 0; i < 1000; ++i) many[i].n = kBig;
  EXPECT(wm_clip_grads_workspace_bytes(1000, many) == 0);
}

int main() {
  sizes();
  embed();
  norm();
  linrec();
  clip();
  std::printf("sequence driver: %d failures\n", g_failures);
  return g_failures ? 1 : 0;
}
