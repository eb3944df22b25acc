// Maps of the gated linear recurrence and their composition along a chain of
// segments (wm_linrec.hip); plain arithmetic, on the device and the host alike.
//
// A run of steps is an affine map of the state that enters it, h -> U + A h.
// A map whose run holds a reset does not depend on the state at all: A = -1
// says so (a true A is never negative), because 0 * inf would not.
#pragma once

#include <hip/hip_runtime.h>

namespace wm {

struct Map {
  float A, U;
};
__host__ __device__ __forceinline__ float apply(Map m, float h) {
  const float u = fmaf(m.A, h, m.U);
  return m.A < 0.0f ? m.U : u;
}
// A product of two gates or of their products.  One that leaves fp32's range is
// held at its least positive number, so that an infinite state stays infinite
// however the steps are cut into maps (0 * inf is NaN); that moves a finite h by
// at most 1.4e-45 |h|, the spacing of products there.  A gate that is 0 itself
// (-inf) keeps its product 0.
__host__ __device__ __forceinline__ float both(float a, float b) {
  const int x = __builtin_bit_cast(int, a), y = __builtin_bit_cast(int, b), p = __builtin_bit_cast(int, a * b);
  const int least = x < y ? (x < 1 ? x : 1) : (y < 1 ? y : 1);  // (positive floats lie in the order of their bits)
  return __builtin_bit_cast(float, p > least ? p : least);
}
// ... where neither is 0.
__host__ __device__ __forceinline__ float both_positive(float a, float b) {
  const int p = __builtin_bit_cast(int, a * b);
  return __builtin_bit_cast(float, p > 1 ? p : 1);
}
// first m, then n
__host__ __device__ __forceinline__ Map then(Map m, Map n) {
  const float a = both(n.A, m.A);
  return {n.A < 0.0f || m.A < 0.0f ? -1.0f : a, apply(n, m.U)};
}

// Segments whose maps are composed into one for the segments after them.
// Measured, 32768 steps of 1024 channels in bf16, both directions: 4 157 us, 8
// 154, 16 162.
constexpr int kFan = 8;

// Composes the maps of segments [s, s1), in order.  A whole fan (s is one's
// first) comes from the fan's map if that is there; if not, its segments' maps,
// which are published earlier, are composed in the order of the fan's own, from
// the identity: the bits do not depend on which of the two came in time.
//   fan(s, f)          whether the map of the fan from segment s on is there (f)
//   members(s, e, f)   calls f with the maps of segments [s, e), in order
template <typename Fan, typename Members>
__host__ __device__ __forceinline__ Map compose(int s, int s1, Fan fan, Members members) {
  Map m{1.0f, 0.0f};
#pragma unroll 1
  while (s < s1) {
    const int e = s1 - s < kFan ? s1 : s + kFan;
    const bool whole = e - s == kFan;
    Map f{1.0f, 0.0f};
    if (!whole) f = m;
    if (!whole || !fan(s, f)) members(s, e, [&](Map n) { f = then(f, n); });
    m = whole ? then(m, f) : f;
    s = e;
  }
  return m;
}

}  // namespace wm
