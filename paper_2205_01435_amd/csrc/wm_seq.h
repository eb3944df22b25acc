// Shared by the sequence-core operators (wm_embed.hip, wm_norm.hip,
// wm_linrec.hip, wm_clip.hip): launch arguments and device helpers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wm_device.h"

namespace wm {

// An output of at least this size goes past the caches: it is half of the
// last-level one, which it would empty of what is read again (the values of a
// gradient list, the input of a norm for its gradient).  A smaller one is left
// there for the next call.  Measured, past the caches against through them: a
// gradient list of 270 MB, summed and scaled, 138 and 164 us; a norm of 256 MB
// and its gradient 231 and 246 us (forward alone 92 and 89); a recurrence of 128
// MB and its gradient 157 and 181 us.
constexpr int64_t kStreamBytes = (int64_t)128 << 20;

struct EmbedArgs {
  long n;
  int V, H;
  const int32_t* tokens;
  const void* table;
  float scale;
  void* out;
  long out_ld;
};
hipError_t launch_embed(int dtype, const EmbedArgs& a, hipStream_t s);

struct EmbedGradArgs {
  long n;
  int V, H;
  const int32_t* tokens;
  const void* dout;
  long dout_ld;
  float scale;
  float* dtable;
  void* ws;
};
size_t embed_grad_workspace(long n, int V, int H);
hipError_t launch_embed_grad(int dtype, const EmbedGradArgs& a, hipStream_t s);

constexpr int kNormMaxH = 8192;
struct NormArgs {
  long rows;
  int H;
  const void* x;
  long x_ld;
  const float *gamma, *beta;
  float eps;
  void* y;
  long y_ld;
  float *mean, *rstd;
};
hipError_t launch_layer_norm(int dtype, const NormArgs& a, hipStream_t s);

struct NormGradArgs {
  long rows;
  int H;
  const void* x;
  long x_ld;
  const void* dy;
  long dy_ld;
  const float *gamma, *mean, *rstd;
  void* dx;
  long dx_ld;
  float *dgamma, *dbeta;
  float* part;  // workspace
};
size_t layer_norm_grad_workspace(long rows, int H);
hipError_t launch_layer_norm_grad(int dtype, const NormGradArgs& a, hipStream_t s);

// A [T, B, H] array: element strides of the steps and the rows, unit stride
// along H.
struct SeqView {
  const void* p;
  long t, b;
};
struct LinrecArgs {
  int T, B, H;
  SeqView x, gate;
  const float* h0;        // [B, H] or null (0)
  const uint8_t* resets;  // [T, B] or null
  const int32_t* lengths; // [B] or null (T)
  void* y;                // [T, B, H]
  float* h_T;             // [B, H] or null
  float* states;          // linrec_states floats or null
  void* ws;
};
struct LinrecGradArgs {
  int T, B, H;
  SeqView x, gate, dy, dx, dgate;  // dx, dgate are written
  const uint8_t* resets;
  const int32_t* lengths;
  const float* dh_T;      // [B, H] or null (0)
  const float* states;
  float* dh0;             // [B, H] or null
  void* ws;
};
size_t linrec_states(int T, int B, int H);     // bytes
size_t linrec_workspace(int T, int B, int H);  // bytes
hipError_t launch_linrec(int dtype, const LinrecArgs& a, hipStream_t s);
hipError_t launch_linrec_grad(int dtype, const LinrecGradArgs& a, hipStream_t s);

size_t clip_workspace(int n, const wm_grad_tensor* t);
hipError_t launch_clip(int n, const wm_grad_tensor* t, float max_norm, float* norm, void* ws, hipStream_t s);

// (sigmoid(g), sigmoid(-g)), each to full relative precision, from e^-|g|:
// 1 / (1 + e) by one Newton step from the hardware's reciprocal, and e times it.
// Only g's sign is looked at, that of a zero too (e itself may carry it).
__device__ __forceinline__ float2 gate_pair_of(float g, float e) {
  const float w = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(w);
  r = fmaf(fmaf(-w, r, 1.0f), r, r);
  const float q = e * r;
  return __float_as_int(g) >= 0 ? make_float2(r, q) : make_float2(q, r);
}

// e^-|g| for |g| <= kGateMost, in half of expf's instructions: with p =
// -|g| log2(e) rounded and d = -|g| - p ln 2 what the rounding left over it is
// 2^p (1 + d).
constexpr float kGateMost = 87.0f;  // e^-87 is still a normal number
__device__ __forceinline__ float gate_exp_small(float g) {
  const float n = fabsf(g);
  const float p = n * -1.44269504088896341f;
  const float d = fmaf(p, -0.693147180559945309f, -n);
  const float t = __builtin_amdgcn_exp2f(p);
  return fmaf(t, d, t);
}

// The same pair for |g| <= kGateMost without looking at the sign, three
// instructions fewer: from e = e^-g, which neither overflows nor leaves 1 / (1 + e)
// below the normal numbers; an error of e counts in each of the two at most once.
__device__ __forceinline__ float2 gate_pair_small(float g) {
  const float p = g * -1.44269504088896341f;
  const float d = fmaf(p, -0.693147180559945309f, -g);
  const float t = __builtin_amdgcn_exp2f(p), e = fmaf(t, d, t), w = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(w);
  r = fmaf(fmaf(-w, r, 1.0f), r, r);
  return make_float2(r, e * r);
}

}  // namespace wm
