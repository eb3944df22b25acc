// Gated linear recurrence over [T, B, H], each channel for itself:
//   a_t = sigmoid(gate_t),  h_t = a_t h_{t-1} + (1 - a_t) x_t,  y_t = h_t,
// where a reset step takes h_{t-1} = 0 and a step past the row's length keeps
// h and puts out 0.  Gradient, with R_t what the later steps add to dh_t:
//   D = dy_t + R_t, dx_t = (1 - a_t) D, dgate_t = a_t (1 - a_t) (h_{t-1} - x_t) D,
//   R_{t-1} = a_t D, or 0 at a reset.
#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kThreads = 256;

// One thread per channel, step by step.
template <typename DT>
__global__ void __launch_bounds__(kThreads) k_linrec(const LinrecArgs a) {
  const long C = (long)a.B * a.H, c = (long)blockIdx.x * kThreads + threadIdx.x;
  if (c >= C) return;
  const int b = (int)(c / a.H), h = (int)(c % a.H);
  const int n = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const DT* x = reinterpret_cast<const DT*>(a.x.p) + b * a.x.b + h;
  const DT* g = reinterpret_cast<const DT*>(a.gate.p) + b * a.gate.b + h;
  DT* y = reinterpret_cast<DT*>(a.y);
  float s = a.h0 ? a.h0[c] : 0.0f;
  for (int t = 0; t < a.T; ++t) {
    const bool live = t < n;
    if (live) {
      if (a.resets && a.resets[(long)t * a.B + b]) s = 0.0f;
      if (a.states) a.states[t * C + c] = s;
      const float2 p = gate_pair(DType<DT>::load(g, t * a.gate.t));
      s = p.x * s + p.y * DType<DT>::load(x, t * a.x.t);
    }
    DType<DT>::store(y, t * C + c, live ? s : 0.0f);
  }
  if (a.h_T) a.h_T[c] = s;
}

template <typename DT>
__global__ void __launch_bounds__(kThreads) k_linrec_grad(const LinrecGradArgs a) {
  const long C = (long)a.B * a.H, c = (long)blockIdx.x * kThreads + threadIdx.x;
  if (c >= C) return;
  const int b = (int)(c / a.H), h = (int)(c % a.H);
  const int n = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const DT* x = reinterpret_cast<const DT*>(a.x.p) + b * a.x.b + h;
  const DT* g = reinterpret_cast<const DT*>(a.gate.p) + b * a.gate.b + h;
  const DT* dy = reinterpret_cast<const DT*>(a.dy.p) + b * a.dy.b + h;
  DT* dx = reinterpret_cast<DT*>(const_cast<void*>(a.dx.p)) + b * a.dx.b + h;
  DT* dg = reinterpret_cast<DT*>(const_cast<void*>(a.dgate.p)) + b * a.dgate.b + h;
  float R = a.dh_T ? a.dh_T[c] : 0.0f;
  for (int t = a.T - 1; t >= 0; --t) {
    float ox = 0.0f, og = 0.0f;
    if (t < n) {
      const float2 p = gate_pair(DType<DT>::load(g, t * a.gate.t));
      const float D = R + DType<DT>::load(dy, t * a.dy.t);
      ox = p.y * D;
      og = p.x * p.y * (a.states[t * C + c] - DType<DT>::load(x, t * a.x.t)) * D;
      R = a.resets && a.resets[(long)t * a.B + b] ? 0.0f : p.x * D;
    }
    DType<DT>::store(dx, t * a.dx.t, ox);
    DType<DT>::store(dg, t * a.dgate.t, og);
  }
  if (a.dh0) a.dh0[c] = R;
}

}  // namespace

size_t linrec_states(int T, int B, int H) { return (size_t)T * B * H * sizeof(float); }
size_t linrec_workspace(int, int, int) { return 256; }

hipError_t launch_linrec(int dtype, const LinrecArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(((long)a.B * a.H + kThreads - 1) / kThreads);
  return dtype == WM_FP32 ? launch("linrec", k_linrec<float>, dim3(grid), dim3(kThreads), 0, s, a)
                          : launch("linrec", k_linrec<bf16_t>, dim3(grid), dim3(kThreads), 0, s, a);
}

hipError_t launch_linrec_grad(int dtype, const LinrecGradArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(((long)a.B * a.H + kThreads - 1) / kThreads);
  return dtype == WM_FP32 ? launch("linrec_grad", k_linrec_grad<float>, dim3(grid), dim3(kThreads), 0, s, a)
                          : launch("linrec_grad", k_linrec_grad<bf16_t>, dim3(grid), dim3(kThreads), 0, s, a);
}

}  // namespace wm
