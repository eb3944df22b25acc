// Shared by the attending core's operators (wm_qknorm.hip, wm_linattn.hip,
// wm_glu.hip): launch arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wm_seq.h"

namespace wm {

constexpr int kQkMaxD = 512;
// One of queries and keys: rows of `heads` x D values, `ld` elements apart.
struct QkSide {
  int heads;
  const void* x;
  long x_ld;
  const float* gamma;  // [D] or null (1)
  const void* dout;    // gradient only
  long dout_ld;
  void* out;  // the outputs, or the gradients
  long out_ld;
  float* dgamma;  // [D] or null, gradient only
};
struct QkArgs {
  long rows;
  int D, R;
  int neighbours;  // pairs (2i, 2i + 1), else (i, i + R / 2)
  float eps;
  const int32_t* pos;
  const uint64_t* table;  // [R / 2]
  QkSide side[2];
  float* part;  // gradient: workspace
  int group;    // heads of one work item (set by the launcher)
};
size_t qk_norm_grad_workspace(long rows, int Hq, int Hk, int D);
hipError_t launch_qk_norm(int dtype, const QkArgs& a, hipStream_t s);
hipError_t launch_qk_norm_grad(int dtype, const QkArgs& a, hipStream_t s);

constexpr int kAttnMax = 128;  // widest head
struct LinattnArgs {
  int T, B, N, K, V;
  SeqView q, k, v;
  const float* decay;  // [N]
  float scale;
  const float* h0;         // [B, N, K, V] or null (0)
  const uint8_t* resets;   // [T, B] or null
  const int32_t* lengths;  // [B] or null (T)
  void* y;                 // [T, B, N, V]
  float* h_T;              // [B, N, K, V] or null
  float* states;           // linattn_states bytes or null
  void* ws;
};
struct LinattnGradArgs {
  int T, B, N, K, V;
  SeqView q, k, v, dy, dq, dk, dv;  // dq, dk, dv are written
  const float* decay;
  float scale;
  const float* h0;    // or null (0)
  const uint8_t* resets;
  const int32_t* lengths;
  const float* dh_T;  // [B, N, K, V] or null (0)
  const float* states;
  float* dh0;  // or null
  void* ws;
};
size_t linattn_states(int T, int B, int N, int K, int V);     // bytes
size_t linattn_workspace(int T, int B, int N, int K, int V);  // bytes
hipError_t launch_linattn(int dtype, const LinattnArgs& a, hipStream_t s);
hipError_t launch_linattn_grad(int dtype, const LinattnGradArgs& a, hipStream_t s);

struct GluArgs {
  long rows;
  int D, F, act;
  const void* x;
  long x_ld;
  const void* W;  // [2F, D]: the gate's rows, then the other factor's
  void* h;
  long h_ld;
  void* pre;  // [rows, 2F] or null
};
struct GluGradArgs {
  long rows;
  int D, F, act;
  const void* x;
  long x_ld;
  const void* W;
  const void* pre;
  const void* dh;
  long dh_ld;
  void* dx;
  long dx_ld;
  void* dW;  // [2F, D], or null
  void* ws;
};
size_t glu_grad_workspace(int dtype, long rows, int D, int F);
hipError_t launch_glu(int dtype, const GluArgs& a, hipStream_t s);
hipError_t launch_glu_grad(int dtype, const GluGradArgs& a, hipStream_t s);

}  // namespace wm
