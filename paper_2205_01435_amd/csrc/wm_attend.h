// Shared by the attending core's operators (wm_qknorm.hip, wm_linattn.hip,
// wm_glu.hip): launch arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wm_seq.h"

namespace wm {

constexpr int kQkMaxD = 256;
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
  // set by the launcher: items of a step, and the gradient's work-groups of each side
  int parts, groups[2];
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
  void* saved;  // glu_saved bytes, or null
};
struct GluGradArgs {
  long rows;
  int D, F, act;
  const void* x;
  long x_ld;
  const void* W;
  const void* saved;
  const void* dh;
  long dh_ld;
  void* dx;
  long dx_ld;
  void* dW;  // [2F, D], or null
  void* ws;
};
size_t glu_saved(int dtype, long rows, int F);
size_t glu_grad_workspace(int dtype, long rows, int D, int F);
hipError_t launch_glu(int dtype, const GluArgs& a, hipStream_t s);
hipError_t launch_glu_grad(int dtype, const GluGradArgs& a, hipStream_t s);

// Sixteen bytes of a row, at any alignment of its elements.
typedef uint32_t __attribute__((ext_vector_type(4))) v4u;
typedef uint32_t __attribute__((ext_vector_type(2))) v2u;
typedef v4u __attribute__((aligned(2))) v4u_2;
typedef v4u __attribute__((aligned(4))) v4u_4;
typedef v2u __attribute__((aligned(2))) v2u_2;
template <typename DT> struct Mem16;
template <> struct Mem16<float> { typedef v4u_4 type; };
template <> struct Mem16<bf16_t> { typedef v4u_2 type; };

// The elements of r from number n on (1 .. VEC), zeros behind them.
template <typename DT>
__device__ __forceinline__ v4u elements_from(v4u r, int n) {
  if constexpr (sizeof(DT) == 2) {
    // an odd element first: half a word down
    if (n & 1)
      r = v4u{r.x >> 16 | r.y << 16, r.y >> 16 | r.z << 16, r.z >> 16 | r.w << 16, r.w >> 16};
    n >>= 1;
  }
  if (n & 1) r = v4u{r.y, r.z, r.w, 0};
  if (n & 2) r = v4u{r.z, r.w, 0, 0};
  return n & 4 ? v4u{0, 0, 0, 0} : r;
}

// 16 bytes of a row from column c on, zeros past its `width`.  The end of a row is read
// as its last 16 bytes: value by value, each load behind a branch of its own, a
// tile's edge takes longer than the tile.
template <typename DT>
__device__ __forceinline__ v4u load_piece(const DT* row, long c, long width) {
  constexpr int V = 16 / (int)sizeof(DT);
  if (c + V <= width) return *reinterpret_cast<const typename Mem16<DT>::type*>(row + c);
  if (c >= width) return v4u{0, 0, 0, 0};
  if (width >= V)
    return elements_from<DT>(*reinterpret_cast<const typename Mem16<DT>::type*>(row + width - V), (int)(c + V - width));
  v4u r = {0, 0, 0, 0};
  DT v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = row[min(c + i, width - 1)];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool in = c + i < width;
    if constexpr (sizeof(DT) == 4)
      r[i] = in ? __float_as_uint(v[i]) : 0u;
    else
      r[i / 2] |= in ? (uint32_t)v[i] << (16 * (i & 1)) : 0u;
  }
  return r;
}

// Four rows of one column from a row-major bf16 matrix in LDS: sixteen lanes read
// four rows of sixteen columns, four values each (p: row j / 4, columns 4 (j % 4)
// on, j the lane of the sixteen), and get column j.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v2u read_tr(const bf16_t* p) {
  typedef __attribute__((address_space(3))) s16x4* lds_t;
  return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)p));
}

}  // namespace wm
