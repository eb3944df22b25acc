// Rows of an action table for logged actions, scaled, and the table's
// gradient (the one-hot product of the world model's input as a gather, and
// its transpose).
//   y_i = s E[a_i], 0 where a_i is outside [0, V);  dE_v = s sum_{a_i = v} dy_i.
#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

template <typename DT>
__global__ void __launch_bounds__(256) k_embed(const EmbedArgs a) {
  const DT* table = reinterpret_cast<const DT*>(a.table);
  DT* out = reinterpret_cast<DT*>(a.out);
  for (long i = blockIdx.x; i < a.n; i += gridDim.x) {
    const int tok = a.tokens[i];
    const bool ok = tok >= 0 && tok < a.V;
    for (int h = threadIdx.x; h < a.H; h += 256)
      DType<DT>::store(out, i * a.out_ld + h, ok ? a.scale * DType<DT>::load(table, (long)tok * a.H + h) : 0.0f);
  }
}

// One work-group per table row: its tokens' positions are collected 256 at a
// time in order, and their rows summed.
template <typename DT>
__global__ void __launch_bounds__(256) k_embed_grad(const EmbedGradArgs a) {
  __shared__ int pos[256];
  __shared__ int cnt[4];
  const DT* dout = reinterpret_cast<const DT*>(a.dout);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int v = blockIdx.x; v < a.V; v += gridDim.x) {
    for (int h0 = 0; h0 < a.H; h0 += 256) {
      const int h = h0 + threadIdx.x;
      float acc = 0.0f;
      for (long i0 = 0; i0 < a.n; i0 += 256) {
        const long i = i0 + threadIdx.x;
        const bool hit = i < a.n && a.tokens[i] == v;
        const unsigned long long m = __ballot(hit);
        if (lane == 0) cnt[wave] = __popcll(m);
        __syncthreads();
        int base = 0, total = 0;
        for (int w = 0; w < 4; ++w) {
          if (w < wave) base += cnt[w];
          total += cnt[w];
        }
        if (hit) pos[base + __popcll(m & ((1ull << lane) - 1))] = (int)i;
        __syncthreads();
        for (int k = 0; k < total; ++k)
          if (h < a.H) acc += DType<DT>::load(dout, (long)pos[k] * a.dout_ld + h);
        __syncthreads();
      }
      if (h < a.H) a.dtable[(long)v * a.H + h] = a.scale * acc;
    }
  }
}

}  // namespace

hipError_t launch_embed(int dtype, const EmbedArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n < 65536 ? a.n : 65536);
  return dtype == WM_FP32 ? launch("embed", k_embed<float>, dim3(grid), dim3(256), 0, s, a)
                          : launch("embed", k_embed<bf16_t>, dim3(grid), dim3(256), 0, s, a);
}

size_t embed_grad_workspace(long n, int, int) { return 256 + (size_t)n * 8; }  // (token, position) pairs

hipError_t launch_embed_grad(int dtype, const EmbedGradArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.V < 65536 ? a.V : 65536);
  return dtype == WM_FP32 ? launch("embed_grad", k_embed_grad<float>, dim3(grid), dim3(256), 0, s, a)
                          : launch("embed_grad", k_embed_grad<bf16_t>, dim3(grid), dim3(256), 0, s, a);
}

}  // namespace wm
