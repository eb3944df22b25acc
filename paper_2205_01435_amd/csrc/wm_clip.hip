// The global norm of a list of gradient tensors, and the tensors scaled to it:
//   N = sqrt(sum over all tensors of sum g^2),  out = g (N > max ? max / N : 1).
// Squares are summed in 64 bits: fp32 squares overflow from |g| = 1.8e19 and
// vanish below 1e-23, and the sum runs over up to billions of terms.  The
// tensors are cut into chunks; every chunk's sum has its place in the
// workspace and the second launch adds them in one order, so that the result
// depends on the tensors alone.
#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16384;  // elements
constexpr int kPerLaunch = 64; // tensors whose table fits a launch's arguments

struct Table {
  int n;                      // tensors of this launch
  long part0;                 // place of its first chunk's sum
  long first[kPerLaunch + 1]; // chunks before each tensor
  const void* in[kPerLaunch];
  void* out[kPerLaunch];
  long len[kPerLaunch];
  int32_t dtype[kPerLaunch];
};

__device__ __forceinline__ int find(const Table& t, long c) {
  int i = 0;
  while (c >= t.first[i + 1]) ++i;
  return i;
}

__device__ double block_sum(double v, double* sh) {
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__global__ void __launch_bounds__(kThreads) k_clip_sum(const Table t, double* part) {
  __shared__ double sh[4];
  const long c = blockIdx.x;
  const int i = find(t, c);
  const long at = (c - t.first[i]) * kChunk, end = min(at + (long)kChunk, t.len[i]);
  double s = 0.0;
  for (long k = at + threadIdx.x; k < end; k += kThreads) {
    const double g = t.dtype[i] == WM_FP32 ? DType<float>::load((const float*)t.in[i], k)
                                           : DType<bf16_t>::load((const bf16_t*)t.in[i], k);
    s += g * g;
  }
  s = block_sum(s, sh);
  if (threadIdx.x == 0) part[t.part0 + c] = s;
}

__global__ void __launch_bounds__(kThreads) k_clip_scale(const Table t, const double* part, long nparts, float max_norm,
                                                         float* norm) {
  __shared__ double sh[4];
  double s = 0.0;
  for (long k = threadIdx.x; k < nparts; k += kThreads) s += part[k];
  const double N = sqrt(block_sum(s, sh));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)N;
  const float f = N > (double)max_norm && N < (double)INFINITY ? (float)((double)max_norm / N) : 1.0f;
  const long c = blockIdx.x;
  const int i = find(t, c);
  const long at = (c - t.first[i]) * kChunk, end = min(at + (long)kChunk, t.len[i]);
  if (t.in[i] == t.out[i] && f == 1.0f) return;
  for (long k = at + threadIdx.x; k < end; k += kThreads) {
    if (t.dtype[i] == WM_FP32)
      ((float*)t.out[i])[k] = f * ((const float*)t.in[i])[k];
    else
      DType<bf16_t>::store((bf16_t*)t.out[i], k, f * DType<bf16_t>::load((const bf16_t*)t.in[i], k));
  }
}

long chunks(long n) { return (n + kChunk - 1) / kChunk; }

// Runs f on the table of each launch.
template <typename F>
hipError_t tables(int n, const wm_grad_tensor* t, F f) {
  long part0 = 0;
  for (int i = 0; i < n;) {
    Table tab{};
    tab.part0 = part0;
    for (; i < n && tab.n < kPerLaunch; ++i) {
      if (t[i].n == 0) continue;
      const int k = tab.n++;
      tab.in[k] = t[i].grad;
      tab.out[k] = t[i].out;
      tab.len[k] = t[i].n;
      tab.dtype[k] = t[i].dtype;
      tab.first[k + 1] = tab.first[k] + chunks(t[i].n);
    }
    if (tab.n == 0) break;
    part0 += tab.first[tab.n];
    const hipError_t e = f(tab, (unsigned)tab.first[tab.n]);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

__global__ void k_clip_none(float* norm) { *norm = 0.0f; }

}  // namespace

size_t clip_workspace(int n, const wm_grad_tensor* t) {
  long c = 0;
  for (int i = 0; i < n; ++i) c += chunks(t[i].n);
  return (size_t)(c > 0 ? c : 1) * sizeof(double);
}

hipError_t launch_clip(int n, const wm_grad_tensor* t, float max_norm, float* norm, void* ws, hipStream_t s) {
  double* part = reinterpret_cast<double*>(ws);
  long total = 0;
  for (int i = 0; i < n; ++i) total += chunks(t[i].n);
  if (total == 0) return launch("clip_none", k_clip_none, dim3(1), dim3(1), 0, s, norm);
  hipError_t e = tables(n, t, [&](const Table& tab, unsigned grid) {
    return launch("clip_sum", k_clip_sum, dim3(grid), dim3(kThreads), 0, s, tab, part);
  });
  if (e != hipSuccess) return e;
  return tables(n, t, [&](const Table& tab, unsigned grid) {
    return launch("clip_scale", k_clip_scale, dim3(grid), dim3(kThreads), 0, s, tab, (const double*)part, total,
                  max_norm, tab.part0 == 0 ? norm : nullptr);
  });
}

}  // namespace wm
