// Layer norm over rows and its gradient:
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, y = xh gamma + beta;
//   q = dy gamma, dx = r (q - mean q - xh mean(q xh)), dgamma = sum dy xh, dbeta = sum dy.
#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPart = 512;  // work-groups of the gradient, each with one row of partial sums

__device__ __forceinline__ float block_sum(float v, float* sh) {
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

template <typename DT>
__global__ void __launch_bounds__(kThreads) k_norm(const NormArgs a) {
  __shared__ float sh[4];
  for (long i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const DT* x = reinterpret_cast<const DT*>(a.x) + i * a.x_ld;
    DT* y = reinterpret_cast<DT*>(a.y) + i * a.y_ld;
    float s = 0.0f;
    for (int h = threadIdx.x; h < a.H; h += kThreads) s += DType<DT>::load(x, h);
    const float mu = block_sum(s, sh) / (float)a.H;
    s = 0.0f;
    for (int h = threadIdx.x; h < a.H; h += kThreads) {
      const float d = DType<DT>::load(x, h) - mu;
      s += d * d;
    }
    const float r = 1.0f / sqrtf(block_sum(s, sh) / (float)a.H + a.eps);
    for (int h = threadIdx.x; h < a.H; h += kThreads) {
      const float xh = (DType<DT>::load(x, h) - mu) * r;
      DType<DT>::store(y, h, (a.gamma ? xh * a.gamma[h] : xh) + (a.beta ? a.beta[h] : 0.0f));
    }
    if (threadIdx.x == 0 && a.mean) a.mean[i] = mu, a.rstd[i] = r;
  }
}

// part [gridDim.x, 2, H]: this work-group's sums of dy xh and dy
template <typename DT>
__global__ void __launch_bounds__(kThreads) k_norm_grad(const NormGradArgs a) {
  __shared__ float sh[4];
  constexpr int kCols = kNormMaxH / kThreads;
  float dg[kCols], db[kCols];
  for (int c = 0; c < kCols; ++c) dg[c] = db[c] = 0.0f;
  for (long i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const DT* x = reinterpret_cast<const DT*>(a.x) + i * a.x_ld;
    const DT* dy = reinterpret_cast<const DT*>(a.dy) + i * a.dy_ld;
    DT* dx = reinterpret_cast<DT*>(a.dx) + i * a.dx_ld;
    const float mu = a.mean[i], r = a.rstd[i];
    float s = 0.0f, sx = 0.0f;
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      const int h = c * kThreads + threadIdx.x;
      if (h < a.H) {
        const float xh = (DType<DT>::load(x, h) - mu) * r, d = DType<DT>::load(dy, h);
        const float q = a.gamma ? d * a.gamma[h] : d;
        s += q;
        sx += q * xh;
        dg[c] += d * xh;
        db[c] += d;
      }
    }
    const float m = block_sum(s, sh) / (float)a.H, mx = block_sum(sx, sh) / (float)a.H;
    for (int h = threadIdx.x; h < a.H; h += kThreads) {
      const float xh = (DType<DT>::load(x, h) - mu) * r, d = DType<DT>::load(dy, h);
      const float q = a.gamma ? d * a.gamma[h] : d;
      DType<DT>::store(dx, h, r * (q - m - xh * mx));
    }
  }
#pragma unroll
  for (int c = 0; c < kCols; ++c) {
    const int h = c * kThreads + threadIdx.x;
    if (h < a.H) {
      a.part[((long)blockIdx.x * 2) * a.H + h] = dg[c];
      a.part[((long)blockIdx.x * 2 + 1) * a.H + h] = db[c];
    }
  }
}

__global__ void __launch_bounds__(kThreads) k_norm_grad_sum(const NormGradArgs a, int n) {
  const int j = blockIdx.x * kThreads + threadIdx.x;
  if (j >= 2 * a.H) return;
  float s = 0.0f;
  for (int i = 0; i < n; ++i) s += a.part[(long)i * 2 * a.H + j];
  float* out = j < a.H ? a.dgamma : a.dbeta;
  if (out) out[j < a.H ? j : j - a.H] = s;
}

int parts(long rows) { return (int)(rows < kMaxPart ? (rows > 0 ? rows : 1) : kMaxPart); }

}  // namespace

hipError_t launch_layer_norm(int dtype, const NormArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.rows < 65536 ? a.rows : 65536);
  return dtype == WM_FP32 ? launch("norm", k_norm<float>, dim3(grid), dim3(kThreads), 0, s, a)
                          : launch("norm", k_norm<bf16_t>, dim3(grid), dim3(kThreads), 0, s, a);
}

size_t layer_norm_grad_workspace(long rows, int H) { return (size_t)parts(rows) * 2 * H * sizeof(float); }

hipError_t launch_layer_norm_grad(int dtype, const NormGradArgs& a, hipStream_t s) {
  const int n = parts(a.rows);
  hipError_t e = dtype == WM_FP32 ? launch("norm_grad", k_norm_grad<float>, dim3(n), dim3(kThreads), 0, s, a)
                                  : launch("norm_grad", k_norm_grad<bf16_t>, dim3(n), dim3(kThreads), 0, s, a);
  if (e != hipSuccess) return e;
  return launch("norm_grad_sum", k_norm_grad_sum, dim3((2 * a.H + kThreads - 1) / kThreads), dim3(kThreads), 0, s, a, n);
}

}  // namespace wm
