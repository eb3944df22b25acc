// Layer norm over rows and its gradient:
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, y = xh gamma + beta;
//   q = dy gamma, dx = r (q - mean q - xh mean(q xh)), dgamma = sum dy xh, dbeta = sum dy.
//
// A row is read once, in pieces of 16 bytes, and stays in registers: the mean,
// then the sum of squares about it (not the difference of two large sums), then
// the output.  kLanes lanes share a row: 16 for narrow ones, a wave up to 1024
// values, and four waves, which add their parts in LDS, beyond (up to 32 values
// a lane).  A group of lanes goes over rows in strides with gamma and beta in
// registers, and requests the next row before it works on the present one.
// Rows are aligned to their element only: the hardware takes 16-byte accesses
// at such addresses, and only a row's last, partial piece goes value by value.
//
// The gradient keeps the sums of dy xh and dy for its lanes' columns in
// registers as well; every work-group leaves one row of partial sums, which a
// second launch adds in order.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2048;  // work-groups at most: eight a CU
constexpr int kParts = 512;    // ... of the gradient: two a CU

// Sixteen bytes of a row; piece p of lane t holds columns (kLanes p + t) VEC on.
template <typename DT> struct Piece;
template <> struct Piece<float> {
  static constexpr int VEC = 4;
  typedef uint4 raw;
  __device__ static void get(raw r, float* v) {
    v[0] = __uint_as_float(r.x);
    v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z);
    v[3] = __uint_as_float(r.w);
  }
  __device__ static raw put(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Piece<bf16_t> {
  static constexpr int VEC = 8;
  typedef uint4 raw;
  __device__ static void get(raw r, float* v) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ static raw put(const float* v) {
    return make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
  }
};
typedef uint32_t __attribute__((ext_vector_type(4))) u32x4;
typedef u32x4 __attribute__((aligned(2))) u32x4_2;
typedef u32x4 __attribute__((aligned(4))) u32x4_4;
template <typename DT> struct Memory;
template <> struct Memory<float> { typedef u32x4_4 type; };
template <> struct Memory<bf16_t> { typedef u32x4_2 type; };

// The piece at column c of a row of width H; 0 past its end.
template <typename DT>
__device__ __forceinline__ uint4 load_piece(const DT* row, int c, int H) {
  if (c + Piece<DT>::VEC <= H) {
    const u32x4 v = *reinterpret_cast<const typename Memory<DT>::type*>(row + c);
    return make_uint4(v.x, v.y, v.z, v.w);
  }
  float v[Piece<DT>::VEC];
#pragma unroll
  for (int j = 0; j < Piece<DT>::VEC; ++j) v[j] = c + j < H ? DType<DT>::load(row, c + j) : 0.0f;
  return Piece<DT>::put(v);
}
template <typename DT>
__device__ __forceinline__ void store_piece(DT* row, int c, int H, const float* v) {
  if (c + Piece<DT>::VEC <= H) {
    const uint4 r = Piece<DT>::put(v);
    *reinterpret_cast<typename Memory<DT>::type*>(row + c) = u32x4{r.x, r.y, r.z, r.w};
    return;
  }
#pragma unroll
  for (int j = 0; j < Piece<DT>::VEC; ++j)
    if (c + j < H) DType<DT>::store(row, c + j, v[j]);
}
template <typename DT, int P, int L>
__device__ __forceinline__ void load_row(uint4 (&r)[P], const void* base, long row, long ld, int t, int H) {
  const DT* p = reinterpret_cast<const DT*>(base) + row * ld;
#pragma unroll
  for (int i = 0; i < P; ++i) r[i] = load_piece(p, (L * i + t) * Piece<DT>::VEC, H);
}
// The lane's values of a per-column array, `none` where there is none and past the row's end.
template <typename DT, int P, int L>
__device__ __forceinline__ void load_columns(float (&g)[P][Piece<DT>::VEC], const float* a, float none, int t, int H) {
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < Piece<DT>::VEC; ++j) {
      const int c = (L * p + t) * Piece<DT>::VEC + j;
      g[p][j] = a && c < H ? a[c] : none;
    }
}

// Sums over the lanes of a row; two at a time.
template <int L>
__device__ __forceinline__ float2 row_sum(float2 v, float2 (*sh)[4], int& turn) {
#pragma unroll
  for (int k = (L < 64 ? L : 64) / 2; k; k >>= 1) {
    v.x += __shfl_xor(v.x, k);
    v.y += __shfl_xor(v.y, k);
  }
  if constexpr (L > 64) {
    // two places in turn: a wave may be one sum ahead of another
    if ((threadIdx.x & 63) == 0) sh[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[turn][0];
#pragma unroll
    for (int i = 1; i < L / 64; ++i) {
      v.x += sh[turn][i].x;
      v.y += sh[turn][i].y;
    }
    turn ^= 1;
  }
  return v;
}

template <typename DT, int P, int L>
__global__ void __launch_bounds__(kThreads) k_norm(const NormArgs a) {
  constexpr int V = Piece<DT>::VEC, kRows = kThreads / L;
  __shared__ float2 sh[2][4];
  int turn = 0;
  const int t = threadIdx.x % L;
  const long step = (long)gridDim.x * kRows;
  long row = (long)blockIdx.x * kRows + threadIdx.x / L;
  if (row >= a.rows) return;
  uint4 next[P];
  load_row<DT, P, L>(next, a.x, row, a.x_ld, t, a.H);
  float g[P][V], b[P][V];
  load_columns<DT, P, L>(g, a.gamma, 1.0f, t, a.H);
  load_columns<DT, P, L>(b, a.beta, 0.0f, t, a.H);
  const float inv = 1.0f / (float)a.H;
  for (; row < a.rows; row += step) {
    float v[P][V];
    float2 s = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      Piece<DT>::get(next[p], v[p]);
#pragma unroll
      for (int j = 0; j < V; ++j) s.x += v[p][j];
    }
    if (row + step < a.rows) load_row<DT, P, L>(next, a.x, row + step, a.x_ld, t, a.H);
    const float mu = row_sum<L>(s, sh, turn).x * inv;
    s = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[p][j] = (L * p + t) * V + j < a.H ? v[p][j] - mu : 0.0f;
        s.x = fmaf(v[p][j], v[p][j], s.x);
      }
    const float rs = 1.0f / sqrtf(row_sum<L>(s, sh, turn).x * inv + a.eps);
    DT* y = reinterpret_cast<DT*>(a.y) + row * a.y_ld;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (L * p + t) * V;
#pragma unroll
      for (int j = 0; j < V; ++j) v[p][j] = fmaf(v[p][j] * rs, g[p][j], b[p][j]);
      if (c < a.H) store_piece(y, c, a.H, v[p]);
    }
    if (t == 0 && a.mean) {
      a.mean[row] = mu;
      a.rstd[row] = rs;
    }
  }
}

// part [gridDim.x][2][H]: this work-group's sums of dy xh, then of dy.
template <typename DT, int P, int L>
__global__ void __launch_bounds__(kThreads) k_norm_grad(const NormGradArgs a) {
  constexpr int V = Piece<DT>::VEC, kRows = kThreads / L;
  constexpr bool kAhead = P * V <= 16;  // registers for the next row
  __shared__ float2 sh[2][4];
  __shared__ float add[L < kThreads ? kThreads * P * V : 1];
  int turn = 0;
  const int t = threadIdx.x % L;
  const float inv = 1.0f / (float)a.H;
  const long step = (long)gridDim.x * kRows;
  long row = (long)blockIdx.x * kRows + threadIdx.x / L;
  uint4 xr[P], dr[P];
  float mu = 0.0f, rs = 0.0f;
  auto load = [&](long i) {
    load_row<DT, P, L>(xr, a.x, i, a.x_ld, t, a.H);
    load_row<DT, P, L>(dr, a.dy, i, a.dy_ld, t, a.H);
    mu = a.mean[i];
    rs = a.rstd[i];
  };
  if (row < a.rows) load(row);
  float g[P][V], dg[P][V], db[P][V];
  load_columns<DT, P, L>(g, a.gamma, 1.0f, t, a.H);
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < V; ++j) dg[p][j] = db[p][j] = 0.0f;
  for (; row < a.rows; row += step) {
    if (!kAhead && row >= step) load(row);
    // (past the row's end dy is 0, and so is all that counts there)
    const float m0 = mu, r0 = rs;
    uint4 x0[P], d0[P];
    float2 s = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      x0[p] = xr[p];
      d0[p] = dr[p];
      float v[V], d[V];
      Piece<DT>::get(x0[p], v);
      Piece<DT>::get(d0[p], d);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = (v[j] - m0) * r0, q = d[j] * g[p][j];
        s.x += q;
        s.y = fmaf(q, xh, s.y);
        dg[p][j] = fmaf(d[j], xh, dg[p][j]);
        db[p][j] += d[j];
      }
    }
    if (kAhead && row + step < a.rows) load(row + step);
    s = row_sum<L>(s, sh, turn);
    const float m = s.x * inv, mx = s.y * inv;
    DT* dx = reinterpret_cast<DT*>(a.dx) + row * a.dx_ld;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (L * p + t) * V;
      float v[V], d[V];
      Piece<DT>::get(x0[p], v);
      Piece<DT>::get(d0[p], d);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xh = (v[j] - m0) * r0;
        v[j] = r0 * (d[j] * g[p][j] - m - xh * mx);
      }
      if (c < a.H) store_piece(dx, c, a.H, v);
    }
  }
  // the groups' sums in order: a thread adds one column at a time
  float* part = a.part + (long)blockIdx.x * 2 * a.H;
  for (int which = 0; which < 2; ++which, part += a.H) {
    if constexpr (L < kThreads) {
      __syncthreads();
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) add[(p * V + j) * kThreads + threadIdx.x] = which ? db[p][j] : dg[p][j];
      __syncthreads();
      for (int i = threadIdx.x; i < P * V * L; i += kThreads) {  // value i / L of lane i % L
        const int c = (L * (i / L / V) + i % L) * V + i / L % V;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kRows; ++k) v += add[i / L * kThreads + k * L + i % L];
        if (c < a.H) part[c] = v;
      }
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int c = (L * p + t) * V + j;
          if (c < a.H) part[c] = which ? db[p][j] : dg[p][j];
        }
    }
  }
}

// Adds the n rows of partial sums: 16 columns a work-group, 16 rows at a time,
// each of the 16 in its own order, then these.
__global__ void __launch_bounds__(kThreads) k_norm_sum(const NormGradArgs a, int n) {
  __shared__ float sh[16][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, j = blockIdx.x * 16 + c;
  float s = 0.0f;
  if (j < 2 * a.H) {
    const float* p = a.part + j;
#pragma unroll 8
    for (int i = r; i < n; i += 16) s += p[(long)i * 2 * a.H];
  }
  sh[r][c] = s;
  __syncthreads();
  if (r > 0 || j >= 2 * a.H) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sh[i][c];
  float* out = j < a.H ? a.dgamma : a.dbeta;
  if (out) out[j < a.H ? j : j - a.H] = s;
}

// Lanes of a row, by its width.
int lanes(int dtype, int H) {
  const int v = dtype == WM_FP32 ? 4 : 8;
  return H <= 16 * v ? 16 : H <= 1024 ? 64 : 256;
}
// Work-groups of the gradient: enough to fill the device, few rows of partial
// sums.  (The narrowest rows of the type that packs more of them.)
int parts(long rows, int H) {
  const long per = kThreads / lanes(WM_FP32, H);
  return (int)std::max<long>(1, std::min<long>((rows + per - 1) / per, kParts));
}

// Runs f with the pieces of a lane and the lanes of a row as constants.
template <int N> using Const = std::integral_constant<int, N>;
template <typename DT, typename F>
hipError_t by_width(int H, F f) {
  constexpr int V = Piece<DT>::VEC, k = V / 4;  // bf16 pieces hold twice the values
  if (H <= 16 * V) return f(Const<1>(), Const<16>());
  if (H <= 64 * V) return f(Const<1>(), Const<64>());
  if (k == 1 && H <= 512) return f(Const<2 / k>(), Const<64>());
  if (H <= 1024) return f(Const<4 / k>(), Const<64>());
  if (H <= 2048) return f(Const<2 / k>(), Const<256>());
  if (H <= 4096) return f(Const<4 / k>(), Const<256>());
  return f(Const<8 / k>(), Const<256>());
}

}  // namespace

hipError_t launch_layer_norm(int dtype, const NormArgs& a, hipStream_t s) {
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    return by_width<DT>(a.H, [&](auto p, auto l) {
      const long per = kThreads / l, groups = std::min<long>((a.rows + per - 1) / per, kGroups);
      return launch("norm", k_norm<DT, p, l>, dim3((unsigned)groups), dim3(kThreads), 0, s, a);
    });
  };
  return dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
}

size_t layer_norm_grad_workspace(long rows, int H) { return (size_t)parts(rows, H) * 2 * H * sizeof(float); }

hipError_t launch_layer_norm_grad(int dtype, const NormGradArgs& a, hipStream_t s) {
  const int n = parts(a.rows, a.H);
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    return by_width<DT>(a.H, [&](auto p, auto l) {
      return launch("norm_grad", k_norm_grad<DT, p, l>, dim3(n), dim3(kThreads), 0, s, a);
    });
  };
  const hipError_t e = dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
  if (e != hipSuccess) return e;
  return launch("norm_sum", k_norm_sum, dim3((unsigned)((2 * a.H + 15) / 16)), dim3(kThreads), 0, s, a, n);
}

}  // namespace wm
