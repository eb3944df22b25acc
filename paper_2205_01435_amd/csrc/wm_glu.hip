// The gated projection of a feed-forward block and its gradient:
//   [g | u] = x W^T, h = act(g) u;
//   [dg | du] = [dh u act'(g) | dh act(g)], dx = [dg | du] W, dW = [dg | du]^T x.
//
// One product kernel serves all three, out[m, n] = sum over k of Q[m, k] P[n, k],
// with either operand stored along k (x, W and dg | du as rows) or across it (W and
// x where the sum goes over their rows): the first kind is read from LDS as 16-byte
// pieces, the second four rows at a time by the transposing read.  The forward
// product takes the same 64 columns of both factors into one tile, so that the
// activation and the product are its epilogue and the two factors leave the chip
// only where the gradient needs them.  Where the tiles are too few for the device
// the sum is split over work-groups, whose fp32 parts a second launch adds in order.
//
// Bound by the matrix unit from some hundred rows on, by reading W below.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_attend.h"
#include "wm_profile.h"
#include "wm_split.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;  // outputs of a tile in each direction

typedef uint32_t __attribute__((ext_vector_type(4))) v4u;
typedef uint32_t __attribute__((ext_vector_type(2))) v2u;
typedef v4u __attribute__((aligned(2))) v4u_2;
typedef v4u __attribute__((aligned(4))) v4u_4;
typedef v2u __attribute__((aligned(2))) v2u_2;

template <typename DT> struct El;
template <> struct El<float> {
  static constexpr int VEC = 4, BK = 32, SL = 16;  // SL: k of one 16-byte piece of a fragment for each lane group
  typedef v4u_4 mem;
};
template <> struct El<bf16_t> {
  static constexpr int VEC = 8, BK = 64, SL = 32;
  typedef v4u_2 mem;
};

template <typename DT>
__device__ __forceinline__ v4u load_piece(const DT* row, long c, long width) {
  constexpr int V = El<DT>::VEC;
  if (c + V <= width) return *reinterpret_cast<const typename El<DT>::mem*>(row + c);
  v4u r = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (c + i < width) {
      if constexpr (sizeof(DT) == 4)
        r[i] = __float_as_uint(row[c + i]);
      else
        r[i / 2] |= (uint32_t)row[c + i] << (16 * (i & 1));
    }
  return r;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ v2u read_tr(const bf16_t* p) {
  typedef __attribute__((address_space(3))) s16x4* lds_t;
  return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)p));
}

// One operand: rows of `ld` elements.  Along k: row i of the tile is output i,
// columns are k.  Across: row k, columns are outputs.
struct Operand {
  const void* p;
  long ld;
};

// A tile's 128 outputs x BK of one operand, from memory through registers into LDS.
template <typename DT, bool ACROSS>
struct Stage {
  static constexpr int V = El<DT>::VEC, BK = El<DT>::BK;
  // pitches: rows of 16 neighbouring outputs (four of k) on different banks
  static constexpr int PITCH = ACROSS ? kTile + 32 / (int)sizeof(DT) : BK + (sizeof(DT) == 2 ? 16 : 4);
  static constexpr int ROWS = ACROSS ? BK : kTile, COLS = ACROSS ? kTile : BK;
  static constexpr int N = ROWS * (COLS / V) / kThreads;
  static constexpr int SIZE = ROWS * PITCH;
  v4u r[N];
  // outputs [o0, o0 + 128) of `outs`, k [k0, k0 + BK) up to kend; `split` rows of the
  // tile on, outputs count from o1 (the other factor's columns)
  __device__ __forceinline__ void load(const Operand& a, long o0, long o1, int split, long outs, long k0, long kend) {
    const DT* p = reinterpret_cast<const DT*>(a.p);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = threadIdx.x + i * kThreads, row = q / (COLS / V), col = q % (COLS / V) * V;
      if constexpr (ACROSS) {
        r[i] = k0 + row < kend ? load_piece<DT>(p + (k0 + row) * a.ld, o0 + col, outs) : v4u{0, 0, 0, 0};
      } else {
        const int in = row < split ? row : row - split;
        const long o = row < split ? o0 + row : o1 + in;
        r[i] = o0 + in < outs ? load_piece<DT>(p + o * a.ld, k0 + col, kend) : v4u{0, 0, 0, 0};
      }
    }
  }
  __device__ __forceinline__ void store(DT* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = threadIdx.x + i * kThreads;
      *reinterpret_cast<v4u*>(lds + q / (COLS / V) * PITCH + q % (COLS / V) * V) = r[i];
    }
  }
  // the fragment of sixteen outputs from o on, k from k on
  __device__ __forceinline__ static uint4 frag(const DT* lds, int o, int k) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
    if constexpr (!ACROSS) {
      return *reinterpret_cast<const uint4*>(lds + (o + j) * PITCH + k + V * g);
    } else if constexpr (sizeof(DT) == 4) {
      const float* p = lds + (k + 4 * g) * PITCH + o + j;
      return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[PITCH]), __float_as_uint(p[2 * PITCH]),
                        __float_as_uint(p[3 * PITCH]));
    } else {
      const bf16_t* p = lds + (k + 8 * g + j / 4) * PITCH + o + 4 * (j % 4);
      const v2u a = read_tr(p), b = read_tr(p + 4 * PITCH);
      return make_uint4(a.x, a.y, b.x, b.y);
    }
  }
};

__device__ __forceinline__ float normal_cdf(float x) { return 0.5f * erfcf(x * -0.70710678118654752f); }
// act(g) and its derivative
__device__ __forceinline__ float2 activate(int act, float g) {
  if (act == WM_ACT_SILU) {
    const float2 s = gate_pair_of(g, expf(-fabsf(g)));
    return make_float2(g * s.x, s.x * fmaf(g, s.y, 1.0f));
  }
  const float c = normal_cdf(g);
  return make_float2(g * c, fmaf(g * 0.39894228040143268f, expf(-0.5f * g * g), c));
}

template <typename DT>
__device__ __forceinline__ void store4(DT* row, long c, long width, const float (&v)[4]) {
  if (c + 4 <= width) {
    if constexpr (sizeof(DT) == 4)
      *reinterpret_cast<v4u_4*>(row + c) =
          v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else
      *reinterpret_cast<v2u_2*>(row + c) = v2u{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < width) DType<DT>::store(row, c + e, v[e]);
  }
}

struct ProductArgs {
  Operand P, Q;
  long M, N, K;     // outputs of Q and P, the sum's length
  void* out;        // [M, N] (GLU: h [M, N] with N = F)
  long out_ld;
  void* pre;        // GLU: [M, 2 N] or null
  int act;
  float* part;      // splits > 1: [splits][M][N]
  int splits;
  long per;         // k of a split, a multiple of BK
  int tiles_n;
};

template <typename DT, bool PX, bool QX, bool GLU>
__global__ void __launch_bounds__(kThreads) k_product(const ProductArgs a) {
  typedef Stage<DT, PX> SP;
  typedef Stage<DT, QX> SQ;
  constexpr int BK = El<DT>::BK, SL = El<DT>::SL;
  __shared__ __align__(16) DT pl[SP::SIZE];
  __shared__ __align__(16) DT ql[SQ::SIZE];
  const int w = threadIdx.x >> 6, wp = w & 1, wq = w >> 1, lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const long tile = blockIdx.x / a.splits;
  const int split = (int)(blockIdx.x % a.splits);
  const long n0 = tile % a.tiles_n * (GLU ? kTile / 2 : kTile), m0 = tile / a.tiles_n * kTile;
  const long k0 = split * a.per, k1 = min(k0 + a.per, a.K);

  f32x4 acc[4][4];  // [block of P][block of Q]
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  // where this wave's blocks of P start in the tile: half a tile together, or 32 outputs of both factors
  auto block = [&](int i) { return GLU ? 64 * (i >> 1) + 32 * wp + 16 * (i & 1) : 64 * wp + 16 * i; };

  SP sp;
  SQ sq;
  const int half = GLU ? kTile / 2 : kTile;
  sp.load(a.P, n0, a.N + n0, half, a.N, k0, k1);
  sq.load(a.Q, m0, 0, kTile, a.M, k0, k1);
  for (long k = k0; k < k1; k += BK) {
    __syncthreads();
    sp.store(pl);
    sq.store(ql);
    __syncthreads();
    if (k + BK < k1) {
      sp.load(a.P, n0, a.N + n0, half, a.N, k + BK, k1);
      sq.load(a.Q, m0, 0, kTile, a.M, k + BK, k1);
    }
#pragma unroll
    for (int s = 0; s < BK; s += SL) {
      uint4 p[4], q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = SP::frag(pl, block(i), s);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = SQ::frag(ql, 64 * wq + 16 * i, s);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int l = 0; l < 4; ++l) Mfma<DT>::step(acc[i][l], p[i], q[l]);
    }
  }

#pragma unroll
  for (int l = 0; l < 4; ++l) {
    const long m = m0 + 64 * wq + 16 * l + j;
    if (m >= a.M) continue;
    if constexpr (GLU) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const long n = n0 + 32 * wp + 16 * i + 4 * g;
        float gate[4], up[4], h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          gate[e] = acc[i][l][e];
          up[e] = acc[i + 2][l][e];
          h[e] = activate(a.act, gate[e]).x * up[e];
        }
        store4(reinterpret_cast<DT*>(a.out) + m * a.out_ld, n, a.N, h);
        if (a.pre) {
          DT* pre = reinterpret_cast<DT*>(a.pre) + m * 2 * a.N;
          store4(pre, n, a.N, gate);
          store4(pre + a.N, n, a.N, up);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long n = n0 + block(i) + 4 * g;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][l][e];
        if (a.splits > 1)
          store4(a.part + ((long)split * a.M + m) * a.N, n, a.N, v);
        else
          store4(reinterpret_cast<DT*>(a.out) + m * a.out_ld, n, a.N, v);
      }
    }
  }
}

// Adds the splits' parts in order.
template <typename DT>
__global__ void __launch_bounds__(kThreads) k_product_sum(const ProductArgs a) {
  const long i = (long)blockIdx.x * kThreads + threadIdx.x, n = a.M * a.N;
  if (i >= n) return;
  float s = 0.0f;
#pragma unroll 4
  for (int k = 0; k < a.splits; ++k) s += a.part[k * n + i];
  DType<DT>::store(reinterpret_cast<DT*>(a.out) + i / a.N * a.out_ld, i % a.N, s);
}

// dpre [rows, 2F] from pre and dh.
template <typename DT>
__global__ void __launch_bounds__(kThreads) k_glu_back(const GluGradArgs a, DT* dpre) {
  const long parts = (a.F + 3) / 4, i = (long)blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.rows * parts) return;
  const long row = i / parts;
  const int c = (int)(i % parts) * 4;
  const DT* pre = reinterpret_cast<const DT*>(a.pre) + row * 2 * a.F;
  const DT* dh = reinterpret_cast<const DT*>(a.dh) + row * a.dh_ld;
  float dg[4], du[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int k = min(c + e, a.F - 1);
    const float d = DType<DT>::load(dh, k), u = DType<DT>::load(pre, a.F + k);
    const float2 v = activate(a.act, DType<DT>::load(pre, k));
    dg[e] = d * u * v.y;
    du[e] = d * v.x;
  }
  DT* out = dpre + row * 2 * a.F;
  store4(out, c, a.F, dg);
  store4(out + a.F, c, a.F, du);
}

// Splits of a sum of length K for M x N outputs.
int splits_of(long M, long N, long K, int bk) {
  const long tiles = std::max(1L, (M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
  if (tiles >= 256) return 1;
  return (int)std::max<long>(1, std::min<long>(512 / tiles, K / (8 * bk)));
}

template <typename DT, bool PX, bool QX, bool GLU>
hipError_t product(const char* name, ProductArgs a, hipStream_t s) {
  constexpr int BK = El<DT>::BK;
  const int width = GLU ? kTile / 2 : kTile;
  a.tiles_n = (int)((a.N + width - 1) / width);
  const long tiles = (a.M + kTile - 1) / kTile * a.tiles_n;
  a.splits = GLU ? 1 : splits_of(a.M, a.N, a.K, BK);
  a.per = ((a.K + a.splits - 1) / a.splits + BK - 1) / BK * BK;
  const hipError_t e =
      launch(name, k_product<DT, PX, QX, GLU>, dim3((unsigned)(tiles * a.splits)), dim3(kThreads), 0, s, a);
  if (e != hipSuccess || a.splits == 1) return e;
  return launch("glu_sum", k_product_sum<DT>, dim3((unsigned)((a.M * a.N + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
size_t part_bytes(long M, long N, long K, int bk) {
  const int s = splits_of(M, N, K, bk);
  return s > 1 ? (size_t)s * M * N * sizeof(float) : 0;
}

}  // namespace

hipError_t launch_glu(int dtype, const GluArgs& a, hipStream_t s) {
  const ProductArgs p{{a.W, a.D}, {a.x, a.x_ld}, a.rows, a.F, a.D, a.h, a.h_ld, a.pre, a.act, nullptr, 1, 0, 0};
  return dtype == WM_FP32 ? product<float, false, false, true>("glu", p, s) : product<bf16_t, false, false, true>("glu", p, s);
}

size_t glu_grad_workspace(int dtype, long rows, int D, int F) {
  const int bk = dtype == WM_FP32 ? El<float>::BK : El<bf16_t>::BK, size = dtype == WM_FP32 ? 4 : 2;
  return align256((size_t)rows * 2 * F * size) +
         align256(std::max(part_bytes(rows, D, 2L * F, bk), part_bytes(2L * F, D, rows, bk)));
}

hipError_t launch_glu_grad(int dtype, const GluGradArgs& a, hipStream_t s) {
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    DT* dpre = reinterpret_cast<DT*>(a.ws);
    float* part = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + align256((size_t)a.rows * 2 * a.F * sizeof(DT)));
    hipError_t e = hipSuccess;
    if (a.rows > 0) {
      const long n = a.rows * ((a.F + 3) / 4);
      e = launch("glu_back", k_glu_back<DT>, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a, dpre);
      if (e != hipSuccess) return e;
      const ProductArgs dx{{a.W, a.D}, {dpre, 2L * a.F}, a.rows, a.D, 2L * a.F, a.dx, a.dx_ld, nullptr, 0, part, 1, 0, 0};
      if ((e = product<DT, true, false, false>("glu_dx", dx, s)) != hipSuccess) return e;
    }
    if (!a.dW) return e;
    const ProductArgs dw{{a.x, a.x_ld}, {dpre, 2L * a.F}, 2L * a.F, a.D, a.rows, a.dW, a.D, nullptr, 0, part, 1, 0, 0};
    return product<DT, true, true, false>("glu_dw", dw, s);
  };
  return dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
}

}  // namespace wm
