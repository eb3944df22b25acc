// The gated projection of a feed-forward block and its gradient:
//   [g | u] = x W^T, h = act(g) u;
//   [dg | du] = [dh u act'(g) | dh act(g)], dx = [dg | du] W, dW = [dg | du]^T x.
//
// Every product is out[m, n] = sum over k of Q[m, k] P[n, k], with either operand
// stored along k (x, W and dg | du as rows) or across it (W and x where the sum goes
// over their rows): the first kind is read from LDS as 16-byte pieces, the second
// four rows at a time by the transposing read.  The forward product takes the same
// columns of both factors into one tile, so that the activation and the product are
// its epilogue and the two factors leave the chip only where the gradient needs
// them.  Three kernels: large bf16 products in tiles of 256 x 256 straight into LDS;
// any product in tiles of 128 x 128 through registers; the forward product of up to
// 256 rows straight from memory.  Where the tiles are too few for the device the sum is
// split over work-groups, whose fp32 parts another launch adds in order.
//
// fp32 values multiply as three bf16 terms each, six products of them (wm_split.h),
// split once on their way into LDS: 2.4 times the rate of the fp32 instructions, with
// errors below theirs.
//
// Bound by the matrix unit from some hundred rows on, and there by power: the clock
// falls as instructions are saved.  Measured, the least and the mean of twelve calls one
// after the other, 65536 rows, D 1024, F 2816 bf16: outputs and what is saved 860 and 907
// us (880 and 830 TFLOP/s), dg | du 455 and 461 (4.8 TB/s), dx 615 and 683 (1230 and
// 1110), dW 703 and 766 (1080 and 990) and 32 for its sums; a library's plain products of
// these sizes took 703, 727 and 1067 us.  D 512, F 1408 fp32: 1067 and 1152, 358 and 367,
// 963 and 1033, 1144 and 1241 us (152 to 196 TFLOP/s; the library's 1455, 1495 and 2257).
// 16 rows, D 1024, F 2816 bf16 5.4 us, W at 2.1 TB/s: launch and first loads.
//
// Registers: the large tiles of dx spill 12, and fp32 products of rows more than 2^20
// elements apart up to 62; the others none.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_attend.h"
#include "wm_profile.h"
#include "wm_split.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;  // outputs of a tile in each direction

template <typename DT> struct El;
template <> struct El<float> {
  static constexpr int VEC = 4, BK = 32;
};
template <> struct El<bf16_t> {
  static constexpr int VEC = 8, BK = 64;
};

// One operand: rows of `ld` elements.  Along k: row i of the tile is output i,
// columns are k.  Across: row k, columns are outputs.
struct Operand {
  const void* p;
  long ld;
};

// How a tile lies in LDS: in the operands' type, or, SPLIT, fp32 values as three
// planes of bf16 terms (wm_split.h).
template <typename DT, bool SPLIT> struct Kind;
template <> struct Kind<bf16_t, false> {
  typedef bf16_t T;
  static constexpr int PLANES = 1, SL = 32, ALONG = 16, ACROSS = 16;  // SL: k of a fragment; what pads a row
  typedef uint4 Frag;
};
template <> struct Kind<float, false> {
  typedef float T;
  static constexpr int SL = 16, ALONG = 4, ACROSS = 8, PLANES [[maybe_unused]] = 1;
  typedef uint4 Frag;
};
template <> struct Kind<float, true> {
  typedef bf16_t T;
  static constexpr int PLANES = 3, SL = 32, ALONG = 8, ACROSS = 16;
  typedef Split3 Frag;
};

// A tile's 128 outputs x BK of one operand, from memory through registers into LDS.
template <typename DT, bool ACROSS>
struct Stage {
  static constexpr int V = El<DT>::VEC, BK = El<DT>::BK;
  static constexpr int ROWS = ACROSS ? BK : kTile, COLS = ACROSS ? kTile : BK;
  static constexpr int N = ROWS * (COLS / V) / kThreads;
  template <bool SPLIT>
  static constexpr int pitch() { return COLS + (ACROSS ? Kind<DT, SPLIT>::ACROSS : Kind<DT, SPLIT>::ALONG); }
  template <bool SPLIT>
  static constexpr int bytes() { return Kind<DT, SPLIT>::PLANES * ROWS * pitch<SPLIT>() * (int)sizeof(typename Kind<DT, SPLIT>::T); }
  v4u r[N];
  int left;  // of k, when they were loaded
  // fp32 rows lie on the 4 bytes that range-checked loads need: where they are near enough
  // for 32-bit offsets, a piece takes one instruction, with none for its address
  uint32_t off[N];
  const DT* at;
  uint32_t size;
  __device__ __forceinline__ void aim(const Operand& a, long o0, long o1, int split, long outs, long K, long k0) {
    const DT* p = reinterpret_cast<const DT*>(a.p);
    const bool both = split < kTile;
    at = ACROSS ? p + k0 * a.ld + o0 : both ? p : p + o0 * a.ld;
    size = (uint32_t)(ACROSS ? min(outs - o0, (long)kTile) * 4 : (((both ? 2 * outs : min(outs - o0, (long)kTile)) - 1) * a.ld + K) * 4);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = threadIdx.x + i * kThreads, row = q / (COLS / V), col = q % (COLS / V) * V;
      if constexpr (ACROSS) {
        off[i] = (uint32_t)((row * a.ld + col) * 4);
      } else {
        const int in = row < split ? row : row - split;
        const long o = both ? (row < split ? o0 + row : o1 + in) : row;
        off[i] = o0 + in < outs ? (uint32_t)((o * a.ld + k0 + col) * 4) : kOffNone;
      }
    }
  }
  // the next BK, of which `left` are there
  __device__ __forceinline__ void fetch(const Operand& a, long left) {
    const rsrc_t rs = uniform_rsrc(at, ACROSS ? (uint32_t)((min(left, (long)BK) - 1) * a.ld * 4) + size : size);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint4 v = bload16(rs, off[i]);
      r[i] = v4u{v.x, v.y, v.z, v.w};
      if constexpr (!ACROSS) off[i] = off[i] == kOffNone ? kOffNone : off[i] + BK * 4;
    }
    if constexpr (ACROSS) {
      at += BK * a.ld;
    } else if (left < BK) {  // the end of k, where a row goes on with something else
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int col = (threadIdx.x + i * kThreads) % (COLS / V) * V;
#pragma unroll
        for (int e = 0; e < V; ++e) r[i][e] = col + e < left ? r[i][e] : 0u;
      }
    }
  }
  // outputs [o0, o0 + 128) of `outs`, k [k0, k0 + BK) up to kend; `split` rows of the
  // tile on, outputs count from o1 (the other factor's columns).  What lies behind the
  // end of a row is read as its last 16 bytes, and rows behind the last as that one,
  // without a branch, and put right by settle before it is stored: a branch at each
  // load would make each wait for the one before (8192 rows, D 1001, F 2811 bf16 263 -> 239 us, gradient 1132 -> 507).
  __device__ __forceinline__ void load(const Operand& a, long o0, long o1, int split, long outs, long k0, long kend) {
    const DT* p = reinterpret_cast<const DT*>(a.p);
    left = (int)min(kend - k0, (long)BK);
    const long width = ACROSS ? outs : kend, most = outs - 1 - o0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = threadIdx.x + i * kThreads, row = q / (COLS / V), col = q % (COLS / V) * V;
      const DT* const at = ACROSS ? p + (k0 + min(row, left - 1)) * a.ld
                                  : p + (row < split ? o0 + min((long)row, most) : o1 + min((long)(row - split), most)) * a.ld;
      const long c = (ACROSS ? o0 : k0) + col;
      r[i] = width < V ? load_piece<DT>(at, c, width) : *reinterpret_cast<const typename Mem16<DT>::type*>(at + min(c, width - V));
    }
  }
  // the pieces that load was to give; outputs that do not exist keep what they have
  __device__ __forceinline__ void settle(long o0, long outs, long kend) {
    const long over = ACROSS ? o0 + kTile - outs : BK - left;  // how far the tile goes beyond its rows' end
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = threadIdx.x + i * kThreads, row = q / (COLS / V), col = q % (COLS / V) * V;
      if (over > 0 && (ACROSS ? outs : kend) >= V) {
        const int past = col + V - ((ACROSS ? kTile : BK) - (int)over);
        if (past > 0) r[i] = past < V ? elements_from<DT>(r[i], past) : v4u{0, 0, 0, 0};
      }
      if (ACROSS && left < BK && row >= left) r[i] = v4u{0, 0, 0, 0};
    }
  }
  template <bool SPLIT>
  __device__ __forceinline__ void store(char* lds) const {
    typedef typename Kind<DT, SPLIT>::T T;
    T* const t = reinterpret_cast<T*>(lds);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int q = threadIdx.x + i * kThreads;
      T* const p = t + q / (COLS / V) * pitch<SPLIT>() + q % (COLS / V) * V;
      if constexpr (SPLIT) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(r[i][e]);
        constexpr int plane = ROWS * pitch<SPLIT>();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          const v2u h = {pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3])};
          *reinterpret_cast<v2u*>(p + k * plane) = h;
          x[0] -= __uint_as_float(h.x << 16);
          x[1] -= __uint_as_float(h.x & 0xffff0000u);
          x[2] -= __uint_as_float(h.y << 16);
          x[3] -= __uint_as_float(h.y & 0xffff0000u);
        }
      } else {
        *reinterpret_cast<v4u*>(p) = r[i];
      }
    }
  }
  // the fragment of sixteen outputs from o on, k from k on
  template <bool SPLIT>
  __device__ __forceinline__ static typename Kind<DT, SPLIT>::Frag frag(const char* lds, int o, int k) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
    constexpr int P = pitch<SPLIT>();
    if constexpr (sizeof(typename Kind<DT, SPLIT>::T) == 4) {
      const float* const t = reinterpret_cast<const float*>(lds);
      if constexpr (!ACROSS) return *reinterpret_cast<const uint4*>(t + (o + j) * P + k + 4 * g);
      const float* const p = t + (k + 4 * g) * P + o + j;
      return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[P]), __float_as_uint(p[2 * P]), __float_as_uint(p[3 * P]));
    } else {
      const bf16_t* const t = reinterpret_cast<const bf16_t*>(lds);
      auto one = [&](int plane) {
        const bf16_t* const q = t + plane * ROWS * P;
        if constexpr (!ACROSS) return *reinterpret_cast<const uint4*>(q + (o + j) * P + k + 8 * g);
        const bf16_t* const p = q + (k + 8 * g + j / 4) * P + o + 4 * (j % 4);
        const v2u a = read_tr(p), b = read_tr(p + 4 * P);
        return make_uint4(a.x, a.y, b.x, b.y);
      };
      if constexpr (SPLIT)
        return Split3{__builtin_bit_cast(bf16x8, one(0)), __builtin_bit_cast(bf16x8, one(1)), __builtin_bit_cast(bf16x8, one(2))};
      else
        return one(0);
    }
  }
};

// act(g) and its derivative.  fp32: to full precision.  bf16, whose results are rounded
// to 2^-9 of their value: sigmoid(g) from the hardware's exponential and reciprocal, off
// by some 10^-7 of itself times |g|, and the normal distribution function by the formula
// 7.1.26 of Abramowitz and Stegun's handbook, off by at most 10^-7 absolutely; of the
// time of a tile of 256 x 256 with D 1024, the precise ones took a fifth.
template <typename DT>
__device__ __forceinline__ float2 activate(int act, float g) {
  constexpr bool F32 = sizeof(DT) == 4;
  if (act == WM_ACT_SILU) {
    if constexpr (F32) {
      // (sigmoid(g), sigmoid(-g)); beyond kGateMost the smaller is 0 to any product's precision
      const float n = fabsf(g);
      const float2 s = gate_pair_of(g, n > kGateMost ? 0.0f : gate_exp_small(n));
      return make_float2(g * s.x, s.x * fmaf(g, s.y, 1.0f));
    } else {
      const float s = fsigmoid(g);
      return make_float2(g * s, s * fmaf(g, 1.0f - s, 1.0f));
    }
  }
  const float density = fexp(-0.5f * g * g);
  float c;
  if constexpr (F32) {
    c = 0.5f * erfcf(g * -0.70710678118654752f);
    return make_float2(g * c, fmaf(g * 0.39894228040143268f, expf(-0.5f * g * g), c));
  } else {
    // with x = |g| / sqrt 2, t = 1 / (1 + 0.3275911 x): erfc(x) = (a1 t + .. + a5 t^5) e^(-x^2)
    const float t = frcp(fmaf(fabsf(g), 0.3275911f * 0.70710678118654752f, 1.0f));
    const float tail = 0.5f * density * t *
                       fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    c = g < 0.0f ? tail : 1.0f - tail;
    return make_float2(g * c, fmaf(g * 0.39894228040143268f, density, c));
  }
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
  void* saved;      // GLU: the factors for the gradient, or null
  int act;
  float* part;      // splits > 1: [splits][M][N]
  int splits;
  long per;         // k of a split, a multiple of BK
  long tiles_m, tiles_n;
};

// Four outputs of each of two neighbouring blocks of sixteen columns, of row m: a lane
// holds columns 4 g .. + 3 of both, and stores them where n, the first block's first
// column, says.  bf16 lanes first trade halves with the lanes of the next sixteen, so
// that each has eight columns in a row of one block, 16 bytes to store in place of
// two times 8.
template <typename DT>
__device__ __forceinline__ void store_blocks(DT* row, long n, long width, int g, f32x4 x, f32x4 y) {
  if constexpr (sizeof(DT) == 4) {
    const float u[4] = {x[0], x[1], x[2], x[3]}, v[4] = {y[0], y[1], y[2], y[3]};
    store4(row, n + 4 * g, width, u);
    store4(row, n + 16 + 4 * g, width, v);
  } else {
    const auto p = __builtin_amdgcn_permlane16_swap(pack2_bf16(x[0], x[1]), pack2_bf16(y[0], y[1]), false, false);
    const auto q = __builtin_amdgcn_permlane16_swap(pack2_bf16(x[2], x[3]), pack2_bf16(y[2], y[3]), false, false);
    const v4u r = {p[0], q[0], p[1], q[1]};
    const long c = n + 16 * (g & 1) + 8 * (g >> 1);
    if (c + 8 <= width) {
      *reinterpret_cast<v4u_2*>(row + c) = r;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < width) row[c + e] = (bf16_t)(r[e / 2] >> (16 * (e & 1)));
    }
  }
}
// What the gradient needs of the two factors, [rows, 2F]: fp32 values as they are; of
// bf16 calls the upper 24 bits of the fp32 sums, as 16 in one plane and 8 in another:
// rounded to bf16 they would put as much error into dx and dW as the rounding of these
// themselves (2-norm of the error against the result 0.0030, with 24 bits 0.0024; 0.0017
// is the outputs' own rounding).
size_t low_plane(long rows, long F) { return ((size_t)rows * 2 * F * 2 + 255) / 256 * 256; }
__device__ __forceinline__ char* low_of(void* saved, long rows, long F) {
  return reinterpret_cast<char*>(saved) + (rows * 2 * F * 2 + 255) / 256 * 256;
}
typedef uint32_t __attribute__((aligned(1))) u32_1;
typedef v2u __attribute__((aligned(1))) v2u_1;
// the upper halves of two, and the third bytes of four
__device__ __forceinline__ uint32_t upper2(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ uint32_t third4(f32x4 v) {
  const uint32_t a = __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x0c0c0501u);
  const uint32_t b = __builtin_amdgcn_perm(__float_as_uint(v[3]), __float_as_uint(v[2]), 0x05010c0cu);
  return a | b;
}
template <typename DT>
__device__ __forceinline__ void save_blocks(void* saved, long rows, long F, long m, long n, long width, int g, f32x4 x, f32x4 y) {
  if constexpr (sizeof(DT) == 4) {
    store_blocks(reinterpret_cast<float*>(saved) + m * 2 * F, n, width, g, x, y);
  } else {
    const auto p = __builtin_amdgcn_permlane16_swap(upper2(x[0], x[1]), upper2(y[0], y[1]), false, false);
    const auto q = __builtin_amdgcn_permlane16_swap(upper2(x[2], x[3]), upper2(y[2], y[3]), false, false);
    const auto t = __builtin_amdgcn_permlane16_swap(third4(x), third4(y), false, false);
    const long c = n + 16 * (g & 1) + 8 * (g >> 1);
    bf16_t* const hi = reinterpret_cast<bf16_t*>(saved) + m * 2 * F;
    char* const lo = low_of(saved, rows, F) + m * 2 * F;
    const v4u r = {p[0], q[0], p[1], q[1]};
    const v2u l = {t[0], t[1]};
    if (c + 8 <= width) {
      *reinterpret_cast<v4u_2*>(hi + c) = r;
      *reinterpret_cast<v2u_1*>(lo + c) = l;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < width) {
          hi[c + e] = (bf16_t)(r[e / 2] >> (16 * (e & 1)));
          lo[c + e] = (char)(l[e / 4] >> (8 * (e & 3)));
        }
    }
  }
}
template <typename DT>
__device__ __forceinline__ void put_glu(const ProductArgs& a, long m, long n, int g, const f32x4 (&gate)[2], const f32x4 (&up)[2]) {
  f32x4 h[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) h[i][e] = activate<DT>(a.act, gate[i][e]).x * up[i][e];
  store_blocks(reinterpret_cast<DT*>(a.out) + m * a.out_ld, n, a.N, g, h[0], h[1]);
  if (a.saved) {
    save_blocks<DT>(a.saved, a.M, a.N, m, n, a.N, g, gate[0], gate[1]);
    save_blocks<DT>(a.saved, a.M, a.N, m, a.N + n, 2 * a.N, g, up[0], up[1]);
  }
}
template <typename DT>
__device__ __forceinline__ void put(const ProductArgs& a, int split, long m, long n, int g, f32x4 x, f32x4 y) {
  if (a.splits > 1)
    store_blocks(a.part + ((long)split * a.M + m) * a.N, n, a.N, g, x, y);
  else
    store_blocks(reinterpret_cast<DT*>(a.out) + m * a.out_ld, n, a.N, g, x, y);
}

// Columns n .. + 3 alone.
template <typename DT>
__device__ __forceinline__ void put_one(const ProductArgs& a, long m, long n, f32x4 gate, f32x4 up) {
  float h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = activate<DT>(a.act, gate[e]).x * up[e];
  store4(reinterpret_cast<DT*>(a.out) + m * a.out_ld, n, a.N, h);
  if (!a.saved) return;
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const f32x4 v = f ? up : gate;
    if constexpr (sizeof(DT) == 4) {
      const float x[4] = {v[0], v[1], v[2], v[3]};
      store4(reinterpret_cast<float*>(a.saved) + m * 2 * a.N + f * a.N, n, a.N, x);
    } else {
      bf16_t* const hi = reinterpret_cast<bf16_t*>(a.saved) + m * 2 * a.N + f * a.N;
      char* const lo = low_of(a.saved, a.M, a.N) + m * 2 * a.N + f * a.N;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) {
          hi[n + e] = (bf16_t)(__float_as_uint(v[e]) >> 16);
          lo[n + e] = (char)(__float_as_uint(v[e]) >> 8);
        }
    }
  }
}

// Any sizes, strides and alignments: tiles of 128 x 128, four waves of 64 x 64,
// the next k's pieces on their way in registers.
template <typename DT, bool PX, bool QX, bool GLU, bool NEAR>
__global__ void __launch_bounds__(kThreads, 2) k_product(const ProductArgs a) {
  typedef Stage<DT, PX> SP;
  typedef Stage<DT, QX> SQ;
  constexpr int BK = El<DT>::BK;
  constexpr bool F32 = sizeof(DT) == 4;
  constexpr int PB = SP::template bytes<F32>(), QB = SQ::template bytes<F32>();
  __shared__ __align__(16) char lds[PB + QB];
  char *const pl = lds, *const ql = lds + PB;
  const int w = threadIdx.x >> 6, wp = w & 1, wq = w >> 1, lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const long tile = blockIdx.x / a.splits;
  const int split = (int)(blockIdx.x % a.splits);
  const long n0 = tile % a.tiles_n * (GLU ? kTile / 2 : kTile), m0 = tile / a.tiles_n * kTile;
  const long k0 = split * a.per, k1 = min(k0 + a.per, a.K);

  f32x4 acc[4][4];  // [block of Q][block of P]
  // where this wave's blocks of P start in the tile: half a tile together, or 32 outputs of both factors
  auto block = [&](int i) { return GLU ? 64 * (i >> 1) + 32 * wp + 16 * (i & 1) : 64 * wp + 16 * i; };
  const int half = GLU ? kTile / 2 : kTile;
  SP sp;
  SQ sq;
  // sums of the wave's blocks of Q from l0 on
  auto run = [&](auto split_terms, auto& acc, int l0) {
    constexpr bool SPLIT = decltype(split_terms)::value;
    constexpr int L = sizeof(acc) / sizeof(acc[0]);
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto load = [&](long k) {
      if constexpr (NEAR) {
        sp.fetch(a.P, k1 - k);
        sq.fetch(a.Q, k1 - k);
      } else {
        sp.load(a.P, n0, a.N + n0, half, a.N, k, k1);
        sq.load(a.Q, m0, 0, kTile, a.M, k, k1);
      }
    };
    if constexpr (NEAR) {
      sp.aim(a.P, n0, a.N + n0, half, a.N, a.K, k0);
      sq.aim(a.Q, m0, 0, kTile, a.M, a.K, k0);
    }
    if (k0 < k1) load(k0);
    for (long k = k0; k < k1; k += BK) {
      __syncthreads();
      if constexpr (!NEAR) {
        sp.settle(n0, a.N, k1);
        sq.settle(m0, a.M, k1);
      }
      sp.template store<SPLIT>(pl);
      sq.template store<SPLIT>(ql);
      __syncthreads();
      if (k + BK < k1) load(k + BK);
#pragma unroll
      for (int s = 0; s < BK; s += Kind<DT, SPLIT>::SL) {
        typename Kind<DT, SPLIT>::Frag p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = SP::template frag<SPLIT>(pl, block(i), s);
#pragma unroll
        for (int l = 0; l < L; ++l) {
          const auto q = SQ::template frag<SPLIT>(ql, 64 * wq + 16 * (l0 + l), s);
          if constexpr (SPLIT) {
            mfma_split(acc[l], p, q);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) Mfma<DT>::step(acc[l][i], p[i], q);
          }
        }
      }
    }
  };
  run(std::integral_constant<bool, F32>(), acc, 0);
  if constexpr (F32) {
    // An infinity, or a value that rounds to one in bf16, leaves NaN in the sums that
    // it enters: these are taken again on the fp32 unit, a block of Q at a time.
    bool bad = false;
#pragma unroll
    for (int l = 0; l < 4; ++l)
#pragma unroll
      for (int i = 0; i < 4; ++i) bad |= any_nan(acc[l][i]);
    if (__syncthreads_or(bad)) {
#pragma unroll
      for (int l = 0; l < 4; ++l) {
        f32x4 again[1][4];
        run(std::false_type(), again, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[l][i] = nan_to(acc[l][i], again[0][i]);
      }
    }
  }

#pragma unroll
  for (int l = 0; l < 4; ++l) {
    const long m = m0 + 64 * wq + 16 * l + j;
    if (m < a.M) {
      if constexpr (GLU) {
        const f32x4 gate[2] = {acc[l][0], acc[l][1]}, up[2] = {acc[l][2], acc[l][3]};
        put_glu<DT>(a, m, n0 + 32 * wp, g, gate, up);
      } else {
        put<DT>(a, split, m, n0 + block(0), g, acc[l][0], acc[l][1]);
        put<DT>(a, split, m, n0 + block(2), g, acc[l][2], acc[l][3]);
      }
    }
  }
}

// bf16 with rows on 16-byte boundaries: tiles of 256 x 256, eight waves of 128 x 64,
// k 64 at a time straight from memory into one of two buffers in LDS.  A wave's load
// is 1 KB in a row, so that padding cannot keep rows apart; the order of a row's
// 16-byte pieces is changed instead, by the row's number, so that the lanes of one
// read find different banks.  The products of one half of a step's k run while the
// next half's operands are read from LDS; the one barrier of a step stands between
// its halves, where all of its operands are read and its buffer takes the pieces of
// the step after the next.  A work-group takes tile after tile, and its loads run on
// into the next one, so that a tile's stores are beside the next one's products.
constexpr int kBigGroups = 256;  // one a CU
constexpr int kBig = 256, kBigThreads = 512, kBigK = 64, kBigBytes = kBig * kBigK * 2;
constexpr int kBigLoads = 8;  // of a wave in a step, four for each operand
__device__ __forceinline__ int turn_along(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int turn_across(int row) { return ((row & 3) | ((row >> 1) & 4)) << 1; }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

template <bool ACROSS, bool GLU>
struct Direct {
  uint32_t off[4];  // per lane: where its piece of each of this wave's four loads lies
  uint32_t lo, hi, bytes, row;  // the resource, and the bytes that a step of k moves it by (ACROSS)
  // outputs [o0, o0 + 256) of `outs`, GLU: 128 of each factor; k from k0 on
  __device__ __forceinline__ void set(const Operand& a, long o0, long outs, long K, long k0, int wave, int lane) {
    const bf16_t* p = reinterpret_cast<const bf16_t*>(a.p);
    long size;
    if constexpr (ACROSS) {
      p += k0 * a.ld + o0;
      // of the last row, in whole dwords: one that reaches over the end would be read as 0, and
      // with it an odd row's last value.  The half behind it lies in the row's own 16 bytes and
      // belongs to an output that does not exist.
      size = (min(outs - o0, (long)kBig) + 1) / 2 * 4;
    } else if constexpr (GLU) {
      size = ((2 * outs - 1) * a.ld + K) * 2;
    } else {
      p += o0 * a.ld;
      size = ((min(outs - o0, (long)kBig) - 1) * a.ld + K) * 2;
    }
    // (the same in every lane, which the compiler does not see through the tile's divisions)
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    lo = uniform((uint32_t)at);
    hi = uniform((uint32_t)(at >> 32));
    bytes = uniform((uint32_t)size);
    row = (uint32_t)(a.ld * 2);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int q = 4 * wave + t;
      if constexpr (ACROSS) {
        const int r = 2 * q + (lane >> 5), c = (lane & 31) ^ turn_across(r);
        off[t] = (uint32_t)((r * a.ld + 8 * c) * 2);
      } else {
        const int r = 8 * q + (lane >> 3), c = (lane & 7) ^ turn_along(r), in = GLU ? r & 127 : r;
        const long at = GLU ? (r < 128 ? o0 + in : outs + o0 + in) : r;
        off[t] = o0 + in < outs ? (uint32_t)((at * a.ld + 8 * c + k0) * 2) : kOffNone;
      }
    }
  }
  // the pieces of the next step, which has `left` of k, into LDS
  __device__ __forceinline__ void issue(uint32_t lds, int left, int wave, int lane) {
    u32x4 rs;
    rs.x = uniform(lo);
    rs.y = uniform(hi & 0xffffu);
    rs.z = uniform(ACROSS ? (uint32_t)(min(left, kBigK) - 1) * row + bytes : bytes);
    rs.w = 0x00020000u;
    lds = uniform(lds);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t o = off[t];
      if (left < kBigK) {  // the end of k: zeros from there on
        const int r = ACROSS ? 2 * (4 * wave + t) + (lane >> 5) : 8 * (4 * wave + t) + (lane >> 3);
        if ((ACROSS ? r : 8 * ((lane & 7) ^ turn_along(r))) >= left) o = kOffNone;
      }
      dma16(rs, o, lds + (uint32_t)(4 * wave + t) * 1024u);
      if (!ACROSS) off[t] = off[t] == kOffNone ? kOffNone : off[t] + kBigK * 2;
    }
    if (ACROSS) {
      const uint64_t at = ((uint64_t)hi << 32 | lo) + (uint64_t)kBigK * row;
      lo = (uint32_t)at;
      hi = (uint32_t)(at >> 32);
    }
  }
  // the fragment of sixteen outputs from o on, half s of the step's k
  __device__ __forceinline__ static uint4 frag(const char* lds, int o, int s) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
    if constexpr (!ACROSS) {
      return *reinterpret_cast<const uint4*>(lds + (o + j) * (kBigK * 2) + (((4 * s + g) ^ turn_along(j)) << 4));
    } else {
      const int row = 32 * s + 8 * g + j / 4;
      const char* const p = lds + row * (kBig * 2) + (((o / 8) ^ turn_across(row)) << 4) + 8 * (j % 4);
      const v2u a = read_tr(reinterpret_cast<const bf16_t*>(p)), b = read_tr(reinterpret_cast<const bf16_t*>(p + 4 * kBig * 2));
      return make_uint4(a.x, a.y, b.x, b.y);
    }
  }
};

template <bool PX, bool QX, bool GLU>
__global__ void __launch_bounds__(kBigThreads) k_product_big(const ProductArgs a) {
  __shared__ __align__(1024) char lds[4 * kBigBytes];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = w & 3, wq = w >> 2;
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  // the XCDs take work-groups in turn: each gets a run of tiles, eight rows of tiles at a time
  const uint32_t tiles_m = (uint32_t)a.tiles_m, tiles_n = (uint32_t)a.tiles_n, tiles = tiles_m * tiles_n;
  const uint32_t all = tiles * (uint32_t)a.splits, xcd = blockIdx.x % 8, run8 = all / 8, extra = all % 8;
  const uint32_t end = (xcd + 1) * run8 + min(xcd + 1, extra), stride = gridDim.x / 8;
  struct Tile {
    uint32_t at;
    long m0, n0;
    int split, left;  // what is left of its k
    long k0;
  };
  auto tile_at = [&](uint32_t i) {
    Tile t;
    t.at = i;
    t.split = (int)(i / tiles);
    const uint32_t n = i - t.split * tiles, band = n / (8 * tiles_n), high = min(8u, tiles_m - 8 * band);
    const uint32_t in = n - band * 8 * tiles_n;
    t.m0 = (long)(8 * band + in % high) * kBig;
    t.n0 = (long)(in / high) * (GLU ? kBig / 2 : kBig);
    t.k0 = t.split * a.per;
    t.left = (int)uniform((uint32_t)(min(t.k0 + a.per, a.K) - t.k0));
    return t;
  };
  const uint32_t begin = xcd * run8 + min(xcd, extra) + blockIdx.x / 8;
  if (begin >= end) return;
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
  auto block = [&](int i) { return GLU ? 128 * (i >> 1) + 32 * wp + 16 * (i & 1) : 64 * wp + 16 * i; };

  // the loads' own place among the tiles, two steps ahead of the products'
  Tile ahead = tile_at(begin);
  Tile now = ahead;
  bool more = true;
  Direct<PX, GLU> dp;
  Direct<QX, false> dq;
  auto aim = [&]() {
    dp.set(a.P, ahead.n0, a.N, a.K, ahead.k0, w, lane);
    dq.set(a.Q, ahead.m0, a.M, a.K, ahead.k0, w, lane);
  };
  auto issue = [&](int buf) {
    const uint32_t to = lds0 + (uint32_t)buf * 2 * kBigBytes;
    dp.issue(to, ahead.left, w, lane);
    dq.issue(to + kBigBytes, ahead.left, w, lane);
    ahead.left -= kBigK;
    if (ahead.left <= 0) {
      more = ahead.at + stride < end;
      if (more) {
        ahead = tile_at(ahead.at + stride);
        aim();
      }
    }
  };
  // operands: Q's are read for the next half as soon as their last product is under way,
  // P's are held for both halves
  uint4 p[4], q[8];
  f32x4 acc[8][4];  // [block of Q][block of P]
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  auto half = [&](const char* from, int s) {
    uint4 next[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = Direct<PX, GLU>::frag(from, block(i), s);
#pragma unroll
    for (int l = 0; l < 8; ++l) {
#pragma unroll
      for (int i = 0; i < 4; ++i) Mfma<bf16_t>::step(acc[l][i], p[i], q[l]);
      q[l] = Direct<QX, false>::frag(from + kBigBytes, 128 * wq + 16 * l, s);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = next[i];
  };
  aim();
  issue(0);
  const bool second = more;
  if (second) issue(1);
  if (second)
    vm_wait<kBigLoads>();
  else
    vm_wait<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = Direct<PX, GLU>::frag(lds, block(i), 0);
#pragma unroll
  for (int l = 0; l < 8; ++l) q[l] = Direct<QX, false>::frag(lds + kBigBytes, 128 * wq + 16 * l, 0);
  clear();
  int stores = 0;  // a whole tile's, which are younger than the loads in flight
  for (int buf = 0;; buf ^= 1) {
    const char* const here = lds + buf * 2 * kBigBytes;
    half(here, 1);
    // the next step's pieces are in LDS and this one's operands in registers, in every wave
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    if (stores == 0) vm_wait<0>();
    else if (stores == 40) vm_wait<40>();
    else if (stores == 16) vm_wait<16>();
    else if (stores == 8) vm_wait<8>();
    else vm_wait<32>();
    stores = 0;
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    if (more) issue(buf);
    // (after the last step the other buffer holds old pieces, which nothing uses)
    half(lds + (buf ^ 1) * 2 * kBigBytes, 0);
    now.left -= kBigK;
    if (now.left > 0) continue;
    // the tile is complete
#pragma unroll
    for (int l = 0; l < 8; ++l) {
      const long m = now.m0 + 128 * wq + 16 * l + j;
      if (m < a.M) {
        if constexpr (GLU) {
          const f32x4 gate[2] = {acc[l][0], acc[l][1]}, up[2] = {acc[l][2], acc[l][3]};
          put_glu<bf16_t>(a, m, now.n0 + 32 * wp, g, gate, up);
        } else {
          put<bf16_t>(a, now.split, m, now.n0 + block(0), g, acc[l][0], acc[l][1]);
          put<bf16_t>(a, now.split, m, now.n0 + block(2), g, acc[l][2], acc[l][3]);
        }
      }
    }
    // A whole tile's stores, one an instruction, are the youngest of what is in flight at the
    // next wait; of others there may be fewer, and that wait is for all.
    const bool whole = now.m0 + kBig <= a.M && now.n0 + (GLU ? kBig / 2 : kBig) <= a.N;
    stores = !whole ? 0 : GLU ? (a.saved ? 40 : 8) : a.splits > 1 ? 32 : 16;
    if (now.at + stride >= end) return;
    now = tile_at(now.at + stride);
    clear();
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

template <typename DT>
__device__ __forceinline__ void unpack(v4u r, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(DT) == 4) {
      v[i] = __uint_as_float(r[i]);
    } else {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
}
template <typename DT>
__device__ __forceinline__ void store_piece(DT* row, long c, long width, const float* v) {
  constexpr int V = El<DT>::VEC;
  if (c + V <= width) {
    v4u r;
    if constexpr (sizeof(DT) == 4)
      r = v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else
      r = v4u{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
    *reinterpret_cast<typename Mem16<DT>::type*>(row + c) = r;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (c + e < width) DType<DT>::store(row, c + e, v[e]);
  }
}

// Up to 256 rows, where the tiles are few and the time is that of reading W: a work-group
// takes sixteen columns of both factors for up to 64 rows, its eight waves a share of k each, straight from memory
// into matrix operands, kFewAhead slices on their way at a time; the waves' sums are
// added in LDS in order.  Measured so and in tiles, D 1024, F 2816: bf16 16 rows 5.1 and
// 19.2 us, 64 rows 8.2 and 21.1, 128 rows 15.5 and 21.8, 256 rows 22.8 and 22.4, 512 rows
// 44 and 23; fp32 10 and 57, 20 and 59, 39 and 60, 57 and 61, 109 and 63; D 256, F 640 bf16,
// 256 rows 4.3 and 8.7.
constexpr int kFewRows = 256, kFewWaves = 8, kFewAhead = 4;
template <typename DT, int MB>
__global__ void __launch_bounds__(64 * kFewWaves) k_glu_few(const ProductArgs a) {
  constexpr int V = El<DT>::VEC, SL = 4 * V;
  __shared__ f32x4 sum[kFewWaves][2 * MB][64];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const long n0 = (long)blockIdx.x * 16, m0 = (long)blockIdx.y * 64;
  const DT* const W = reinterpret_cast<const DT*>(a.P.p);
  const DT* const pg = W + min(n0 + j, a.N - 1) * a.P.ld;
  const DT* const pu = pg + a.N * a.P.ld;
  const DT* px[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) px[m] = reinterpret_cast<const DT*>(a.Q.p) + min(m0 + 16 * m + j, a.M - 1) * a.Q.ld;
  f32x4 acc[2][MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) acc[0][m] = acc[1][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  // slices of k in runs of kFewAhead, dealt to the waves in turn
  const long slices = (a.K + SL - 1) / SL;
  for (long s0 = (long)w * kFewAhead; s0 < slices; s0 += kFewWaves * kFewAhead) {
    v4u rg[kFewAhead], ru[kFewAhead], rx[kFewAhead][MB];
#pragma unroll
    for (int t = 0; t < kFewAhead; ++t) {
      const long k = (s0 + t) * SL + V * g;
      rg[t] = load_piece<DT>(pg, k, a.K);
      ru[t] = load_piece<DT>(pu, k, a.K);
#pragma unroll
      for (int m = 0; m < MB; ++m) rx[t][m] = load_piece<DT>(px[m], k, a.K);
    }
#pragma unroll
    for (int t = 0; t < kFewAhead; ++t)
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const uint4 x = make_uint4(rx[t][m].x, rx[t][m].y, rx[t][m].z, rx[t][m].w);
        Mfma<DT>::step(acc[0][m], make_uint4(rg[t].x, rg[t].y, rg[t].z, rg[t].w), x);
        Mfma<DT>::step(acc[1][m], make_uint4(ru[t].x, ru[t].y, ru[t].z, ru[t].w), x);
      }
  }
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    sum[w][2 * m][lane] = acc[0][m];
    sum[w][2 * m + 1][lane] = acc[1][m];
  }
  __syncthreads();
  for (int m = w; m < MB; m += kFewWaves) {
    f32x4 gate = sum[0][2 * m][lane], up = sum[0][2 * m + 1][lane];
#pragma unroll
    for (int k = 1; k < kFewWaves; ++k) {
      gate += sum[k][2 * m][lane];
      up += sum[k][2 * m + 1][lane];
    }
    if (m0 + 16 * m + j < a.M) put_one<DT>(a, m0 + 16 * m + j, n0 + 4 * g, gate, up);
  }
}

// A piece of one factor of a row.
template <typename DT>
__device__ __forceinline__ void saved_piece(const void* saved, long rows, long F, long row, int f, int c, float* v) {
  if constexpr (sizeof(DT) == 4) {
    unpack<float>(load_piece<float>(reinterpret_cast<const float*>(saved) + row * 2 * F + f * F, c, F), v);
  } else {
    const v4u hi = load_piece<bf16_t>(reinterpret_cast<const bf16_t*>(saved) + row * 2 * F + f * F, c, F);
    const char* const lo = low_of(const_cast<void*>(saved), rows, F) + row * 2 * F + f * F;
    v2u l;
    if (c + 8 <= F) {
      l = *reinterpret_cast<const v2u_1*>(lo + c);
    } else {
      uint8_t b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = (uint8_t)lo[min(c + e, (int)F - 1)];
      l = v2u{b[0] | b[1] << 8 | b[2] << 16 | (uint32_t)b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | (uint32_t)b[7] << 24};
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t h = e & 1 ? hi[e / 2] & 0xffff0000u : hi[e / 2] << 16;
      v[e] = __uint_as_float(h | ((l[e / 4] >> (8 * (e & 3))) & 255u) << 8);
    }
  }
}
// One piece of a row.
template <typename DT>
__device__ __forceinline__ void back_piece(const GluGradArgs& a, DT* dpre, long row, int c) {
  constexpr int V = El<DT>::VEC;
  float g[V], u[V], d[V];
  const v4u rd = load_piece<DT>(reinterpret_cast<const DT*>(a.dh) + row * a.dh_ld, c, a.F);
  saved_piece<DT>(a.saved, a.rows, a.F, row, 0, c, g);
  saved_piece<DT>(a.saved, a.rows, a.F, row, 1, c, u);
  unpack<DT>(rd, d);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float2 v = activate<DT>(a.act, g[e]);
    g[e] = d[e] * u[e] * v.y;
    u[e] = d[e] * v.x;
  }
  DT* out = dpre + row * 2 * a.F;
  store_piece(out, c, a.F, g);
  store_piece(out + a.F, c, a.F, u);
}

constexpr long kBackGroups = 4096;
// dpre [rows, 2F] from the factors and dh: 16 bytes of a row a lane.
template <typename DT>
__global__ void __launch_bounds__(kThreads) k_glu_back(const GluGradArgs a, DT* dpre) {
  constexpr int V = El<DT>::VEC;
  const uint32_t parts = (uint32_t)(a.F + V - 1) / V;
  const long pieces = a.rows * (long)parts, step = (long)gridDim.x * kThreads;
  long at = (long)blockIdx.x * kThreads + threadIdx.x;
  // row and piece advance by the stride's own
  long row = at / parts;
  uint32_t p = (uint32_t)(at % parts);
  const long step_row = step / parts;
  const uint32_t step_p = (uint32_t)(step % parts);
  for (; at < pieces; at += step, row += step_row, p += step_p) {
    if (p >= parts) p -= parts, ++row;
    const int c = (int)p * V;
    back_piece<DT>(a, dpre, row, c);
  }
}
// Splits of a sum of length K for M x N outputs in tiles of 128 x 128: up to 512 work-groups,
// two a CU.  Gradient with up to 256, 512 and 1024 of them, fp32: 2048 rows, D 512, F 1408
// 127, 104 and 115 us (276 without splits), 8192 rows 424, 338 and 329; 16384 rows, D 256,
// F 640 195, 181 and 202.
int splits_of(long M, long N, long K, int bk) {
  const long tiles = std::max(1L, (M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
  if (tiles >= 256) return 1;
  return (int)std::max<long>(1, std::min<long>(512 / tiles, K / (8 * bk)));
}
// The same for tiles of 256 x 256, of which 256 are under way at a time: as many as take the
// least time, in steps of the sum.  A tile's results are written in that of 6 steps,
// and the parts of 20 tiles are read and added in that of one.  Gradient, D 1024, F 2816,
// with 512 work-groups in all and so: 2048 rows 128 and 113 us, 4096 rows 196 and 172, 8192
// rows 297 and 287.
int splits_of_big(long M, long N, long K) {
  const long tiles = std::max(1L, (M + kBig - 1) / kBig) * ((N + kBig - 1) / kBig), steps = (K + kBigK - 1) / kBigK;
  if (tiles >= kBigGroups) return 1;
  int best = 1;
  long least = steps + 6;
  for (int s = 2; s <= 16 && 8 * s <= steps; ++s) {
    const long t = (tiles * s + kBigGroups - 1) / kBigGroups * ((steps + s - 1) / s + 6) + tiles * s / 20;
    if (t < least) least = t, best = s;
  }
  return best;
}
// The kernel of a product goes by its sizes: bf16 products in at least 64 tiles of
// 256 x 256 take those, the outputs' (no splits) in at least 160.  Measured in large tiles
// and in small ones, D 1024, F 2816: outputs in 88 tiles 39 and 33 us, 132 tiles 38 and 32,
// 176 tiles 39 and 49, 352 tiles 72 and 86; dW (88 tiles) over 1024 rows 33 and 32 us, 2048
// rows 52 and 52, 4096 rows 77 and 97; dx and what goes before it in 64 tiles 94 and 134.
bool big(int dtype, long M, long N, long K, bool glu) {
  return dtype == WM_BF16 && K > 0 && K % 8 == 0 && (M + kBig - 1) / kBig * ((N + kBig - 1) / kBig) >= (glu ? 160 : 64);
}
// Whether an operand's rows lie on 16-byte boundaries, and near enough for 32-bit offsets.
bool direct(const Operand& a) {
  return (reinterpret_cast<uintptr_t>(a.p) & 15) == 0 && a.ld % 8 == 0 && a.ld <= 1 << 20;
}

// A product's launch names, by the kernel that it takes.
struct Names {
  const char *few, *tiles, *big;
};

template <typename DT, bool PX, bool QX, bool GLU>
hipError_t product(const Names& name, ProductArgs a, hipStream_t s) {
  constexpr int BK = El<DT>::BK;
  const int dtype = sizeof(DT) == 4 ? WM_FP32 : WM_BF16;
  const bool wide = big(dtype, a.M, GLU ? 2 * a.N : a.N, a.K, GLU);
  if constexpr (GLU) {
    if (a.M <= kFewRows) {
      const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 63) / 64)), block(64 * kFewWaves);
      if (a.M <= 16) return launch(name.few, k_glu_few<DT, 1>, grid, block, 0, s, a);
      return launch(name.few, a.M <= 32 ? k_glu_few<DT, 2> : k_glu_few<DT, 4>, grid, block, 0, s, a);
    }
  }
  if constexpr (sizeof(DT) == 2) {
    if (wide && direct(a.P) && direct(a.Q) && (!GLU || 2 * a.N * a.P.ld < (1L << 30))) {
      const int width = GLU ? kBig / 2 : kBig;
      a.tiles_n = (a.N + width - 1) / width;
      a.tiles_m = (a.M + kBig - 1) / kBig;
      a.splits = GLU ? 1 : splits_of_big(a.M, a.N, a.K);
      a.per = ((a.K + a.splits - 1) / a.splits + kBigK - 1) / kBigK * kBigK;
      a.splits = (int)((a.K + a.per - 1) / a.per);  // none empty
      const hipError_t e = launch(name.big, k_product_big<PX, QX, GLU>, dim3(kBigGroups), dim3(kBigThreads), 0, s, a);
      if (e != hipSuccess || a.splits == 1) return e;
      return launch("glu_sum", k_product_sum<DT>, dim3((unsigned)((a.M * a.N + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
    }
  }
  const int width = GLU ? kTile / 2 : kTile;
  a.tiles_n = (a.N + width - 1) / width;
  a.tiles_m = (a.M + kTile - 1) / kTile;
  a.splits = GLU ? 1 : splits_of(a.M, a.N, a.K, BK);
  a.per = ((a.K + a.splits - 1) / a.splits + BK - 1) / BK * BK;
  const dim3 grid((unsigned)(a.tiles_m * a.tiles_n * a.splits));
  hipError_t e;
  if constexpr (sizeof(DT) == 4) {
    const bool near = a.P.ld <= 1 << 20 && a.Q.ld <= 1 << 20 && (!GLU || 2 * a.N * a.P.ld < (1L << 29));
    e = launch(name.tiles, near ? k_product<DT, PX, QX, GLU, true> : k_product<DT, PX, QX, GLU, false>, grid, dim3(kThreads), 0, s, a);
  } else {
    e = launch(name.tiles, k_product<DT, PX, QX, GLU, false>, grid, dim3(kThreads), 0, s, a);
  }
  if (e != hipSuccess || a.splits == 1) return e;
  return launch("glu_sum", k_product_sum<DT>, dim3((unsigned)((a.M * a.N + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
// What either kernel of the product needs.
size_t part_bytes(int dtype, long M, long N, long K) {
  const int s = std::max(splits_of(M, N, K, dtype == WM_FP32 ? El<float>::BK : El<bf16_t>::BK),
                         big(dtype, M, N, K, false) ? splits_of_big(M, N, K) : 1);
  return s > 1 ? (size_t)s * M * N * sizeof(float) : 0;
}

}  // namespace

hipError_t launch_glu(int dtype, const GluArgs& a, hipStream_t s) {
  const ProductArgs p{{a.W, a.D}, {a.x, a.x_ld}, a.rows, a.F, a.D, a.h, a.h_ld, a.saved, a.act, nullptr, 1, 0, 0, 0};
  const Names name{"glu/few", "glu/128", "glu/256"};
  return dtype == WM_FP32 ? product<float, false, false, true>(name, p, s) : product<bf16_t, false, false, true>(name, p, s);
}

size_t glu_saved(int dtype, long rows, int F) {
  return dtype == WM_FP32 ? (size_t)rows * 2 * F * 4 : low_plane(rows, F) + (size_t)rows * 2 * F;
}

size_t glu_grad_workspace(int dtype, long rows, int D, int F) {
  return align256((size_t)rows * 2 * F * (dtype == WM_FP32 ? 4 : 2)) +
         align256(std::max(part_bytes(dtype, rows, D, 2L * F), part_bytes(dtype, 2L * F, D, rows)));
}

hipError_t launch_glu_grad(int dtype, const GluGradArgs& a, hipStream_t s) {
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    DT* dpre = reinterpret_cast<DT*>(a.ws);
    float* part = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + align256((size_t)a.rows * 2 * a.F * sizeof(DT)));
    hipError_t e = hipSuccess;
    if (a.rows > 0) {
      const long pieces = a.rows * ((a.F + El<DT>::VEC - 1) / El<DT>::VEC);
      e = launch("glu_back", k_glu_back<DT>, dim3((unsigned)std::min<long>((pieces + kThreads - 1) / kThreads, kBackGroups)),
                 dim3(kThreads), 0, s, a, dpre);
      if (e != hipSuccess) return e;
      const ProductArgs dx{{a.W, a.D}, {dpre, 2L * a.F}, a.rows, a.D, 2L * a.F, a.dx, a.dx_ld, nullptr, 0, part, 1, 0, 0, 0};
      if ((e = product<DT, true, false, false>({nullptr, "glu_dx/128", "glu_dx/256"}, dx, s)) != hipSuccess) return e;
    }
    if (!a.dW) return e;
    const ProductArgs dw{{a.x, a.x_ld}, {dpre, 2L * a.F}, 2L * a.F, a.D, a.rows, a.dW, a.D, nullptr, 0, part, 1, 0, 0, 0};
    return product<DT, true, true, false>({nullptr, "glu_dw/128", "glu_dw/256"}, dw, s);
  };
  return dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
}

}  // namespace wm
