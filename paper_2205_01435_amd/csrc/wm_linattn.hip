// Linear attention with one decay a head, and its gradient:
//   S_t = a S_{t-1} + k_t v_t^T,  y_t = scale S_t^T q_t;
//   G_t = dL/dS_t: dq_t = scale S_t dy_t, dk_t = F_t v_t, dv_t = F_t^T k_t with
//   F_t = G_t + scale q_t dy_t^T, G_{t-1} = a F_t.
//
// All four results are one form ("mix"), of rows A, sources B and values C:
//   out_r = sum over sources s of a^|r-s| (A_r . B_s) C_s  +  a^(distance) A_r S
// with S the state that enters a chunk of 64 steps from its side:
//   y:  A = q, B = k, C = v;   dq: A = dy, B = v, C = k, S transposed;  s <= r
//   dv: A = k, B = q, C = dy;  dk: A = v, B = dy, C = q, G transposed;  s >= r.
// A chunk is three products on the matrix unit: the weights' 64 x 64 matrix
// A B^T, masked to the sources of the row's own trajectory; its product with C;
// and the state's part; then the state takes the chunk's sources in, weighted by
// what is left of them at its end.  A work-group sweeps through the chunks of one
// head with the state in registers: rows come from memory as matrix operands,
// sources through LDS, where the transposing read serves the products that sum over
// steps.  dk and dv share their sources and state, so that one reverse sweep gives
// both (heads up to 64 wide); wider heads take one sweep for each.
//
// Where sequences and heads are too few to fill the device, the time axis is split
// into segments: a first launch sums up each segment's own state, a second one runs
// through them, and the main launch starts every segment from the state that enters
// it.  The forward call's entering states are kept for dq.  A single step is a
// kernel of its own, which streams the states.
//
// The products take a source that a row does not see as 0 times its value, which is NaN
// where that is not finite.  What comes out as NaN is taken again step by step (by_steps).
//
// Precision: fp32 values multiply on the fp32 matrix instructions.  bf16 values
// enter exactly; the 64 x 64 weights and the state that meets the rows are held as
// two bf16 terms each (2^-17 of their value is left out, against the 2^-9 of the
// output's rounding), and the sources times their weights, which make up the fp32
// state, as three (2^-24).  All sums are fp32.
//
// Measured: one step of 256 x 8 states of 64 x 64 12 us (5.7 TB/s, part of it from the
// caches).  The least and the mean of twelve calls one after the other: T 128, B 512, 8
// heads of 64 fp32, padded, 151 and 160 us, gradient 367 and 397; the matrix
// unit is busy 40 % and the vector unit 30 % of it, the rest is waiting at three
// work-groups a CU.  T 32768, 16 heads of 64 bf16: states 28 and 30, through the segments
// 7, outputs 61 and 66 us; gradient 30 and 32, 8, 152 and 166; two thirds of it the vector
// unit's splits, weights and addresses.  Heads of 128, whose gradient takes three sweeps, T
// 128, B 512, 8 heads: bf16 273 us, with gradient 1085 (64: 100 and 304); fp32, one wave a
// SIMD by its 85 KB of LDS, 906 and 3642 (181 and 638).  T 32768, 16 heads of 128: 290 and
// 976, fp32 930 and 3305 (64: 89 and 274, 247 and 756).
#include <algorithm>

#include "../../include/wm.h"
#include "wm_attend.h"
#include "wm_profile.h"
#include "wm_split.h"

namespace wm {
namespace {

constexpr int kChunk = 64;
__host__ __device__ constexpr int chunks_of(int T) { return T / kChunk + (T % kChunk != 0); }
constexpr int kThreads = 256;  // four waves, 16 of a chunk's rows each

struct MixArgs {
  int T, B, N;
  int ka, kc;  // widths of A and B, and of C and the output
  SeqView a, b, c, out;
  SeqView v;  // the pair of dk and dv: v
  const float* decay;
  float s_intra, s_inter, s_upd;  // factors of the chunk's own part, the state's, and of sources on their way into it
  const float* s0;  // [B, N, ka, kc] with the strides below, or null (0)
  float* s1;        // the state that leaves, or null
  int st_a, st_c;   // the states' strides
  const uint8_t* resets;
  const int32_t* lengths;
  int nseg, per;   // segments, and chunks in each
  float* seg;      // [B N][nseg][ka][kc]: what enters each segment (state launch: its own sum, with strides st_a, st_c)
  float* hold;     // [B N][nseg] state launch: what a segment leaves of the state that enters it, -1 with a reset
};

template <typename DT> struct Tile;
template <> struct Tile<bf16_t> {
  static constexpr int VEC = 8, PAD = 8, SLICE = 32, PLANES = 2;
};
template <> struct Tile<float> {
  static constexpr int VEC = 4, PAD = 4, SLICE = 16, PLANES = 1;
};

__device__ __forceinline__ bf16x8 join(v2u a, v2u b) { return __builtin_bit_cast(bf16x8, v4u{a.x, a.y, b.x, b.y}); }

// The same value, which the compiler takes for another one in every round of a loop:
// what follows from it (weights, places in LDS, the sources' numbers) is computed
// again for each chunk in place of a hundred registers held over all of them.
__device__ __forceinline__ int anew(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
__device__ __forceinline__ float anew(float v) {
  asm volatile("" : "+v"(v));
  return v;
}

// a^n from log2 a (finite: log2 of 0 is held at kLogZero, so that a^0 = 1 there too).
constexpr float kLogZero = -1e30f;
__device__ __forceinline__ float decayed(float la, int n) { return __builtin_amdgcn_exp2f(la * (float)n); }

// Rows of one sequence and head of a [T, B, N, width] array.  FAST: as wide as the
// tile, on 16-byte boundaries and near enough for 32-bit offsets: range-checked
// loads and stores, which give zeros and nothing past the rows that exist.  Others
// load without a branch, the last piece of a row and the last row in the place of
// what lies behind them, and put that right where the piece is used (settle): a branch
// at each load would make each wait for the one before (T 128, B 512, 8 heads of 50
// and 37 bf16: outputs 106 -> 81 us, gradient 284 -> 225; fp32 303 -> 214 and 700 -> 552).
template <typename DT, int W, bool FAST>
struct Rows {
  static constexpr int V = Tile<DT>::VEC;
  DT* p;
  long t;     // elements between steps
  int width;  // of this tile
  __device__ __forceinline__ Rows(const SeqView& a, int b, int n, int heads_width, int col, int width_)
      : p(reinterpret_cast<DT*>(const_cast<void*>(a.p)) + (long)b * a.b + (long)n * heads_width + col), t(a.t), width(width_) {}
  // rows [t0, t0 + count)
  struct Chunk {
    rsrc_t r;
    DT* p;
    int count;
  };
  __device__ __forceinline__ Chunk at(int t0, int count) const {
    Chunk c;
    c.p = p + (long)t0 * t;
    c.count = count;
    if constexpr (FAST) c.r = make_rsrc(c.p, count > 0 ? (uint32_t)(((long)(count - 1) * t + W) * (long)sizeof(DT)) : 0u);
    return c;
  }
  // 16 bytes of row s from column c on
  __device__ __forceinline__ v4u load(const Chunk& k, int s, int c) const {
    if constexpr (FAST) {
      const uint4 v = bload16(k.r, ((uint32_t)s * (uint32_t)t + (uint32_t)c) * (uint32_t)sizeof(DT));
      return v4u{v.x, v.y, v.z, v.w};
    } else {
      if (width < V) return s < k.count ? load_piece<DT>(k.p + (long)s * t, c, width) : v4u{0, 0, 0, 0};
      const DT* const row = k.p + (long)max(min(s, k.count - 1), 0) * t;
      return *reinterpret_cast<const typename Mem16<DT>::type*>(row + min(c, width - V));
    }
  }
  // the piece that load(k, s, c) was to give, from what it gave
  __device__ __forceinline__ v4u settle(v4u v, int count, int s, int c) const {
    if constexpr (!FAST) {
      if (width < V) return v;
      if (s >= count || c >= width) return v4u{0, 0, 0, 0};
      if (c + V > width) return elements_from<DT>(v, c + V - width);
    }
    return v;
  }
  // four values of row s from column c on
  __device__ __forceinline__ void store(const Chunk& k, int s, int c, const float (&v)[4]) const {
    if constexpr (FAST) {
      const uint32_t o = ((uint32_t)s * (uint32_t)t + (uint32_t)c) * (uint32_t)sizeof(DT);
      if constexpr (sizeof(DT) == 4)
        bstore16(k.r, o, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
      else
        bstore8(k.r, o, make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])));
    } else if (s < k.count) {
      DT* const row = k.p + (long)s * t;
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
  }
};

// Columns 16 cb + 4 g .. + 3 and 16 (cb + 1) + 4 g .. + 3 of row s.  bf16 lanes first
// trade halves with the lanes of the next sixteen, so that each has eight columns in a
// row of one block, 16 bytes to store in place of two times 8.
template <typename DT, int W, bool FAST>
__device__ __forceinline__ void store_pair(const Rows<DT, W, FAST>& rows, const typename Rows<DT, W, FAST>::Chunk& k, int s, int cb,
                                           int g, const float (&x)[4], const float (&y)[4]) {
  if constexpr (FAST && sizeof(DT) == 2) {
    const auto p = __builtin_amdgcn_permlane16_swap(pack2_bf16(x[0], x[1]), pack2_bf16(y[0], y[1]), false, false);
    const auto q = __builtin_amdgcn_permlane16_swap(pack2_bf16(x[2], x[3]), pack2_bf16(y[2], y[3]), false, false);
    const uint32_t c = (uint32_t)(16 * cb + 16 * (g & 1) + 8 * (g >> 1));
    bstore16(k.r, ((uint32_t)s * (uint32_t)rows.t + c) * 2u, make_uint4(p[0], q[0], p[1], q[1]));
  } else {
    if (16 * cb < rows.width) rows.store(k, s, 16 * cb + 4 * g, x);
    if (16 * (cb + 1) < rows.width) rows.store(k, s, 16 * (cb + 1) + 4 * g, y);
  }
}

// A chunk's 64 rows in LDS, by all threads.
template <typename DT, int W>
struct Panel {
  static constexpr int V = Tile<DT>::VEC, PITCH = W + Tile<DT>::PAD, N = kChunk * (W / V) / kThreads, SIZE = kChunk * PITCH;
  static_assert(N > 0, "a piece or more for every thread");
  v4u r[N];
  template <bool FAST>
  __device__ __forceinline__ void load(const Rows<DT, W, FAST>& rows, const typename Rows<DT, W, FAST>::Chunk& c) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + i * kThreads;
      r[i] = rows.load(c, p / (W / V), p % (W / V) * V);
    }
  }
  template <bool FAST>
  __device__ __forceinline__ void store(DT* lds, const Rows<DT, W, FAST>& rows, int count) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + i * kThreads;
      *reinterpret_cast<v4u*>(lds + p / (W / V) * PITCH + p % (W / V) * V) = rows.settle(r[i], count, p / (W / V), p % (W / V) * V);
    }
  }
};
// The lane's row of a chunk as a matrix operand, along the row.
template <typename DT, int W>
struct RowFrag {
  static constexpr int SL = Tile<DT>::SLICE, V = Tile<DT>::VEC, N = W / SL;
  v4u r[N];
  template <bool FAST>
  __device__ __forceinline__ void load(const Rows<DT, W, FAST>& rows, const typename Rows<DT, W, FAST>::Chunk& c, int s, int g) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = rows.load(c, s, i * SL + V * g);
  }
  template <bool FAST>
  __device__ __forceinline__ void settle(const Rows<DT, W, FAST>& rows, int count, int s, int g) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = rows.settle(r[i], count, s, i * SL + V * g);
  }
  __device__ __forceinline__ uint4 operator[](int i) const { return make_uint4(r[i].x, r[i].y, r[i].z, r[i].w); }
};

// What a work-group is at: a sequence, a head and a segment.
struct Place {
  int b, n, seg, len, first, last;
  long bn, part;
  float la;  // log2 of the decay
  __device__ __forceinline__ Place(const MixArgs& a, long at) : part(at) {
    seg = (int)(at % a.nseg);
    bn = at / a.nseg;
    n = (int)(bn % a.N);
    b = (int)(bn / a.N);
    len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    la = fmaxf(log2f(fminf(fmaxf(a.decay[n], 0.0f), 1.0f)), kLogZero);
    const int chunks = chunks_of(a.T);
    first = seg * a.per;
    last = min(first + a.per, chunks);
  }
};

// The masks of a chunk: bit s of `starts` for a step that begins a trajectory.
template <bool REV>
struct Mask {
  int lo, hi;    // a row's sources
  bool entered;  // whether the state that enters reaches the row
  __device__ __forceinline__ Mask(uint64_t starts, int live, int r) {
    const uint64_t upto = ~0ull >> (63 - r), cut = REV ? starts & ~upto : starts & upto;
    lo = REV ? r : cut ? 63 - __clzll((long long)cut) : 0;
    hi = REV ? (cut ? __ffsll((long long)cut) - 2 : live - 1) : r;
    entered = cut == 0;
  }
};

// What a chunk's sources weigh: for the lane's row, the source s = 16 j + 4 g + e;
// and on their way into the state, s = 32 jj + 16 (e / 4) + 4 g + e % 4.  bf16 sweeps,
// whose time goes to such arithmetic, keep both in registers and compute them again
// only where a chunk has resets or padding, or follows one that has (T 32768, 16
// heads of 64: outputs 81 -> 76 us, gradient 193 -> 186, states 42 -> 35); fp32 ones, whose time goes
// to the matrix unit, have no registers for them.
template <typename DT, bool REV>
struct Weights {
  static constexpr bool KEPT = sizeof(DT) == 2;
  float w[KEPT ? 4 : 1][4], u[KEPT ? 2 : 1][8];
  bool whole = false;  // those of a whole chunk of one trajectory
  // the sources that the state takes
  __device__ __forceinline__ static float taken(uint64_t starts, int live, int s, float la, float upd) {
    const int lo = REV ? 0 : starts ? 63 - __clzll((long long)starts) : 0;
    const int hi = REV ? (starts ? __ffsll((long long)starts) - 2 : live - 1) : live - 1;
    return s >= lo && s <= hi ? upd * decayed(la, REV ? s + 1 : live - 1 - s) : 0.0f;
  }
  __device__ __forceinline__ void update(const Mask<REV>& mask, uint64_t starts, int live, int r, int g, float la, float intra,
                                         float upd) {
    if constexpr (KEPT) {
      const bool plain = starts == 0 && live == kChunk;
      if (plain && whole) return;
      whole = plain;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) w[j][e] = of(mask, 16 * j + 4 * g + e, r, la, intra);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int e = 0; e < 8; ++e) u[jj][e] = taken(starts, live, 32 * jj + 16 * (e / 4) + 4 * g + e % 4, la, upd);
    }
  }
  __device__ __forceinline__ static float of(const Mask<REV>& mask, int s, int r, float la, float intra) {
    return s >= mask.lo && s <= mask.hi ? intra * decayed(la, REV ? s - r : r - s) : 0.0f;
  }
};

// The state of a head, [KA][KC], in the registers of four waves: blocks of rows
// 16 (wk KAB + i) + 4 g + 0..3 and column 16 (wc KCB + k) + j16.
template <typename DT, int KA, int KC>
struct State {
  static constexpr bool F32 = sizeof(DT) == 4;
  static constexpr int WK = KA >= 64 ? 4 : 2, WC = 4 / WK, KAB = KA / 16 / WK, KCB = KC / 16 / WC;
  static constexpr int PA = KA + Tile<DT>::PAD, PC = KC + Tile<DT>::PAD, PL = Tile<DT>::PLANES;
  static constexpr int SIZE = PL * KC * PA;  // in LDS, columns first
  f32x4 S[KAB][KCB];
  int wk, wc, g, j16;
  __device__ __forceinline__ State() {
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    wk = w % WK;
    wc = w / WK;
    g = lane >> 4;
    j16 = lane & 15;
  }
  __device__ __forceinline__ int row(int i) const { return 16 * (wk * KAB + i) + 4 * g; }
  __device__ __forceinline__ int col(int k) const { return 16 * (wc * KCB + k) + j16; }
  // p: [ka][..] with strides st_a and st_c; null for zeros
  __device__ __forceinline__ void load(const float* p, int ka, int kc, int st_a, int st_c) {
#pragma unroll
    for (int i = 0; i < KAB; ++i)
#pragma unroll
      for (int k = 0; k < KCB; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          S[i][k][e] = p && row(i) + e < ka && col(k) < kc ? p[(long)(row(i) + e) * st_a + (long)col(k) * st_c] : 0.0f;
  }
  // `finite`: leaves what p holds in the place of NaN
  __device__ __forceinline__ void save(float* p, int ka, int kc, int st_a, int st_c, bool finite) const {
#pragma unroll
    for (int i = 0; i < KAB; ++i)
#pragma unroll
      for (int k = 0; k < KCB; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (row(i) + e < ka && col(k) < kc && !(finite && S[i][k][e] != S[i][k][e]))
            p[(long)(row(i) + e) * st_a + (long)col(k) * st_c] = S[i][k][e];
  }
  __device__ __forceinline__ bool nan() const {
    bool n = false;
#pragma unroll
    for (int i = 0; i < KAB; ++i)
#pragma unroll
      for (int k = 0; k < KCB; ++k) n |= any_nan(S[i][k]);
    return n;
  }
  __device__ __forceinline__ void stage(DT* st) const {
#pragma unroll
    for (int i = 0; i < KAB; ++i)
#pragma unroll
      for (int k = 0; k < KCB; ++k) {
        DT* const p = st + col(k) * PA + row(i);
        const f32x4 v = S[i][k];
        if constexpr (F32) {
          *reinterpret_cast<v4u*>(p) = __builtin_bit_cast(v4u, v);
        } else {
          const v2u h = {pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
          *reinterpret_cast<v2u*>(p) = h;
          *reinterpret_cast<v2u*>(p + KC * PA) =
              v2u{pack2_bf16(v[0] - __uint_as_float(h.x << 16), v[1] - __uint_as_float(h.x & 0xffff0000u)),
                  pack2_bf16(v[2] - __uint_as_float(h.y << 16), v[3] - __uint_as_float(h.y & 0xffff0000u))};
        }
      }
  }
  // S becomes hold S + sum over the sources of their weight times B_s C_s^T, the weights'
  // distances counting to the end of the chunk that the sweep leaves by; at a reset
  // hold S is 0, whatever S is
  template <bool REV>
  __device__ __forceinline__ void take(const DT* bl, const DT* cl, const Weights<DT, REV>& wt, uint64_t starts, int live, int lane,
                                       float la, float upd) {
    const int g = lane >> 4, j16 = lane & 15;
    if (starts) {
#pragma unroll
      for (int i = 0; i < KAB; ++i)
#pragma unroll
        for (int k = 0; k < KCB; ++k) S[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
    } else {
      const float hold = decayed(la, live);
#pragma unroll
      for (int i = 0; i < KAB; ++i)
#pragma unroll
        for (int k = 0; k < KCB; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[i][k][e] *= hold;
    }
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      if (32 * jj >= live) break;  // nothing but padding from here on
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (32 * jj + 16 * (e / 4) >= live) break;
          const int s = 32 * jj + 16 * (e / 4) + 4 * g + e % 4;
          const float ws = Weights<DT, REV>::taken(starts, live, s, la, upd);
          float x[KAB];
#pragma unroll
          for (int i = 0; i < KAB; ++i) {
            const float v = bl[s * PA + 16 * (wk * KAB + i) + j16];
            x[i] = v * ws;
          }
#pragma unroll
          for (int k = 0; k < KCB; ++k) {
            const float y = cl[s * PC + 16 * (wc * KCB + k) + j16];
#pragma unroll
            for (int i = 0; i < KAB; ++i) S[i][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y, S[i][k], 0, 0, 0);
          }
        }
      } else {
        Split3 x[KAB];
#pragma unroll
        for (int i = 0; i < KAB; ++i) {
          const bf16_t* const p = bl + (32 * jj + 4 * g + j16 / 4) * PA + 16 * (wk * KAB + i) + 4 * (j16 % 4);
          const v2u u0 = read_tr(p), u1 = read_tr(p + 16 * PA);
          const uint32_t u[4] = {u0.x, u0.y, u1.x, u1.y};
          float f[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f[2 * e] = __uint_as_float(u[e] << 16) * wt.u[jj][2 * e];
            f[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u) * wt.u[jj][2 * e + 1];
          }
          x[i] = split3(f);
        }
#pragma unroll
        for (int k = 0; k < KCB; ++k) {
          const bf16_t* const p = cl + (32 * jj + 4 * g + j16 / 4) * PC + 16 * (wc * KCB + k) + 4 * (j16 % 4);
          const bf16x8 y = join(read_tr(p), read_tr(p + 16 * PC));
#pragma unroll
          for (int i = 0; i < KAB; ++i) {
            S[i][k] = mfma_bf16(x[i].l, y, S[i][k]);
            S[i][k] = mfma_bf16(x[i].m, y, S[i][k]);
            S[i][k] = mfma_bf16(x[i].h, y, S[i][k]);
          }
        }
      }
    }
  }
};

// The chunk's part of the rows of wave w: the weighted products of a row with its
// sources as a matrix operand, and their product with the sources' values.
template <typename DT, int KA, bool REV>
struct Intra {
  static constexpr bool F32 = sizeof(DT) == 4;
  static constexpr int PA = KA + Tile<DT>::PAD, SL = Tile<DT>::SLICE, V = Tile<DT>::VEC;
  float P[4][4];
  bf16x8 ph[2], pm[2];
  __device__ __forceinline__ Intra(const DT* bl, const RowFrag<DT, KA>& rows, const Weights<DT, REV>& wt, const Mask<REV>& mask,
                                   int r, int w, int g, int j16, int live, float la, float scale) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      if (REV ? j >= w && 16 * j < live : j <= w) {
#pragma unroll
        for (int k = 0; k < KA / SL; ++k) {
          const v4u x = *reinterpret_cast<const v4u*>(bl + (16 * j + j16) * PA + k * SL + V * g);
          Mfma<DT>::step(acc, make_uint4(x.x, x.y, x.z, x.w), rows[k]);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int s = 16 * j + 4 * g + e;
        if constexpr (F32)
          P[j][e] = acc[e] * Weights<DT, REV>::of(mask, s, r, la, scale);
        else
          P[j][e] = acc[e] * wt.w[j][e];
      }
    }
    if constexpr (!F32) {
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        v4u h, m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = P[2 * jj + e / 2][2 * (e & 1)], y = P[2 * jj + e / 2][2 * (e & 1) + 1];
          h[e] = pack2_bf16(x, y);
          m[e] = pack2_bf16(x - __uint_as_float(h[e] << 16), y - __uint_as_float(h[e] & 0xffff0000u));
        }
        ph[jj] = __builtin_bit_cast(bf16x8, h);
        pm[jj] = __builtin_bit_cast(bf16x8, m);
      }
    }
  }
  // columns 16 cb .. + 15 of the values at cl (pitch PC)
  template <int PC>
  __device__ __forceinline__ f32x4 times(const DT* cl, int cb, int w, int g, int j16, int live) const {
    f32x4 out = {0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (REV ? j < w || 16 * j >= live : j > w) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          out = __builtin_amdgcn_mfma_f32_16x16x4f32(cl[(16 * j + 4 * g + e) * PC + 16 * cb + j16], P[j][e], out, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        if (REV ? 2 * jj + 1 < w || 32 * jj >= live : 2 * jj > w) continue;
        const bf16_t* const p = cl + (32 * jj + 4 * g + j16 / 4) * PC + 16 * cb + 4 * (j16 % 4);
        const bf16x8 x = join(read_tr(p), read_tr(p + 16 * PC));
        out = mfma_bf16(x, pm[jj], out);
        out = mfma_bf16(x, ph[jj], out);
      }
    }
    return out;
  }
};

// Columns 16 cb .. + 15 of the rows' products with the state in LDS ([KC][KA]).
template <typename DT, int KA, int KC>
__device__ __forceinline__ f32x4 entered(const DT* st, const RowFrag<DT, KA>& rows, int cb, int g, int j16) {
  constexpr int PA = KA + Tile<DT>::PAD, SL = Tile<DT>::SLICE, V = Tile<DT>::VEC;
  f32x4 in = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < KA / SL; ++k)
#pragma unroll
    for (int p = Tile<DT>::PLANES - 1; p >= 0; --p) {
      const v4u x = *reinterpret_cast<const v4u*>(st + (p * KC + 16 * cb + j16) * PA + k * SL + V * g);
      Mfma<DT>::step(in, make_uint4(x.x, x.y, x.z, x.w), rows[k]);
    }
  return in;
}
// The same with the state's transpose: rows of width KC, columns 16 kb .. + 15 of KA.
template <typename DT, int KA, int KC>
__device__ __forceinline__ f32x4 entered_across(const DT* st, const RowFrag<DT, KC>& rows, int kb, int g, int j16) {
  constexpr int PA = KA + Tile<DT>::PAD, SL = Tile<DT>::SLICE;
  f32x4 in = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < KC / SL; ++k) {
    if constexpr (sizeof(DT) == 4) {
      const float* const p = st + (k * SL + 4 * g) * PA + 16 * kb + j16;
      Mfma<DT>::step(in, make_uint4(__float_as_uint(p[0]), __float_as_uint(p[PA]), __float_as_uint(p[2 * PA]), __float_as_uint(p[3 * PA])),
                     rows[k]);
    } else {
#pragma unroll
      for (int pl = 1; pl >= 0; --pl) {
        const bf16_t* const p = st + (pl * KC + k * SL + 8 * g + j16 / 4) * PA + 16 * kb + 4 * (j16 % 4);
        const v2u x = read_tr(p), y = read_tr(p + 4 * PA);
        Mfma<DT>::step(in, make_uint4(x.x, x.y, y.x, y.y), rows[k]);
      }
    }
  }
  return in;
}

// Whether the lane's step of a chunk begins a trajectory; requested with the chunk's
// pieces, so that no chunk waits for it.
__device__ __forceinline__ uint32_t reset_of(const MixArgs& a, int b, int t0, int live) {
  const int lane = threadIdx.x & 63;
  return a.resets && lane < live ? a.resets[(long)(t0 + lane) * a.B + b] : 0;
}

// Whether `v` holds in any of the work-group's threads (`words`: four, which nothing else uses).
__device__ __forceinline__ bool in_any(bool v, int* words) {
  const bool any = __any(v);
  if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = any;
  __syncthreads();
  return (words[0] | words[1] | words[2] | words[3]) != 0;
}

// The launch's arguments, loaded again, for code that hardly ever runs: the sweeps keep
// no registers for it.  `at`: which bytes of them.
template <typename T>
__device__ __forceinline__ const T& argument(int at) {
  auto p = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const T*)(p + at);
}

// A masked source counts as 0 times its value in the products, which is NaN where the
// value, or its product with the row, is not finite.  A segment that comes out with NaN
// is therefore taken a second time, step by step as the recurrence says, and what this
// gives replaces NaN, so that nothing reaches a step on the other side of its own or
// another trajectory.  Finite results stay as they are.
//   F = (state that enters) + upd B_t C_t^T, out_t = inter A_t . F;
// columns [ct, ct + cols) of C and the output; s0, s1: the state that enters and the one
// that leaves, [ka][kc] with strides st_a and st_c.  Sixteen columns at a time, sixteen
// threads each, up to 16 R rows of the state: little code, which the sweeps have beside
// their own (three times as much of it, and the gradient of T 128, B 512, 8 heads of 64
// fp32 took 388 us in place of 361).  A step takes some 2 us: with NaN in every v that
// call takes 10.6 ms in place of 0.5.
template <typename DT, int R, bool REV, bool OUT>
__device__ __forceinline__ void by_steps(const MixArgs& a, long part, const SeqView& va, const SeqView& vb, const SeqView& vc,
                                         const SeqView& vo, int ka, int kc, int ct, int cols, const float* s0, float* s1, int st_a,
                                         int st_c, float* sum) {
  asm volatile("" : "+s"(part));
  const Place at(a, part);
  auto line = [&](const SeqView& v, int width) { return reinterpret_cast<DT*>(const_cast<void*>(v.p)) + (long)at.b * v.b + (long)at.n * width; };
  const DT *const A = line(va, ka), *const B = line(vb, ka), *const C = line(vc, kc);
  DT* const out = line(vo, kc);
  const float decay = fminf(fmaxf(a.decay[at.n], 0.0f), 1.0f);
  const int begin = at.first * kChunk, steps = min((int)min((long)at.last * kChunk, (long)a.T), at.len) - begin;
  const int row0 = threadIdx.x / 16 * R;
#pragma unroll 1
  for (int c0 = 0; c0 < cols; c0 += 16) {
    const int in = c0 + threadIdx.x % 16, col = ct + min(in, cols - 1);  // (those past the end do the last one's work)
    float S[R];
#pragma unroll
    for (int r = 0; r < R; ++r) S[r] = s0 && row0 + r < ka ? s0[(long)(row0 + r) * st_a + (long)col * st_c] : 0.0f;
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
      const long t = REV ? begin + steps - 1 - i : begin + i;
      const bool start = a.resets && a.resets[t * a.B + at.b] != 0;
      const DT *const x = A + t * va.t, *const z = B + t * vb.t;
      const float c = a.s_upd * DType<DT>::load(C + t * vc.t, col);
      float y = 0.0f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (row0 + r >= ka) break;
        const float b = DType<DT>::load(z, row0 + r) * c;
        S[r] = REV ? S[r] + b : start ? b : fmaf(decay, S[r], b);
        if (OUT) y = fmaf(DType<DT>::load(x, row0 + r), S[r], y);
        if (REV) S[r] = start ? 0.0f : decay * S[r];
      }
      if constexpr (OUT) {
        __syncthreads();
        sum[threadIdx.x] = y;
        __syncthreads();
        if (threadIdx.x == in - c0 && in < cols) {
          for (int g = 16; g < kThreads; g += 16) y += sum[g + threadIdx.x];
          DT* const p = out + t * vo.t;
          const float old = DType<DT>::load(p, col);
          if (old != old) DType<DT>::store(p, col, a.s_inter * y);
        }
      }
    }
    if (s1 && in < cols) {
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (row0 + r < ka) s1[(long)(row0 + r) * st_a + (long)col * st_c] = S[r];
    }
  }
  __syncthreads();
}

// One sweep over a segment's chunks: the outputs of columns [ct, ct + KC), or, STATE,
// the segment's own sum of the state alone.
template <typename DT, int KA, int KC, bool REV, bool STATE, bool FAST>
__device__ __forceinline__ void sweep(const MixArgs& a, const Place& at, int ct, DT* bl, DT* cl, DT* st) {  // a: the launch's first
  constexpr int PC = KC + Tile<DT>::PAD;
  const int w = threadIdx.x >> 6, lane0 = threadIdx.x & 63;
  const int wcols = min(KC, a.kc - ct);
  const Rows<DT, KA, FAST> ra(a.a, at.b, at.n, a.ka, 0, a.ka), rb(a.b, at.b, at.n, a.ka, 0, a.ka);
  const Rows<DT, KC, FAST> rc(a.c, at.b, at.n, a.kc, ct, wcols), ro(a.out, at.b, at.n, a.kc, ct, wcols);
  Panel<DT, KA> pb;
  Panel<DT, KC> pc;
  RowFrag<DT, KA> rows;
  uint32_t reset = 0;
  auto load = [&](int c) {
    const int t0 = c * kChunk, live = min(at.len - t0, kChunk);
    pb.template load<FAST>(rb, rb.at(t0, live));
    pc.template load<FAST>(rc, rc.at(t0, live));
    reset = reset_of(a, at.b, t0, live);
  };
  auto load_rows = [&](int c) {
    if constexpr (!STATE) {
      const int lane = anew(lane0), g = lane >> 4, r = 16 * w + (lane & 15);
      const int t0 = c * kChunk, live = min(at.len - t0, kChunk);
      rows.template load<FAST>(ra, ra.at(t0, live), r, g);
    }
  };
  __shared__ int words[4];
  const int steps = at.last - at.first;
  if (steps > 0) {
    load(REV ? at.last - 1 : at.first);
    load_rows(REV ? at.last - 1 : at.first);
  }
  State<DT, KA, KC> S;
  const float* s0 = STATE ? nullptr : a.seg ? a.seg + at.part * a.ka * a.kc : a.s0 ? a.s0 + at.bn * a.ka * a.kc : nullptr;
  S.load(s0 ? s0 + (long)ct * a.st_c : nullptr, a.ka, wcols, a.st_a, a.st_c);
  Weights<DT, REV> wt;
  float hold = 1.0f;
  float all = 0.0f;  // the outputs' sum, which is not finite where one of them is not
  for (int step = 0; step < steps; ++step) {
    const int c = REV ? at.last - 1 - step : at.first + step, t0 = c * kChunk;
    const int live = min(at.len - t0, kChunk);  // steps of the chunk inside the sequence, 0 or less for none
    const uint64_t starts = __ballot(reset != 0);
    const int lane = anew(lane0), g = lane >> 4, j16 = lane & 15, r = 16 * w + j16;
    const float la = anew(at.la);
    __syncthreads();  // the chunk before is done with
    pb.store(bl, rb, live);
    pc.store(cl, rc, live);
    if constexpr (!STATE) {
      rows.settle(ra, live, r, g);
      S.stage(st);
    }
    // the next chunk's pieces: requested here they are on their way during the whole
    // chunk, where there are registers for them
    constexpr bool EARLY = STATE || sizeof(DT) == 2;
    const int next = REV ? c - 1 : c + 1;
    const bool more = step + 1 < steps;
    if (EARLY && more) load(next);
    __syncthreads();
    const Mask<REV> mask(starts, live, r);
    if (live > 0) wt.update(mask, starts, live, r, g, la, a.s_intra, a.s_upd);
    if constexpr (!STATE) {
      const auto oc = ro.at(t0, min(a.T - t0, kChunk));
      if (16 * w >= live) {  // the wave's rows are padding
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int cb = 0; cb < KC / 16; cb += 2) store_pair(ro, oc, r, cb, g, zero, zero);
      } else {
        const float win = a.s_inter * decayed(la, REV ? live - 1 - r : r + 1);
        const Intra<DT, KA, REV> P(bl, rows, wt, mask, r, w, g, j16, live, la, a.s_intra);
#pragma unroll
        for (int cb = 0; cb < KC / 16; cb += 2) {
          if (16 * cb >= wcols) break;
          float v[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x4 in = entered<DT, KA, KC>(st, rows, cb + i, g, j16), own = P.template times<PC>(cl, cb + i, w, g, j16, live);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = r < live ? own[e] + (mask.entered ? win * in[e] : 0.0f) : 0.0f;
            all += (v[i][0] + v[i][1]) + (v[i][2] + v[i][3]);
          }
          store_pair(ro, oc, r, cb, g, v[0], v[1]);
        }
      }
    }
    if (!EARLY && more) load(next);
    if (more) load_rows(next);
    if (live <= 0) continue;
    if constexpr (STATE) hold = starts || hold < 0.0f ? -1.0f : hold * decayed(la, live);
    S.template take<REV>(bl, cl, wt, starts, live, lane, la, a.s_upd);
  }
  float* const s1 = STATE ? a.seg + at.part * a.ka * a.kc : a.seg || !a.s1 ? nullptr : a.s1 + at.bn * a.ka * a.kc;
  const bool again = in_any(all - all != 0.0f || (s1 && S.nan()), words);
  if (__builtin_expect(again, 0)) {
    const MixArgs& b = argument<MixArgs>(0);
    by_steps<DT, KA / 16, REV, !STATE>(b, at.part, b.a, b.b, b.c, b.out, b.ka, b.kc, ct, wcols, s0, s1, b.st_a, b.st_c,
                                       reinterpret_cast<float*>(bl));
  }
  if (s1) S.save(s1 + (long)ct * a.st_c, a.ka, wcols, a.st_a, a.st_c, again);
  if constexpr (STATE) {
    if (threadIdx.x == 0 && ct == 0) a.hold[at.part] = hold;
  }
}

// Waves a SIMD that the registers are to admit: as many as LDS does, fp32 rows that
// are not FAST one less, and their few spills with it (bf16 gains by the third wave:
// T 128, B 512, 8 heads of 50 and 37 with two 95 and 252 us, with three 81 and 225);
// four for heads of 32 (T 512, B 256, 8 heads fp32, gradient 388 and 366 us).
constexpr int waves(int size, int ka, int kc, bool fast) {
  if (ka > 64) return size == 4 ? (kc > 32 ? 1 : 2) : (kc > 32 ? 2 : 3 - !fast);
  if (ka <= 32 && kc <= 32 && fast) return 4;
  return size == 4 ? 3 - !fast : 3;
}

template <typename DT, int KA, int KC, bool REV, bool STATE, bool FAST>
__global__ void __launch_bounds__(kThreads, waves(sizeof(DT), KA, KC, FAST)) k_mix(const MixArgs a) {
  __shared__ __align__(16) DT bl[Panel<DT, KA>::SIZE];
  __shared__ __align__(16) DT cl[Panel<DT, KC>::SIZE];
  __shared__ __align__(16) DT st[STATE ? 16 : State<DT, KA, KC>::SIZE];
  const int nct = (a.kc + KC - 1) / KC;
  sweep<DT, KA, KC, REV, STATE, FAST>(a, Place(a, blockIdx.x / nct), blockIdx.x % nct * KC, bl, cl, st);
}

// The reverse sweep for both dk and dv: they share the sources q and dy and the
// state G [K][V], which dk's rows v meet across.
template <typename DT, int KP, int VP, bool FAST>
__device__ __forceinline__ void sweep_back(const MixArgs& a, const SeqView& dk, const Place& at, DT* ql, DT* dl, DT* st) {
  constexpr int PK = KP + Tile<DT>::PAD, PV = VP + Tile<DT>::PAD;
  const int w = threadIdx.x >> 6, lane0 = threadIdx.x & 63;
  // of dv: A = k, B = q, C = dy; a row's v are reached through c's place: dk = (A = v, B = dy, C = q)
  const Rows<DT, KP, FAST> rk(a.a, at.b, at.n, a.ka, 0, a.ka), rq(a.b, at.b, at.n, a.ka, 0, a.ka), ok(dk, at.b, at.n, a.ka, 0, a.ka);
  const Rows<DT, VP, FAST> rd(a.c, at.b, at.n, a.kc, 0, a.kc), rv(a.v, at.b, at.n, a.kc, 0, a.kc), ov(a.out, at.b, at.n, a.kc, 0, a.kc);
  Panel<DT, KP> pq;
  Panel<DT, VP> pd;
  RowFrag<DT, KP> k;
  RowFrag<DT, VP> v;
  uint32_t reset = 0;
  auto load = [&](int c) {
    const int t0 = c * kChunk, live = min(at.len - t0, kChunk);
    pq.template load<FAST>(rq, rq.at(t0, live));
    pd.template load<FAST>(rd, rd.at(t0, live));
    reset = reset_of(a, at.b, t0, live);
  };
  auto load_rows = [&](int c) {
    const int lane = anew(lane0), g = lane >> 4, r = 16 * w + (lane & 15);
    const int t0 = c * kChunk, live = min(at.len - t0, kChunk);
    k.template load<FAST>(rk, rk.at(t0, live), r, g);
    v.template load<FAST>(rv, rv.at(t0, live), r, g);
  };
  __shared__ int words[4];
  if (at.last > at.first) {
    load(at.last - 1);
    load_rows(at.last - 1);
  }
  State<DT, KP, VP> S;
  const float* const s0 = a.seg ? a.seg + at.part * a.ka * a.kc : a.s0 ? a.s0 + at.bn * a.ka * a.kc : nullptr;
  S.load(s0, a.ka, a.kc, a.st_a, a.st_c);
  Weights<DT, true> wt;
  float all = 0.0f;  // the outputs' sum, which is not finite where one of them is not
  for (int c = at.last - 1; c >= at.first; --c) {
    const int t0 = c * kChunk, live = min(at.len - t0, kChunk);
    const uint64_t starts = __ballot(reset != 0);
    const int lane = anew(lane0), g = lane >> 4, j16 = lane & 15, r = 16 * w + j16;
    const float la = anew(at.la);
    __syncthreads();
    pq.store(ql, rq, live);
    pd.store(dl, rd, live);
    k.settle(rk, live, r, g);
    v.settle(rv, live, r, g);
    S.stage(st);
    constexpr bool EARLY = sizeof(DT) == 2;
    if (EARLY && c > at.first) load(c - 1);
    __syncthreads();
    const auto ck = ok.at(t0, min(a.T - t0, kChunk));
    const auto cv = ov.at(t0, min(a.T - t0, kChunk));
    const Mask<true> mask(starts, live, r);
    if (live > 0) wt.update(mask, starts, live, r, g, la, a.s_intra, a.s_upd);
    if (16 * w >= live) {  // the wave's rows are padding
      const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int cb = 0; cb < VP / 16; cb += 2) store_pair(ov, cv, r, cb, g, zero, zero);
#pragma unroll
      for (int kb = 0; kb < KP / 16; kb += 2) store_pair(ok, ck, r, kb, g, zero, zero);
    } else {
      const float win = a.s_inter * decayed(la, live - 1 - r);
      const bool on = r < live;
      {
        const Intra<DT, KP, true> P(ql, k, wt, mask, r, w, g, j16, live, la, a.s_intra);
#pragma unroll
        for (int cb = 0; cb < VP / 16; cb += 2) {
          if (16 * cb >= a.kc) break;
          float x[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x4 in = entered<DT, KP, VP>(st, k, cb + i, g, j16), own = P.template times<PV>(dl, cb + i, w, g, j16, live);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = on ? own[e] + (mask.entered ? win * in[e] : 0.0f) : 0.0f;
            all += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
          }
          store_pair(ov, cv, r, cb, g, x[0], x[1]);
        }
      }
      {
        const Intra<DT, VP, true> P(dl, v, wt, mask, r, w, g, j16, live, la, a.s_intra);
#pragma unroll
        for (int kb = 0; kb < KP / 16; kb += 2) {
          if (16 * kb >= a.ka) break;
          float x[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x4 in = entered_across<DT, KP, VP>(st, v, kb + i, g, j16),
                        own = P.template times<PK>(ql, kb + i, w, g, j16, live);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = on ? own[e] + (mask.entered ? win * in[e] : 0.0f) : 0.0f;
            all += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
          }
          store_pair(ok, ck, r, kb, g, x[0], x[1]);
        }
      }
    }
    if (c > at.first) {
      if (!EARLY) load(c - 1);
      load_rows(c - 1);
    }
    if (live > 0) S.template take<true>(ql, dl, wt, starts, live, lane, la, a.s_upd);
  }
  float* const s1 = a.seg || !a.s1 ? nullptr : a.s1 + at.bn * a.ka * a.kc;
  const bool again = in_any(all - all != 0.0f || (s1 && S.nan()), words);
  if (__builtin_expect(again, 0)) {
    const MixArgs& b = argument<MixArgs>(sizeof(MixArgs));
#pragma unroll 1
    for (int of_k = 1; of_k >= 0; --of_k) {
      const SeqView &va = of_k ? b.v : b.a, &vb = of_k ? b.c : b.b, &vc = of_k ? b.b : b.c,
                    &vo = of_k ? argument<SeqView>(2 * sizeof(MixArgs)) : b.out;
      const int ka = of_k ? b.kc : b.ka, kc = of_k ? b.ka : b.kc;
      by_steps<DT, (KP > VP ? KP : VP) / 16, true, true>(b, at.part, va, vb, vc, vo, ka, kc, 0, kc, s0, of_k ? nullptr : s1,
                                                         of_k ? b.st_c : b.st_a, of_k ? b.st_a : b.st_c, reinterpret_cast<float*>(ql));
    }
  }
  if (s1) S.save(s1, a.ka, a.kc, a.st_a, a.st_c, again);
}

// All three gradients of heads up to 64 wide: the forward sweep for dq, then the
// reverse one for dk and dv, which finds k, v and dy in the caches where the
// segment is short; or, `apart`, each in a work-group of its own.  (The arguments stay in
// this order: by_steps finds them by their places.)
template <typename DT, int KP, int VP, bool FAST>
__global__ void __launch_bounds__(kThreads, waves(sizeof(DT), KP, VP, FAST)) k_mix_grad(const MixArgs q, const MixArgs v, const SeqView dk,
                                                                                        int apart) {
  constexpr int SK = Panel<DT, KP>::SIZE, SV = Panel<DT, VP>::SIZE;
  constexpr int ST = State<DT, KP, VP>::SIZE > State<DT, VP, KP>::SIZE ? State<DT, KP, VP>::SIZE : State<DT, VP, KP>::SIZE;
  __shared__ __align__(16) DT kl[SK];
  __shared__ __align__(16) DT vl[SV];
  __shared__ __align__(16) DT st[ST];
  const Place at(q, blockIdx.x >> apart);
  const bool only = apart && (blockIdx.x & 1);
  if (!only) {
    sweep<DT, VP, KP, false, false, FAST>(q, at, 0, vl, kl, st);
    if (apart) return;
    __syncthreads();
  }
  sweep_back<DT, KP, VP, FAST>(v, dk, at, kl, vl, st);
}

// Runs through the segments' own sums: seg[i] becomes the state that enters it.
// One value of a head's state a thread; the sums of kAhead segments are requested
// together (one after the other, each store before the next load, 64 segments of 16
// heads of 64 x 64 take 15 us).
constexpr int kAhead = 16;
template <bool REV>
__global__ void __launch_bounds__(kThreads) k_segments(float* seg, const float* hold, const float* s0, float* s1, int nseg,
                                                       int width) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  const long bn = blockIdx.y;
  if (i >= width) return;
  float s = s0 ? s0[bn * width + i] : 0.0f;
  float* const p = seg + bn * nseg * (long)width + i;
  const float* const h = hold + bn * nseg;
  for (int k = 0; k < nseg; k += kAhead) {
    float own[kAhead], f[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int m = min(k + j, nseg - 1), at = REV ? nseg - 1 - m : m;
      own[j] = p[(long)at * width];
      f[j] = h[at];
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (k + j >= nseg) break;
      p[(long)(REV ? nseg - 1 - k - j : k + j) * width] = s;
      s = f[j] >= 0.0f ? fmaf(f[j], s, own[j]) : own[j];
    }
  }
  if (s1) s1[bn * width + i] = s;
}

// One step: y = scale (a S + k v^T)^T q, VEC columns and every `rows`-th row of the
// state a thread.
template <typename DT, int VEC>
__global__ void __launch_bounds__(kThreads) k_linattn_step(const LinattnArgs a, int lanes) {
  __shared__ float sum[kThreads * VEC];
  const int tid = threadIdx.x, rows = kThreads / lanes, lane = tid % lanes, row0 = tid / lanes;
  const long bn = blockIdx.x;
  const int n = (int)(bn % a.N), b = (int)(bn / a.N);
  const bool live = !a.lengths || a.lengths[b] > 0;
  const bool fresh = live && a.resets && a.resets[b] != 0;
  const float da = fminf(fmaxf(a.decay[n], 0.0f), 1.0f);
  const DT* q = reinterpret_cast<const DT*>(a.q.p) + (long)b * a.q.b + (long)n * a.K;
  const DT* k = reinterpret_cast<const DT*>(a.k.p) + (long)b * a.k.b + (long)n * a.K;
  const DT* v = reinterpret_cast<const DT*>(a.v.p) + (long)b * a.v.b + (long)n * a.V;
  const long base = bn * a.K * a.V;
  const int col = lane * VEC;
  const bool mine = col < a.V;
  float vv[VEC], y[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    vv[e] = live && mine ? DType<DT>::load(v, col + e) : 0.0f;
    y[e] = 0.0f;
  }
  struct alignas(4 * VEC) vec_t {
    float v[VEC];
  };
  if (mine) {
#pragma unroll 4
    for (int r = row0; r < a.K; r += rows) {
      vec_t s = {};
      const long at = base + (long)r * a.V + col;
      if (a.h0 && !fresh) s = *reinterpret_cast<const vec_t*>(a.h0 + at);
      if (live) {
        const float kk = DType<DT>::load(k, r), qq = DType<DT>::load(q, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          s.v[e] = fmaf(da, s.v[e], kk * vv[e]);
          y[e] = fmaf(qq, s.v[e], y[e]);
        }
      }
      if (a.h_T) *reinterpret_cast<vec_t*>(a.h_T + at) = s;
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e * kThreads + tid] = y[e];
  __syncthreads();
  DT* out = reinterpret_cast<DT*>(a.y) + bn * a.V;
  for (int c = tid; c < a.V; c += kThreads) {
    float t = 0.0f;
    for (int r = 0; r < rows; ++r) t += sum[c % VEC * kThreads + r * lanes + c / VEC];
    DType<DT>::store(out, c, live ? t * a.scale : 0.0f);
  }
}

template <int N> using Const = std::integral_constant<int, N>;

// Whether rows of N heads of width w can be read and written 16 bytes at a time with
// 32-bit offsets, a chunk of them as one resource.
bool fast_view(int dtype, const SeqView& v, int w) {
  const long es = dtype == WM_FP32 ? 4 : 2, per = 16 / es;
  return (w == 32 || w == 64 || w == 128) && (reinterpret_cast<uintptr_t>(v.p) & 15) == 0 && v.t % per == 0 && v.b % per == 0 &&
         v.t >= w && v.t * es < (1L << 31) / (kChunk + 1);
}

template <bool REV, bool STATE>
hipError_t launch_mix(const char* name, int dtype, const MixArgs& m, hipStream_t s) {
  const bool fast = (STATE || (fast_view(dtype, m.a, m.ka) && fast_view(dtype, m.out, m.kc))) && fast_view(dtype, m.b, m.ka) &&
                    fast_view(dtype, m.c, m.kc);
  auto go = [&](auto dt, auto ka, auto kc) {
    typedef decltype(dt) DT;
    const unsigned tiles = (unsigned)((m.kc + kc - 1) / kc);
    const dim3 grid((unsigned)((long)m.B * m.N * m.nseg) * tiles);
    return launch(name, fast ? k_mix<DT, ka, kc, REV, STATE, true> : k_mix<DT, ka, kc, REV, STATE, false>, grid, dim3(kThreads), 0,
                  s, m);
  };
  auto by = [&](auto dt) {
    // few work-groups: two take the halves of a head's columns, both with its weights (T 128 bf16
    // in halves and whole, 64 heads 7.8 and 9.9 us, 256 heads 11.5 and 11.0, 384 heads 15.3 and
    // 13.9; fp32 13.3 and 18.2, 20.7 and 20.2, 26.6 and 28.8)
    const bool half = m.kc <= 32 || (!STATE && (long)m.B * m.N * m.nseg < 256);
    auto cols = [&](auto ka) { return half ? go(dt, ka, Const<32>()) : go(dt, ka, Const<64>()); };
    return m.ka <= 32 ? cols(Const<32>()) : m.ka <= 64 ? cols(Const<64>()) : cols(Const<128>());
  };
  return dtype == WM_FP32 ? by(0.0f) : by(bf16_t());
}

// Sequences, heads and segments up to which the gradient's two sweeps run beside each
// other.  Measured beside and after each other, T 128, heads of 64 bf16: 64 of them 13.9
// and 20.0 us, 384 24.2 and 26.6, 512 31.5 and 27.2; fp32 27.8 and 41.3, 54.3 and 62.0,
// 73.5 and 64.5.
constexpr long kApart = 384;
hipError_t launch_mix_grad(int dtype, const MixArgs& q, const MixArgs& v, const SeqView& dk, hipStream_t s) {
  const int K = v.ka, V = v.kc;
  const bool fast = fast_view(dtype, v.a, K) && fast_view(dtype, v.b, K) && fast_view(dtype, v.c, V) && fast_view(dtype, v.v, V) &&
                    fast_view(dtype, v.out, V) && fast_view(dtype, dk, K) && fast_view(dtype, q.out, K);
  const long places = (long)v.B * v.N * v.nseg;
  const int apart = places <= kApart;
  auto go = [&](auto dt, auto kp, auto vp) {
    typedef decltype(dt) DT;
    return launch("linattn_grad", fast ? k_mix_grad<DT, kp, vp, true> : k_mix_grad<DT, kp, vp, false>,
                  dim3((unsigned)(places << apart)), dim3(kThreads), 0, s, q, v, dk, apart);
  };
  auto by = [&](auto dt) {
    auto cols = [&](auto kp) { return V <= 32 ? go(dt, kp, Const<32>()) : go(dt, kp, Const<64>()); };
    return K <= 32 ? cols(Const<32>()) : cols(Const<64>());
  };
  return dtype == WM_FP32 ? by(0.0f) : by(bf16_t());
}

// Segments of the time axis and the chunks in each: as many as run at a time, three
// work-groups a CU.  Measured, T 32768, 16 heads of 64 bf16, 512, 768, 1024 and 1536
// work-groups: outputs in all 116, 114, 126 and 126 us, gradient 255, 213, 238 and 233.
constexpr long kResident = 768;
struct Split {
  int nseg, per;
};
Split split_of(int T, int B, int N) {
  const int chunks = chunks_of(T);
  const long heads = (long)B * N;
  if (heads == 0 || chunks < 4) return {1, std::max(chunks, 1)};
  const int want = (int)std::max(1L, std::min<long>(chunks / 2, kResident / heads));
  const int per = (chunks + want - 1) / want;
  return {(chunks + per - 1) / per, per};
}
size_t align256(size_t n) { return (n + 255) / 256 * 256; }
size_t seg_bytes(long heads, int nseg, int K, int V) { return align256((size_t)heads * nseg * K * V * sizeof(float)); }

template <bool REV>
hipError_t segments(int dtype, MixArgs m, float* s1, hipStream_t s) {
  const float* s0 = m.s0;
  m.s0 = nullptr;
  m.s1 = nullptr;
  hipError_t e = launch_mix<REV, true>("linattn_state", dtype, m, s);
  if (e != hipSuccess) return e;
  const int width = m.ka * m.kc;
  return launch("linattn_segments", k_segments<REV>, dim3((width + kThreads - 1) / kThreads, (unsigned)(m.B * m.N)),
                dim3(kThreads), 0, s, m.seg, m.hold, s0, s1, m.nseg, width);
}

}  // namespace

size_t linattn_states(int T, int B, int N, int K, int V) {
  const Split sp = split_of(T, B, N);
  return sp.nseg > 1 ? seg_bytes((long)B * N, sp.nseg, K, V) : 0;
}
size_t linattn_workspace(int T, int B, int N, int K, int V) {
  const Split sp = split_of(T, B, N);
  const long heads = (long)B * N;
  return sp.nseg > 1 ? seg_bytes(heads, sp.nseg, K, V) + align256((size_t)heads * sp.nseg * sizeof(float)) : 0;
}

hipError_t launch_linattn(int dtype, const LinattnArgs& a, hipStream_t s) {
  if (a.T == 1) {
    auto step = [&](auto dt) {
      typedef decltype(dt) DT;
      const bool wide = a.V % 4 == 0 && ((reinterpret_cast<uintptr_t>(a.h0) | reinterpret_cast<uintptr_t>(a.h_T)) & 15) == 0;
      int lanes = 1;
      while (lanes * (wide ? 4 : 1) < a.V) lanes *= 2;
      return launch("linattn_step", wide ? k_linattn_step<DT, 4> : k_linattn_step<DT, 1>, dim3((unsigned)(a.B * a.N)),
                    dim3(kThreads), 0, s, a, lanes);
    };
    return dtype == WM_FP32 ? step(0.0f) : step(bf16_t());
  }
  const Split sp = split_of(a.T, a.B, a.N);
  const long heads = (long)a.B * a.N;
  MixArgs m{a.T, a.B, a.N, a.K, a.V, a.q, a.k, a.v, SeqView{a.y, (long)a.B * a.N * a.V, (long)a.N * a.V}, {}, a.decay,
            a.scale, a.scale, 1.0f, a.h0, a.h_T, a.V, 1, a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  if (sp.nseg > 1) {
    const size_t own = seg_bytes(heads, sp.nseg, a.K, a.V);
    m.seg = a.states ? a.states : reinterpret_cast<float*>(a.ws);
    m.hold = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + own);
    const hipError_t e = segments<false>(dtype, m, a.h_T, s);
    if (e != hipSuccess) return e;
  }
  return launch_mix<false, false>("linattn", dtype, m, s);
}

hipError_t launch_linattn_grad(int dtype, const LinattnGradArgs& a, hipStream_t s) {
  const Split sp = split_of(a.T, a.B, a.N);
  const long heads = (long)a.B * a.N;
  // the state and its transpose: [K][V] with strides (V, 1) of rows and columns, or (1, V)
  MixArgs dq{a.T, a.B, a.N, a.V, a.K, a.dy, a.v, a.k, a.dq, {}, a.decay, a.scale, a.scale, 1.0f, a.h0, nullptr, 1, a.V,
             a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  MixArgs dv{a.T, a.B, a.N, a.K, a.V, a.k, a.q, a.dy, a.dv, a.v, a.decay, a.scale, 1.0f, a.scale, a.dh_T, a.dh0, a.V, 1,
             a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  MixArgs dk{a.T, a.B, a.N, a.V, a.K, a.v, a.dy, a.q, a.dk, {}, a.decay, a.scale, 1.0f, a.scale, a.dh_T, nullptr, 1, a.V,
             a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  hipError_t e;
  if (sp.nseg > 1) {
    dq.seg = const_cast<float*>(a.states);
    dv.seg = dk.seg = reinterpret_cast<float*>(a.ws);
    dv.hold = reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + seg_bytes(heads, sp.nseg, a.K, a.V));
    if ((e = segments<true>(dtype, dv, a.dh0, s)) != hipSuccess) return e;
  }
  if (a.K <= 64 && a.V <= 64) return launch_mix_grad(dtype, dq, dv, a.dk, s);
  if ((e = launch_mix<false, false>("linattn_dq", dtype, dq, s)) != hipSuccess) return e;
  if ((e = launch_mix<true, false>("linattn_dk", dtype, dk, s)) != hipSuccess) return e;
  return launch_mix<true, false>("linattn_dv", dtype, dv, s);
}

}  // namespace wm
