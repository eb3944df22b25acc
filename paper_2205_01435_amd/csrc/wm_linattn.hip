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
// what is left of them at its end.  A work-group goes through the chunks of one
// head with the state in registers.  Where sequences and heads are too few to fill
// the device, the time axis is split into segments: a first launch sums up each
// segment's own state, a second one runs through them, and the main launch starts
// every segment from the state that enters it.
//
// Precision: fp32 values multiply on the fp32 matrix instructions.  bf16 values
// enter exactly; the 64 x 64 weights and the state that meets the rows are held as
// two bf16 terms each (2^-17 of their value is left out, against the 2^-9 of the
// output's rounding), and the sources times their weights, which make up the fp32
// state, as three (2^-24).  All sums are fp32.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_attend.h"
#include "wm_profile.h"
#include "wm_split.h"

namespace wm {
namespace {

constexpr int kChunk = 64;
constexpr int kThreads = 256;  // four waves, 16 of a chunk's rows each

struct MixArgs {
  int T, B, N;
  int ka, kc;  // widths of A and B, and of C and the output
  SeqView a, b, c, out;
  const float* decay;
  float s_intra, s_inter, s_upd;  // factors of the chunk's own part, the state's, and of sources on their way into it
  const float* s0;  // [B, N, ka, kc] with the strides below, or null (0)
  float* s1;        // the state that leaves, or null
  int st_a, st_c;   // the states' strides
  const uint8_t* resets;
  const int32_t* lengths;
  int nseg, per;   // segments, and chunks in each
  float* seg;      // [B N][nseg][ka][kc]: what enters each segment (state launch: its own sum, with strides st_a, st_c)
  float* hold;     // [B N][nseg] state launch: what a segment leaves of the state that enters it
};

template <typename DT> struct Tile;
template <> struct Tile<bf16_t> {
  static constexpr int VEC = 8, PAD = 8, SLICE = 32, PLANES = 2;
};
template <> struct Tile<float> {
  static constexpr int VEC = 4, PAD = 4, SLICE = 16, PLANES = 1;
};

typedef uint32_t __attribute__((ext_vector_type(4))) v4u;
typedef uint32_t __attribute__((ext_vector_type(2))) v2u;
typedef v4u __attribute__((aligned(2))) v4u_2;
typedef v4u __attribute__((aligned(4))) v4u_4;
typedef v2u __attribute__((aligned(2))) v2u_2;
template <typename DT> struct Mem16;
template <> struct Mem16<float> { typedef v4u_4 type; };
template <> struct Mem16<bf16_t> { typedef v4u_2 type; };

// 16 bytes of a row from column c on, zeros past its `width`.
template <typename DT>
__device__ __forceinline__ v4u load_piece(const DT* row, int c, int width) {
  constexpr int V = Tile<DT>::VEC;
  if (c + V <= width) return *reinterpret_cast<const typename Mem16<DT>::type*>(row + c);
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
// Four rows of one column from a row-major bf16 matrix in LDS: sixteen lanes read
// four rows of sixteen columns, four values each (p: row j / 4, columns 4 (j % 4)
// on, j the lane of the sixteen), and get column j.
__device__ __forceinline__ v2u read_tr(const bf16_t* p) {
  typedef __attribute__((address_space(3))) s16x4* lds_t;
  return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)p));
}
__device__ __forceinline__ bf16x8 join(v2u a, v2u b) { return __builtin_bit_cast(bf16x8, v4u{a.x, a.y, b.x, b.y}); }

// a^n from log2 a, 1 for n = 0 also where a = 0.
__device__ __forceinline__ float decayed(float la, int n) { return n > 0 ? __builtin_amdgcn_exp2f(la * (float)n) : 1.0f; }

template <typename DT, int KA, int KC, bool REV, bool STATE>
__global__ void __launch_bounds__(kThreads) k_mix(const MixArgs a) {
  constexpr int V = Tile<DT>::VEC, SL = Tile<DT>::SLICE, PL = Tile<DT>::PLANES;
  constexpr bool F32 = sizeof(DT) == 4;
  constexpr int PA = KA + Tile<DT>::PAD, PC = KC + Tile<DT>::PAD;  // pitches in LDS
  constexpr int AB = kChunk * (KA / V) / kThreads, CB = kChunk * (KC / V) / kThreads;  // pieces a thread stages
  static_assert(AB > 0 && CB > 0, "a piece or more for every thread");
  constexpr int WK = KA >= 64 ? 4 : 2, WC = 4 / WK;      // waves over the state's rows and columns
  constexpr int KAB = KA / 16 / WK, KCB = KC / 16 / WC;  // its 16 x 16 blocks in a wave
  __shared__ __align__(16) DT bl[kChunk * PA];
  __shared__ __align__(16) DT cl[kChunk * PC];
  __shared__ __align__(16) DT st[STATE ? 16 : PL * KC * PA];  // the state, columns first

  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, g = lane >> 4, j16 = lane & 15;
  const int nct = (a.kc + KC - 1) / KC;
  const int ct = blockIdx.x % nct * KC;
  const long part = blockIdx.x / nct;  // (sequence and head, segment)
  const int seg = (int)(part % a.nseg);
  const long bn = part / a.nseg;
  const int n = (int)(bn % a.N), b = (int)(bn / a.N);
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const float da = fminf(fmaxf(a.decay[n], 0.0f), 1.0f), la = log2f(da);
  const int chunks = (a.T + kChunk - 1) / kChunk, first = seg * a.per, last = min(first + a.per, chunks);
  const int wcols = min(KC, a.kc - ct);
  const DT* const pa = reinterpret_cast<const DT*>(a.a.p) + (long)b * a.a.b + (long)n * a.ka;
  const DT* const pb = reinterpret_cast<const DT*>(a.b.p) + (long)b * a.b.b + (long)n * a.ka;
  const DT* const pc = reinterpret_cast<const DT*>(a.c.p) + (long)b * a.c.b + (long)n * a.kc + ct;

  v4u rb[AB], rc[CB], ra[KA / SL];
  const int r = 16 * w + j16;  // this lane's row of a chunk
  auto load = [&](int c) {
    const int t0 = c * kChunk, live = len - t0;
#pragma unroll
    for (int i = 0; i < AB; ++i) {
      const int p = tid + i * kThreads, s = p / (KA / V);
      rb[i] = s < live ? load_piece<DT>(pb + (long)(t0 + s) * a.b.t, p % (KA / V) * V, a.ka) : v4u{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < CB; ++i) {
      const int p = tid + i * kThreads, s = p / (KC / V);
      rc[i] = s < live ? load_piece<DT>(pc + (long)(t0 + s) * a.c.t, p % (KC / V) * V, wcols) : v4u{0, 0, 0, 0};
    }
    if constexpr (!STATE) {
#pragma unroll
      for (int i = 0; i < KA / SL; ++i)
        ra[i] = r < live ? load_piece<DT>(pa + (long)(t0 + r) * a.a.t, i * SL + V * g, a.ka) : v4u{0, 0, 0, 0};
    }
  };
  auto stage = [&]() {
#pragma unroll
    for (int i = 0; i < AB; ++i) {
      const int p = tid + i * kThreads;
      *reinterpret_cast<v4u*>(bl + p / (KA / V) * PA + p % (KA / V) * V) = rb[i];
    }
#pragma unroll
    for (int i = 0; i < CB; ++i) {
      const int p = tid + i * kThreads;
      *reinterpret_cast<v4u*>(cl + p / (KC / V) * PC + p % (KC / V) * V) = rc[i];
    }
  };

  // the state's blocks of this wave: rows 16 (wk KAB + i) + 4 g + 0..3, column 16 (wc KCB + k) + j16
  const int wk = w % WK, wc = w / WK;
  f32x4 S[KAB][KCB];
  const float* const s0 = a.seg && !STATE ? a.seg + part * a.ka * a.kc : a.s0 && !STATE ? a.s0 + bn * a.ka * a.kc : nullptr;
#pragma unroll
  for (int i = 0; i < KAB; ++i)
#pragma unroll
    for (int k = 0; k < KCB; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 16 * (wk * KAB + i) + 4 * g + e, col = 16 * (wc * KCB + k) + j16;
        S[i][k][e] = s0 && row < a.ka && col < wcols ? s0[(long)row * a.st_a + (long)(ct + col) * a.st_c] : 0.0f;
      }
  auto stage_state = [&]() {
    if constexpr (!STATE) {
#pragma unroll
      for (int i = 0; i < KAB; ++i)
#pragma unroll
        for (int k = 0; k < KCB; ++k) {
          DT* const p = st + (16 * (wc * KCB + k) + j16) * PA + 16 * (wk * KAB + i) + 4 * g;
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
  };

  // a^|r - s| for the sources s = 16 j + 4 g + e of the lane's row
  float wt[4][4];
  if constexpr (!STATE) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) wt[j][e] = a.s_intra * decayed(la, abs(r - (16 * j + 4 * g + e)));
  }

  float hold_all = 1.0f;
  if (first < last) load(REV ? last - 1 : first);
  for (int step = 0; step < last - first; ++step) {
    const int c = REV ? last - 1 - step : first + step, t0 = c * kChunk;
    const int live = min(len - t0, kChunk);  // steps of the chunk inside the sequence, 0 or less for none
    uint64_t starts = 0;
    if (a.resets) {
      const bool one = lane < live && a.resets[(long)(t0 + lane) * a.B + b] != 0;
      starts = __ballot(one);
    }
    __syncthreads();  // the chunk before is done with
    stage();
    stage_state();
    v4u now[KA / SL];
    if constexpr (!STATE) {
#pragma unroll
      for (int i = 0; i < KA / SL; ++i) now[i] = ra[i];
    }
    if (step + 1 < last - first) load(REV ? c - 1 : c + 1);
    __syncthreads();

    if constexpr (!STATE) {
      // the sources [lo, hi] of the row, and whether the entering state reaches it
      const uint64_t upto = ~0ull >> (63 - r);
      const uint64_t cut = REV ? starts & ~upto : starts & upto;
      const int lo = REV ? r : cut ? 63 - __clzll((long long)cut) : 0;
      const int hi = REV ? (cut ? __ffsll((long long)cut) - 2 : live - 1) : r;
      const int dist = REV ? live - 1 - r : r + 1;
      const float win = cut == 0 ? a.s_inter * decayed(la, dist) : 0.0f;
      DT* const orow = reinterpret_cast<DT*>(const_cast<void*>(a.out.p)) + (long)(t0 + r) * a.out.t + (long)b * a.out.b +
                       (long)n * a.kc + ct;
      float P[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        if ((REV ? j >= w : j <= w) && live > 0) {
#pragma unroll
          for (int k = 0; k < KA / SL; ++k) {
            const v4u x = *reinterpret_cast<const v4u*>(bl + (16 * j + j16) * PA + k * SL + V * g);
            Mfma<DT>::step(acc, make_uint4(x.x, x.y, x.z, x.w), make_uint4(now[k].x, now[k].y, now[k].z, now[k].w));
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int s = 16 * j + 4 * g + e;
          P[j][e] = s >= lo && s <= hi ? acc[e] * wt[j][e] : 0.0f;
        }
      }
      bf16x8 ph[2], pm[2];
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
#pragma unroll
      for (int cb = 0; cb < KC / 16; ++cb) {
        if (16 * cb >= wcols) break;
        f32x4 in = {0.f, 0.f, 0.f, 0.f}, out = {0.f, 0.f, 0.f, 0.f};
        if (live > 0) {
#pragma unroll
          for (int k = 0; k < KA / SL; ++k) {
            const uint4 y = make_uint4(now[k].x, now[k].y, now[k].z, now[k].w);
#pragma unroll
            for (int p = PL - 1; p >= 0; --p) {
              const v4u x = *reinterpret_cast<const v4u*>(st + (p * KC + 16 * cb + j16) * PA + k * SL + V * g);
              Mfma<DT>::step(in, make_uint4(x.x, x.y, x.z, x.w), y);
            }
          }
          if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (REV ? j < w : j > w) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                out = __builtin_amdgcn_mfma_f32_16x16x4f32(cl[(16 * j + 4 * g + e) * PC + 16 * cb + j16], P[j][e], out, 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              if (REV ? 2 * jj + 1 < w : 2 * jj > w) continue;
              const bf16_t* const p = cl + (32 * jj + 4 * g + j16 / 4) * PC + 16 * cb + 4 * (j16 % 4);
              const bf16x8 x = join(read_tr(p), read_tr(p + 16 * PC));
              out = mfma_bf16(x, pm[jj], out);
              out = mfma_bf16(x, ph[jj], out);
            }
          }
        }
        if (t0 + r >= a.T) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r < live ? out[e] + (cut == 0 ? win * in[e] : 0.0f) : 0.0f;
        const int col = 16 * cb + 4 * g;
        if (col + 4 <= wcols) {
          if constexpr (F32)
            *reinterpret_cast<v4u_4*>(orow + col) =
                v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
          else
            *reinterpret_cast<v2u_2*>(orow + col) = v2u{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < wcols) DType<DT>::store(orow, col + e, v[e]);
        }
      }
    }

    if (live <= 0) continue;
    // what the state keeps, and the sources [lo, hi] that it takes in
    const float hold = starts ? 0.0f : decayed(la, live);
    const int lo = REV ? 0 : starts ? 63 - __clzll((long long)starts) : 0;
    const int hi = REV ? (starts ? __ffsll((long long)starts) - 2 : live - 1) : live - 1;
    if constexpr (STATE) hold_all = starts ? 0.0f : hold_all * hold;
#pragma unroll
    for (int i = 0; i < KAB; ++i)
#pragma unroll
      for (int k = 0; k < KCB; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[i][k][e] = starts ? 0.0f : S[i][k][e] * hold;
    auto taken = [&](int s) {
      return s >= lo && s <= hi ? a.s_upd * decayed(la, REV ? s + 1 : live - 1 - s) : 0.0f;
    };
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      float ws[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) ws[e] = taken(32 * jj + 16 * (e / 4) + 4 * g + e % 4);
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int s = 32 * jj + 16 * (e / 4) + 4 * g + e % 4;
          float x[KAB];
#pragma unroll
          for (int i = 0; i < KAB; ++i) {
            const float v = bl[s * PA + 16 * (wk * KAB + i) + j16];
            x[i] = ws[e] != 0.0f ? v * ws[e] : 0.0f;
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
            f[2 * e] = ws[2 * e] != 0.0f ? __uint_as_float(u[e] << 16) * ws[2 * e] : 0.0f;
            f[2 * e + 1] = ws[2 * e + 1] != 0.0f ? __uint_as_float(u[e] & 0xffff0000u) * ws[2 * e + 1] : 0.0f;
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

  float* const s1 = STATE ? a.seg + part * a.ka * a.kc : a.seg || !a.s1 ? nullptr : a.s1 + bn * a.ka * a.kc;
  if (s1) {
#pragma unroll
    for (int i = 0; i < KAB; ++i)
#pragma unroll
      for (int k = 0; k < KCB; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 16 * (wk * KAB + i) + 4 * g + e, col = 16 * (wc * KCB + k) + j16;
          if (row < a.ka && col < wcols) s1[(long)row * a.st_a + (long)(ct + col) * a.st_c] = S[i][k][e];
        }
  }
  if constexpr (STATE) {
    if (tid == 0 && ct == 0) a.hold[part] = hold_all;
  }
}

// Runs through the segments' own sums: seg[i] becomes the state that enters it.
// One value of a head's state a thread.
template <bool REV>
__global__ void __launch_bounds__(kThreads) k_segments(float* seg, const float* hold, const float* s0, float* s1, int nseg,
                                                       int width) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  const long bn = blockIdx.y;
  if (i >= width) return;
  float s = s0 ? s0[bn * width + i] : 0.0f;
  float* p = seg + bn * nseg * (long)width + i;
  const float* h = hold + bn * nseg;
#pragma unroll 8
  for (int k = 0; k < nseg; ++k) {
    const int m = REV ? nseg - 1 - k : k;
    const float own = p[(long)m * width], f = h[m];
    p[(long)m * width] = s;
    s = f != 0.0f ? fmaf(f, s, own) : own;
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

template <bool REV, bool STATE>
hipError_t launch_mix(const char* name, int dtype, const MixArgs& m, hipStream_t s) {
  auto go = [&](auto dt, auto ka, auto kc) {
    typedef decltype(dt) DT;
    const unsigned tiles = (unsigned)((m.kc + kc - 1) / kc);
    return launch(name, k_mix<DT, ka, kc, REV, STATE>, dim3((unsigned)((long)m.B * m.N * m.nseg) * tiles), dim3(kThreads), 0,
                  s, m);
  };
  auto by = [&](auto dt) {
    auto cols = [&](auto ka) { return m.kc <= 32 ? go(dt, ka, Const<32>()) : go(dt, ka, Const<64>()); };
    return m.ka <= 32 ? cols(Const<32>()) : m.ka <= 64 ? cols(Const<64>()) : cols(Const<128>());
  };
  return dtype == WM_FP32 ? by(0.0f) : by(bf16_t());
}

// Segments of the time axis and the chunks in each.
struct Split {
  int nseg, per;
};
Split split_of(int T, int B, int N) {
  const int chunks = (T + kChunk - 1) / kChunk;
  const long heads = (long)B * N;
  if (heads == 0 || heads >= 512 || chunks < 4) return {1, std::max(chunks, 1)};
  const int want = (int)std::min<long>(chunks / 2, (1024 + heads - 1) / heads);
  const int per = (chunks + want - 1) / want;
  return {(chunks + per - 1) / per, per};
}
size_t seg_bytes(long heads, int nseg, int K, int V) {
  return ((size_t)heads * nseg * K * V * sizeof(float) + 255) / 256 * 256 + ((size_t)heads * nseg * sizeof(float) + 255) / 256 * 256;
}
void place(MixArgs& m, void* ws, long heads, int K, int V) {
  m.seg = reinterpret_cast<float*>(ws);
  m.hold = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + ((size_t)heads * m.nseg * K * V * sizeof(float) + 255) / 256 * 256);
}

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

size_t linattn_workspace(int T, int B, int N, int K, int V) {
  const Split sp = split_of(T, B, N);
  return sp.nseg > 1 ? seg_bytes((long)B * N, sp.nseg, K, V) : 0;
}
size_t linattn_grad_workspace(int T, int B, int N, int K, int V) { return 2 * linattn_workspace(T, B, N, K, V); }

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
  MixArgs m{a.T, a.B, a.N, a.K, a.V, a.q, a.k, a.v, SeqView{a.y, (long)a.B * a.N * a.V, (long)a.N * a.V}, a.decay,
            a.scale, a.scale, 1.0f, a.h0, a.h_T, a.V, 1, a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  if (sp.nseg > 1) {
    place(m, a.ws, heads, a.K, a.V);
    const hipError_t e = segments<false>(dtype, m, a.h_T, s);
    if (e != hipSuccess) return e;
  }
  return launch_mix<false, false>("linattn", dtype, m, s);
}

hipError_t launch_linattn_grad(int dtype, const LinattnGradArgs& a, hipStream_t s) {
  const Split sp = split_of(a.T, a.B, a.N);
  const long heads = (long)a.B * a.N;
  // the state and its transpose: [K][V] with strides (V, 1) of rows and columns, or (1, V)
  MixArgs dq{a.T, a.B, a.N, a.V, a.K, a.dy, a.v, a.k, a.dq, a.decay, a.scale, a.scale, 1.0f, a.h0, nullptr, 1, a.V,
             a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  MixArgs dv{a.T, a.B, a.N, a.K, a.V, a.k, a.q, a.dy, a.dv, a.decay, a.scale, 1.0f, a.scale, a.dh_T, a.dh0, a.V, 1,
             a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  MixArgs dk{a.T, a.B, a.N, a.V, a.K, a.v, a.dy, a.q, a.dk, a.decay, a.scale, 1.0f, a.scale, a.dh_T, nullptr, 1, a.V,
             a.resets, a.lengths, sp.nseg, sp.per, nullptr, nullptr};
  hipError_t e;
  if (sp.nseg > 1) {
    char* ws = reinterpret_cast<char*>(a.ws);
    place(dq, ws, heads, a.K, a.V);
    place(dv, ws + seg_bytes(heads, sp.nseg, a.K, a.V), heads, a.K, a.V);
    place(dk, ws + seg_bytes(heads, sp.nseg, a.K, a.V), heads, a.K, a.V);
    if ((e = segments<false>(dtype, dq, nullptr, s)) != hipSuccess) return e;
    if ((e = segments<true>(dtype, dv, a.dh0, s)) != hipSuccess) return e;
  }
  if ((e = launch_mix<false, false>("linattn_dq", dtype, dq, s)) != hipSuccess) return e;
  if ((e = launch_mix<true, false>("linattn_dk", dtype, dk, s)) != hipSuccess) return e;
  return launch_mix<true, false>("linattn_dv", dtype, dv, s);
}

}  // namespace wm
