// Norm of every head's queries and keys and their rotation by position, and the
// gradient:
//   r = (mean x^2 + eps)^-1/2, y = Rot(x r gamma);
//   d = Rot^-1 dy, e = d gamma, dx = r (e - x r mean(e x r)), dgamma = sum d x r.
// Rot turns pair i of a head by the angle pos f_i.
//
// The angle as a part of a turn is pos times the table's 64-bit binary fraction,
// modulo 2^64: exact for every position.  Its nearest quarter turn goes into
// signs and order, and what is left, at most an eighth of a turn either side, into
// the Taylor sums of sine and cosine, whose first terms left out are below 2e-9.
//
// A lane holds whole pairs of a head: VEC pairs (8 bf16 or 4 fp32), two pieces of
// 16 bytes, and L lanes hold a head, so that the rotation needs no other lane and
// the sum goes over L lanes.  It computes its pairs' sines and cosines once for a
// step and goes through the step's heads with them; where there are few steps the
// heads are dealt to several lane groups.  The gradient keeps the sums for both
// gammas in registers; a work-group leaves one row of partial sums, which a second
// launch adds in order.
//
// Bound by memory.  Measured, the least and the mean of twelve calls one after the other:
// 65536 rows, 16 heads of 64 fp32 93 and 99 us (5.8 and 5.4 TB/s), gradient 151 and 155
// (5.3 and 5.2); 204800 rows, 20 heads of 64 bf16 204 and 215 us (5.1 and 4.9 TB/s),
// gradient 312 and 326 (5.0 and 4.8); 4500 rows, 9 heads of 61 fp32 10 and 12 us and 4 for
// the sums, their launches and first loads.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_attend.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr long kGroups = 1 << 20;  // work-groups at most, far more than run at a time

template <typename DT> struct Io;
template <> struct Io<float> {
  static constexpr int VEC = 4;
  __device__ static void get(v4u r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
  }
  __device__ static v4u put(const float* v) {
    return v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
template <> struct Io<bf16_t> {
  static constexpr int VEC = 8;
  __device__ static void get(v4u r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  __device__ static v4u put(const float* v) {
    return v4u{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
  }
};

// (cos, sin) of a part of a turn, a 64-bit binary fraction.
__device__ __forceinline__ float2 cos_sin(uint64_t turn) {
  const uint32_t t = (uint32_t)(turn >> 32), quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int)(t - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi 2^-32
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f), 8.3333333333e-3f), -1.6666666667e-1f), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f), -1.3888888889e-3f), 4.1666666667e-2f), -0.5f), 1.0f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter & 2 ? -b : b);
}

template <int CTRL>
__device__ __forceinline__ float dpp_plus(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over L neighbouring lanes, in every one of them.
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (L >= 2) v = dpp_plus<0xB1>(v);   // quad_perm 1 0 3 2
  if constexpr (L >= 4) v = dpp_plus<0x4E>(v);   // quad_perm 2 3 0 1
  if constexpr (L >= 8) v = dpp_plus<0x141>(v);  // row_half_mirror
  if constexpr (L >= 16) v = dpp_plus<0x140>(v); // row_mirror
  if constexpr (L >= 32) v += __shfl_xor(v, 16);
  if constexpr (L >= 64) v += __shfl_xor(v, 32);
  return v;
}

// A lane's pairs of a head, v[0] and v[1] their first and second values, as two pieces
// of VEC neighbouring values.  Neighbours: the pieces follow each other, and pairs are
// put together from them.  Halves: the lanes of the rotated pairs come first, a piece
// from each half of the R values; then those of the rest, whose halves are taken as
// pairs that do not turn (the second one may lack the last).  WHOLE: every piece of
// every lane is full.  Others are loaded from where 16 bytes of the head are left and
// moved and cut when they are used: a branch at each load would make each wait for the
// one before (4500 rows, 9 heads of 61 fp32 11.6 -> 10.4 us, gradient 13.7 -> 11.9).
template <typename DT, bool WHOLE>
struct Lane {
  static constexpr int V = Io<DT>::VEC;
  int at[2], n[2];   // where the pieces start, and their values
  int end[2];        // what a piece may be read up to
  int from[2];       // and where its load starts, -1 where the head is shorter than one
  int turn0, turns;  // the first pair's place in the table, and how many pairs turn
  bool neighbours;
  __device__ Lane(const QkArgs& a, int lane) : neighbours(a.neighbours != 0) {
    const int R2 = a.R / 2, first = (R2 + V - 1) / V, rest = (a.D - a.R + 1) / 2;
    if (neighbours) {
      at[0] = 2 * V * lane;
      at[1] = at[0] + V;
      end[0] = end[1] = a.D;
      turn0 = V * lane;
      turns = min(max(R2 - turn0, 0), V);
    } else if (lane < first) {
      at[0] = turn0 = V * lane;
      at[1] = R2 + at[0];
      end[0] = R2;
      end[1] = a.R;
      turns = min(R2 - turn0, V);
    } else {
      at[0] = a.R + V * (lane - first);
      at[1] = at[0] + rest;
      end[0] = a.R + rest;
      end[1] = a.D;
      turn0 = turns = 0;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      n[i] = min(max(end[i] - at[i], 0), V);
      from[i] = a.D < V ? -1 : min(at[i], a.D - V);
    }
  }
  __device__ void load(v4u (&r)[2], const DT* x) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (WHOLE)
        r[i] = *reinterpret_cast<const typename Mem16<DT>::type*>(x + (n[0] ? at[i] : 0));
      else if (from[i] < 0)
        r[i] = load_piece<DT>(x, at[i], end[i]);
      else
        r[i] = *reinterpret_cast<const typename Mem16<DT>::type*>(x + from[i]);
    }
  }
  // the pieces as pairs
  __device__ void get(const v4u (&r)[2], float (&v)[2][V]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (WHOLE || from[i] < 0 || n[i] == V) {
        Io<DT>::get(r[i], v[i]);
      } else {
        Io<DT>::get(elements_from<DT>(r[i], at[i] - from[i]), v[i]);
#pragma unroll
        for (int k = 0; k < V; ++k) v[i][k] = k < n[i] ? v[i][k] : 0.0f;
      }
    }
    if (neighbours) order<true>(v);
    if (WHOLE && n[0] == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[0][i] = v[1][i] = 0.0f;
    }
  }
  // 2 V values in memory order, as V first and V second ones, and back
  template <bool TO>
  __device__ static void order(float (&v)[2][V]) {
    float w[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (TO) {
        w[2 * i] = v[2 * i / V][2 * i % V];
        w[2 * i + 1] = v[(2 * i + 1) / V][(2 * i + 1) % V];
      } else {
        w[2 * i] = v[0][i];
        w[2 * i + 1] = v[1][i];
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[0][i] = TO ? w[2 * i] : w[i];
      v[1][i] = TO ? w[2 * i + 1] : w[V + i];
    }
  }
  __device__ void store(DT* x, float (&v)[2][V]) const {
    if (neighbours) order<false>(v);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (n[i] == V) {
        *reinterpret_cast<typename Mem16<DT>::type*>(x + at[i]) = Io<DT>::put(v[i]);
      } else if constexpr (!WHOLE) {
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (k < n[i]) DType<DT>::store(x, at[i] + k, v[i][k]);
      }
    }
  }
  // the column of value j (0 first, 1 second) of pair i, -1 where there is none
  __device__ int column(int j, int i) const {
    const int k = neighbours ? 2 * i + j : j * V + i, piece = k / V, in = k % V;
    return in < (piece ? n[1] : n[0]) ? (piece ? at[1] : at[0]) + in : -1;
  }
  // the lane's values of a [D] array (1 without one, 0 where there is no value)
  __device__ void columns(float (&g)[2][V], const float* a) const {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = column(j, i);
        const float v = a ? a[max(c, 0)] : 1.0f;
        g[j][i] = c < 0 ? 0.0f : v;
      }
  }
  __device__ void angles(float (&c)[V], float (&s)[V], const QkArgs& a, int32_t position) const {
    const uint64_t pos = (uint64_t)(int64_t)position;
    if (a.R == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) c[i] = 1.0f, s[i] = 0.0f;
      return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 t = cos_sin(pos * a.table[min(turn0 + i, a.R / 2 - 1)]);
      c[i] = i < turns ? t.x : 1.0f;
      s[i] = i < turns ? t.y : 0.0f;
    }
  }
};

// An item is every `parts`-th head of one step from head item % parts on, so that
// neighbouring lane groups are at neighbouring heads; heads count through queries,
// then keys.
template <typename DT, int L, bool WHOLE>
__global__ void __launch_bounds__(kThreads) k_qk_norm(const QkArgs a) {
  constexpr int V = Io<DT>::VEC, kSlots = kThreads / L;
  const Lane<DT, WHOLE> lane(a, threadIdx.x % L);
  const int heads = a.side[0].heads + a.side[1].heads, parts = a.parts;
  const uint32_t items = (uint32_t)a.rows * (uint32_t)parts;  // (31 bits)
  const float inv = 1.0f / (float)a.D;
  for (uint32_t item = blockIdx.x * kSlots + threadIdx.x / L; item < items; item += gridDim.x * kSlots) {
    const long row = item / (uint32_t)parts;
    const int h0 = (int)(item % (uint32_t)parts);
    auto in = [&](int h) {
      const int w = h >= a.side[0].heads;
      return reinterpret_cast<const DT*>(a.side[w].x) + row * a.side[w].x_ld + (long)(h - (w ? a.side[0].heads : 0)) * a.D;
    };
    v4u next[2];
    lane.load(next, in(h0));
    float c[V], s[V], g[2][V];
    lane.angles(c, s, a, a.pos[row]);
    int held = -1;
    for (int h = h0; h < heads; h += parts) {
      const int w = h >= a.side[0].heads;
      if (w != held) lane.columns(g, a.side[held = w].gamma);
      float v[2][V];
      lane.get(next, v);
      if (h + parts < heads) lane.load(next, in(h + parts));
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaf(v[0][i], v[0][i], fmaf(v[1][i], v[1][i], m));
      const float r = 1.0f / sqrtf(group_sum<L>(m) * inv + a.eps);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float x0 = v[0][i] * r * g[0][i], x1 = v[1][i] * r * g[1][i];
        v[0][i] = fmaf(x0, c[i], -(x1 * s[i]));
        v[1][i] = fmaf(x0, s[i], x1 * c[i]);
      }
      lane.store(reinterpret_cast<DT*>(a.side[w].out) + row * a.side[w].out_ld + (long)(h - (w ? a.side[0].heads : 0)) * a.D, v);
    }
  }
}

// The first groups[0] work-groups take the queries, the others the keys: sums for one
// gamma are half the registers of those for both (4500 rows, 9 heads of 61 fp32
// 19.4 -> 13.5 us).  part [groups][D]: each work-group's sums; where a side has only one,
// they are the result.
// Two waves a SIMD for bf16, whose 172 registers three do not admit without spills (204800
// rows, 20 heads of 64 320 and 307 us).
template <typename DT, int L, bool WHOLE>
__global__ void __launch_bounds__(kThreads, WHOLE && sizeof(DT) == 4 ? 3 : 2) k_qk_norm_grad(const QkArgs a) {
  constexpr int V = Io<DT>::VEC, kSlots = kThreads / L;
  __shared__ float add[2 * V][kThreads + 1];
  const int which = (int)blockIdx.x >= a.groups[0], group = (int)blockIdx.x - (which ? a.groups[0] : 0);
  const QkSide& side = a.side[which];
  const Lane<DT, WHOLE> lane(a, threadIdx.x % L);
  const uint32_t parts = (uint32_t)min(a.parts, max(side.heads, 1)), items = (uint32_t)a.rows * parts;
  const float inv = 1.0f / (float)a.D;
  float g[2][V], dg[2][V];
  lane.columns(g, side.gamma);
#pragma unroll
  for (int i = 0; i < V; ++i) dg[0][i] = dg[1][i] = 0.0f;
  const uint32_t stride = (uint32_t)a.groups[which] * kSlots;
  uint32_t item = (uint32_t)group * kSlots + threadIdx.x / L;
  if (side.heads == 0) item = items;
  v4u nx[2], nd[2];
  // an item's first pieces are requested while the item before is worked on
  auto first = [&](uint32_t it) {
    const uint32_t row = it / parts;
    const long h = (long)(it - row * parts) * a.D;
    lane.load(nx, reinterpret_cast<const DT*>(side.x) + (long)row * side.x_ld + h);
    lane.load(nd, reinterpret_cast<const DT*>(side.dout) + (long)row * side.dout_ld + h);
    return a.pos[row];
  };
  int32_t pos = item < items ? first(item) : 0;
  for (; item < items; item += stride) {
    const uint32_t row = item / parts;
    const int h0 = (int)(item - row * parts), step = (int)parts * a.D;
    const DT* x = reinterpret_cast<const DT*>(side.x) + (long)row * side.x_ld + (long)h0 * a.D;
    const DT* dy = reinterpret_cast<const DT*>(side.dout) + (long)row * side.dout_ld + (long)h0 * a.D;
    DT* out = reinterpret_cast<DT*>(side.out) + (long)row * side.out_ld + (long)h0 * a.D;
    float c[V], s[V];
    lane.angles(c, s, a, pos);
    for (int h = h0; h < side.heads; h += (int)parts, out += step) {
      float v[2][V], d[2][V];
      lane.get(nx, v);
      lane.get(nd, d);
      if (h + (int)parts < side.heads) {
        x += step;
        dy += step;
        lane.load(nx, x);
        lane.load(nd, dy);
      } else if (item + stride < items) {
        pos = first(item + stride);
      }
      float m = 0.0f, ex = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d0 = fmaf(d[0][i], c[i], d[1][i] * s[i]), d1 = fmaf(d[1][i], c[i], -(d[0][i] * s[i]));
        d[0][i] = d0;
        d[1][i] = d1;
        m = fmaf(v[0][i], v[0][i], fmaf(v[1][i], v[1][i], m));
        ex = fmaf(d0 * g[0][i], v[0][i], fmaf(d1 * g[1][i], v[1][i], ex));
      }
      const float r = 1.0f / sqrtf(group_sum<L>(m) * inv + a.eps), k = group_sum<L>(ex) * inv * r * r;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dg[j][i] = fmaf(d[j][i], v[j][i] * r, dg[j][i]);
          v[j][i] = r * (d[j][i] * g[j][i] - v[j][i] * k);
        }
      lane.store(out, v);
    }
  }
  float* const part = a.groups[which] > 1 ? a.part + (long)blockIdx.x * a.D : side.dgamma;
  if (!part) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    add[i][threadIdx.x] = dg[0][i];
    add[V + i][threadIdx.x] = dg[1][i];
  }
  __syncthreads();
  // one column a thread, its slots in order
  for (int j = threadIdx.x; j < 2 * V * L; j += kThreads) {
    const int l = j / (2 * V), i = j % (2 * V);
    const int col = Lane<DT, WHOLE>(a, l).column(i / V, i % V);
    if (col < 0) continue;
    float t = 0.0f;
#pragma unroll 8
    for (int k = 0; k < kSlots; ++k) t += add[i][k * L + l];
    part[col] = t;
  }
}

// Adds a side's rows of partial sums: 16 columns a work-group, 64 rows at a time, each
// in its own order, then these.
constexpr int kSumRows = 64;
__global__ void __launch_bounds__(16 * kSumRows) k_qk_norm_sum(const QkArgs a) {
  __shared__ float sh[kSumRows][17];
  const int which = blockIdx.y, n = a.groups[which];
  float* const out = a.side[which].dgamma;
  if (n < 2 || !out) return;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, j = blockIdx.x * 16 + c;
  float s = 0.0f;
  if (j < a.D) {
    const float* p = a.part + (long)(which ? a.groups[0] : 0) * a.D + j;
    for (int i0 = r; i0 < n; i0 += 16 * kSumRows) {
      float v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = p[(long)min(i0 + k * kSumRows, n - 1) * a.D];
#pragma unroll
      for (int k = 0; k < 16; ++k) s += i0 + k * kSumRows < n ? v[k] : 0.0f;
    }
  }
  sh[r][c] = s;
  __syncthreads();
  if (r > 0 || j >= a.D) return;
#pragma unroll 16
  for (int i = 1; i < kSumRows; ++i) s += sh[i][c];
  out[j] = s;
}

// Lanes of a head.
int lanes(const QkArgs& a, int V) {
  const int need = a.neighbours ? (a.D + 2 * V - 1) / (2 * V) : (a.R / 2 + V - 1) / V + ((a.D - a.R + 1) / 2 + V - 1) / V;
  int l = 1;
  while (l < need) l *= 2;
  return l;
}
bool whole(const QkArgs& a, int V) {
  return a.neighbours ? a.D % (2 * V) == 0 : a.R % (2 * V) == 0 && (a.D - a.R) % (2 * V) == 0;
}
// Items of a step: lane groups beside each other read longer runs of a row, but each
// computes the angles again, of twice as many pairs a lane in bf16; more where that
// gives fewer than kItems (8192, 16384 and 32768 of them: 1000 rows, 16 heads of 64 fp32
// 5.2, 4.5 and 4.5 us, 4500 rows 10.2, 10.2 and 11.5, bf16 17.2, 10.5 and 10.1, gradient
// 14.3, 13.8 and 19.3).  Measured, 1 and 4: 65536 rows, 16 heads of 64 fp32, 115 and
// 100 us, gradient 160 and 154; 204800 rows, 20 heads of 64 bf16, 206 and 239, gradient
// 379 and 463.
constexpr long kItems = 16384;
int parts_of(int dtype, long rows, int heads) {
  return (int)std::min<long>(heads, std::max<long>(dtype == WM_FP32 ? 4 : 1, kItems / std::max<long>(rows, 1)));
}
// Work-groups of the gradient for one side: as many as it has items for (one for a side
// without heads: it writes zeros), up to its share of 1024 by heads, or of kMost where a
// lane group has four items or more.  Measured, 1024 and 2048: 204800 rows, 20 heads of
// 64 bf16 337 and 313 us, fp32 615 and 605, 4500 rows, 9 heads of 61 fp32 19.0 and 20.9.
constexpr long kMost = 2048;
int grad_groups(long rows, int heads, int all, int L, int parts) {
  const long items = rows * std::min(parts, std::max(heads, 1)), slots = kThreads / L, full = (items + slots - 1) / slots;
  return (int)std::max<long>({1, std::min(full, kMost / 2 * heads / all), std::min(full / 4, kMost * heads / all)});
}

template <int N> using Const = std::integral_constant<int, N>;
template <typename DT, typename F>
hipError_t by_lanes(const QkArgs& a, F f) {
  const bool w = whole(a, Io<DT>::VEC);
  auto go = [&](auto l) { return w ? f(l, std::true_type()) : f(l, std::false_type()); };
  switch (lanes(a, Io<DT>::VEC)) {
    case 1: return go(Const<1>());
    case 2: return go(Const<2>());
    case 4: return go(Const<4>());
    case 8: return go(Const<8>());
    case 16: return go(Const<16>());
    case 32: return go(Const<32>());
    default: return go(Const<64>());
  }
}

}  // namespace

hipError_t launch_qk_norm(int dtype, const QkArgs& args, hipStream_t s) {
  QkArgs a = args;
  const int heads = a.side[0].heads + a.side[1].heads;
  a.parts = parts_of(dtype, a.rows, heads);
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    return by_lanes<DT>(a, [&](auto l, auto w) {
      const long items = a.rows * a.parts, slots = kThreads / l;
      return launch("qk_norm", k_qk_norm<DT, l, w>, dim3((unsigned)std::min<long>((items + slots - 1) / slots, kGroups)), dim3(kThreads), 0, s, a);
    });
  };
  return dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
}

size_t qk_norm_grad_workspace(long rows, int Hq, int Hk, int D) {
  (void)rows, (void)Hq, (void)Hk;
  return (size_t)(kMost + 2) * D * sizeof(float);
}

hipError_t launch_qk_norm_grad(int dtype, const QkArgs& args, hipStream_t s) {
  QkArgs a = args;
  const int heads = a.side[0].heads + a.side[1].heads;
  a.parts = parts_of(dtype, a.rows, heads);
  const int l = lanes(a, dtype == WM_FP32 ? 4 : 8);
  for (int w = 0; w < 2; ++w) a.groups[w] = grad_groups(a.rows, a.side[w].heads, heads, l, a.parts);
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    return by_lanes<DT>(a, [&](auto l, auto w) {
      return launch("qk_norm_grad", k_qk_norm_grad<DT, l, w>, dim3(a.groups[0] + a.groups[1]), dim3(kThreads), 0, s, a);
    });
  };
  const hipError_t e = dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
  if (e != hipSuccess || (a.groups[0] < 2 && a.groups[1] < 2)) return e;
  return launch("qk_norm_sum", k_qk_norm_sum, dim3((unsigned)((a.D + 15) / 16), 2), dim3(16 * kSumRows), 0, s, a);
}

}  // namespace wm
