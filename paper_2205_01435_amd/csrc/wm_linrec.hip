// Gated linear recurrence over [T, B, H], each channel for itself:
//   a_t = sigmoid(gate_t),  h_t = a_t h_{t-1} + (1 - a_t) x_t,  y_t = h_t,
// where a reset step takes h_{t-1} = 0 and a step past the row's length keeps
// h and puts out 0.  Gradient, with R_t what the later steps add to dh_t:
//   D = dy_t + R_t, dx_t = (1 - a_t) D, dgate_t = a_t (1 - a_t) (h_{t-1} - x_t) D,
//   R_{t-1} = a_t D, or 0 at a reset.
//
// A run of steps is an affine map of the state that enters it, h -> U + A h,
// and maps compose: that is what splits the time axis.
//   - A wave owns a tile of TT steps of 64 lanes (a lane: one fp32 channel or
//     two bf16 ones), loads it whole, and folds it into the tile's map.
//   - The waves of a work-group own the tiles of one segment of up to kWaves
//     TT steps; their maps meet in LDS.
//   - Longer sequences take several segments, each a work-group of the same
//     launch.  A work-group publishes its segment's map, then composes the
//     maps of the segments before it, and only then runs its steps from the
//     state that enters each tile.  Inputs are read once and outputs written
//     once, whatever T is.
// A segment waits only for maps, and a map is published before its segment
// waits for anything; segments take their numbers from a counter in the order
// in which they start, so every map that is waited for belongs to a work-group
// that already runs: no wait depends on what else occupies the device.  (The
// waits are bounded all the same; one that reached its bound would set the
// workspace's error word.)
// The gradient recomputes h_{t-1} from the inputs and the fp32 state that
// entered the segment (saved by the forward call: 1 / (kWaves TT) of the
// input), in fp32 and without reading y.
//
// A map whose run holds a reset does not depend on the state at all: A = -1
// says so (a true A is never negative), because 0 * inf would not.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_kernels.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kWaves = 8;      // tiles of a segment at most
constexpr int kTT = 16;        // steps of a tile
constexpr int kSeg = kWaves * kTT;
constexpr int kFan = 16;       // segments whose maps are composed into one for the segments after them
constexpr int kMaxSegs = 1024; // segments of a launch; longer sequences take several
constexpr unsigned kSpinLimit = 1u << 22;
constexpr unsigned long long kEmpty = ~0ull;  // a map not yet published (A's bits would be a NaN of this sign)

// V channels of one lane at one step, as loaded.  Rows are aligned to their
// element only; the hardware takes such addresses for wide loads too.
template <typename DT, int V> struct Chan;
template <> struct Chan<float, 1> {
  typedef float raw;
  __device__ static raw load(const char* p) { return *reinterpret_cast<const float*>(p); }
  __device__ static float get(raw r, int) { return r; }
  __device__ static void put(char* p, const float* v) { *reinterpret_cast<float*>(p) = v[0]; }
  __device__ static uint32_t size(raw r) { return __float_as_uint(r) & 0x7fffffffu; }
};
template <> struct Chan<bf16_t, 1> {
  typedef bf16_t raw;
  __device__ static raw load(const char* p) { return *reinterpret_cast<const bf16_t*>(p); }
  __device__ static float get(raw r, int) { return bf16_bits_to_f32(r); }
  __device__ static void put(char* p, const float* v) { *reinterpret_cast<bf16_t*>(p) = (bf16_t)f32_to_bf16_bits(v[0]); }
  __device__ static uint32_t size(raw r) { return (uint32_t)r << 16 & 0x7fffffffu; }
};
template <> struct Chan<bf16_t, 2> {
  typedef uint32_t raw;
  typedef uint32_t __attribute__((aligned(2))) mem;
  __device__ static raw load(const char* p) { return *reinterpret_cast<const mem*>(p); }
  __device__ static float get(raw r, int j) { return __uint_as_float(j ? r & 0xffff0000u : r << 16); }
  __device__ static void put(char* p, const float* v) { *reinterpret_cast<mem*>(p) = pack2_bf16(v[0], v[1]); }
  __device__ static uint32_t size(raw r) { return max(r & 0x7fffffffu, r << 16 & 0x7fffffffu); }
};

struct Map {
  float A, U;
};
// first m, then n
__device__ __forceinline__ Map then(Map m, Map n) {
  if (n.A < 0.0f) return n;
  return {m.A < 0.0f ? -1.0f : n.A * m.A, fmaf(n.A, m.U, n.U)};
}
__device__ __forceinline__ float apply(Map m, float h) { return m.A < 0.0f ? m.U : fmaf(m.A, h, m.U); }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// What a wave knows of its tile: the lane's channels and the masks of its steps.
template <int TT, int V>
struct Tile {
  long c;        // first channel of the lane (row b, column h)
  int b, h, b0;  // b0: the wave's first row
  int t0, nt;
  bool on;       // the channels exist
  int live;      // steps of the tile inside the row's length
  uint32_t rs;   // bit i: step i starts anew

  __device__ Tile(long group, int t0_, int T, int B, int H, const uint8_t* resets, const int32_t* lengths) : t0(t0_) {
    const int lane = threadIdx.x & 63;
    const long C = (long)B * H;
    c = (group * 64 + lane) * V;
    on = c < C;
    const uint32_t cc = (uint32_t)(on ? c : C - V);  // B H is below 2^31
    b = (int)(cc / (uint32_t)H);
    h = (int)(cc - (uint32_t)b * (uint32_t)H);
    b0 = uniform(b);
    nt = min(max(T - t0, 0), TT);
    live = on ? nt : 0;
    if (lengths) live = min(live, max(lengths[b] - t0, 0));
    rs = 0;
    if (resets) {
      // 64 / TT rows by TT steps at a time: one byte per lane, handed round as a ballot
      constexpr int kRows = 64 / TT;
      const int b1 = __builtin_amdgcn_readlane(b, 63), ti = lane % TT;
      for (int r = b0; r <= b1; r += kRows) {
        const int br = r + lane / TT;
        const bool hit = ti < nt && br <= b1 && resets[(long)(t0 + ti) * B + br] != 0;
        const unsigned long long m = __ballot(hit);
        const int k = b - r;
        if (k >= 0 && k < kRows) rs = (uint32_t)(m >> (TT * k)) & ((1u << TT) - 1u);
      }
      rs &= (1u << live) - 1u;
    }
  }
  __device__ bool reset(int i) const { return (rs >> i) & 1u; }
  // whether every step of every lane counts and none starts anew
  __device__ bool whole() const { return __all(live == TT && rs == 0); }
};

// A [T, B, H] array at a wave's tile: the step's row of the wave's first lane
// in scalar registers, the lane's place from there as a 32-bit offset (the
// launch checks that the rows that a wave can reach lie within 2 GiB).
template <typename DT, int TT, int V>
struct At {
  char* p;
  long step;     // bytes
  uint32_t off;
  __device__ At(const void* base, long st, long sb, const Tile<TT, V>& k) {
    p = reinterpret_cast<char*>(const_cast<void*>(base)) + ((long)k.t0 * st + (long)k.b0 * sb) * (long)sizeof(DT);
    step = st * (long)sizeof(DT);
    off = (uint32_t)(((long)(k.b - k.b0) * sb + k.h) * (long)sizeof(DT));
  }
  __device__ char* at(int i) const { return p + i * step + off; }
};

template <typename DT, int V, int TT>
__device__ __forceinline__ void load_tile(typename Chan<DT, V>::raw (&r)[TT], const SeqView& v, const Tile<TT, V>& k) {
  At<DT, TT, V> q(v.p, v.t, v.b, k);
  if (k.nt == TT) {
#pragma unroll
    for (int i = 0; i < TT; ++i, q.p += q.step) r[i] = Chan<DT, V>::load(q.p + q.off);
  } else {
#pragma unroll
    for (int i = 0; i < TT; ++i, q.p += q.step) r[i] = i < k.nt ? Chan<DT, V>::load(q.p + q.off) : typename Chan<DT, V>::raw(0);
  }
}

// The segment maps of a launch, in the workspace: the counter and the status
// words, then [segments][channels] maps, then those of kFan segments each, then
// a copy of the state that enters the launch and the state between launches.
struct Chain {
  unsigned* head;  // [0] next segment; [kSyncErr] the error word
  unsigned long long *seg, *fan;
  const float* enter; // [channels] state that enters the launch, or null (0)
  float* leave;       // [channels] state that leaves it, or null
  int seg0, segs;     // first segment and segments of this launch
  int t0, t1;         // its steps
  long groups;        // channel groups of 64 V
};

__device__ __forceinline__ void publish(unsigned long long* p, Map m) {
  // a NaN of A's is written as the positive one: never the empty pattern
  const uint32_t a = __isnanf(m.A) ? 0x7fc00000u : __float_as_uint(m.A);
  __hip_atomic_store(p, ((unsigned long long)__float_as_uint(m.U) << 32) | a, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long peek(const unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Map await(const unsigned long long* p, unsigned long long v, unsigned* head) {
  for (unsigned n = 0; v == kEmpty; ++n) {
    if (n == kSpinLimit) {
      __hip_atomic_store(head + kSyncErr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      break;
    }
    __builtin_amdgcn_s_sleep(1);
    v = peek(p);
  }
  return {__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Composes n maps, `stride` words apart, in order; four loads in flight.
template <int V>
__device__ __forceinline__ void compose(Map (&m)[V], const unsigned long long* p, int n, long stride, unsigned* head) {
  for (int i = 0; i < n; i += 4) {
    unsigned long long w[4][V];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n)
#pragma unroll
        for (int v = 0; v < V; ++v) w[k][v] = peek(p + (i + k) * stride + v);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n)
#pragma unroll
        for (int v = 0; v < V; ++v) m[v] = then(m[v], await(p + (i + k) * stride + v, w[k][v], head));
  }
}

// What the work-group's waves share: the tiles' maps, and the parts of the
// composition over earlier segments.
template <int V> struct Shared {
  Map tile[kWaves][64][V];
  Map part[kWaves][64][V];
  float enter[64][V];
  unsigned order;
};

// The map of everything before the segment that is `order`th in the chain
// (identity for the first), composed by all waves of the work-group; publishes
// the segment's own map first.  Every wave of the work-group calls it, after
// the barrier that completes sh.tile.
template <int V>
__device__ __forceinline__ void before(Map (&m)[V], Shared<V>& sh, const Chain& ch, int order, long group, int waves,
                                       bool forward) {
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const long stride = ch.groups * 64 * V, at = (group * 64 + lane) * V;
  if (w == waves - 1) {  // the segment's map
    Map s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = {1.0f, 0.0f};
    for (int i = 0; i < waves; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = then(s[v], sh.tile[forward ? i : waves - 1 - i][lane][v]);
#pragma unroll
    for (int v = 0; v < V; ++v) publish(ch.seg + order * stride + at + v, s[v]);
    if (order % kFan == kFan - 1) {  // ... and that of its fan
      Map f[V];
#pragma unroll
      for (int v = 0; v < V; ++v) f[v] = {1.0f, 0.0f};
      compose<V>(f, ch.seg + (order - (kFan - 1)) * stride + at, kFan - 1, stride, ch.head);
#pragma unroll
      for (int v = 0; v < V; ++v) publish(ch.fan + order / kFan * stride + at + v, then(f[v], s[v]));
    }
  }
  // whole fans before it, then the segments of its own fan: dealt to the waves in runs
  const int fans = order / kFan, n = fans + order % kFan;
  const int i0 = n * w / waves, i1 = n * (w + 1) / waves;
  Map p[V];
#pragma unroll
  for (int v = 0; v < V; ++v) p[v] = {1.0f, 0.0f};
  if (i0 < fans) compose<V>(p, ch.fan + i0 * stride + at, min(i1, fans) - i0, stride, ch.head);
  if (i1 > fans) {
    const int j = max(i0, fans);
    compose<V>(p, ch.seg + ((long)fans * kFan + j - fans) * stride + at, i1 - j, stride, ch.head);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) sh.part[w][lane][v] = p[v];
  __syncthreads();
#pragma unroll
  for (int v = 0; v < V; ++v) m[v] = {1.0f, 0.0f};
  for (int i = 0; i < waves; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = then(m[v], sh.part[i][lane][v]);
}

// The work-group's place: which channels, which segment.
__device__ __forceinline__ void place(unsigned* order, const Chain& ch, long& group, int& seg) {
  if (ch.segs > 1) {
    if (threadIdx.x == 0) *order = atomicAdd(ch.head, 1u);
    __syncthreads();
    const uint32_t k = (uint32_t)uniform((int)*order), n = (uint32_t)ch.groups;
    seg = (int)(k / n);
    group = k - (uint32_t)seg * n;
  } else {
    seg = 0;
    group = blockIdx.x;
  }
}

// The tile's steps of a wave, in registers: a, u = (1 - a) x (forward) and
// their map.  MASKED: some step is padding or starts anew, or some gate is
// beyond kGateMost.
template <bool MASKED, typename DT, int V, int TT>
__device__ __forceinline__ void fold(float (&A)[TT][V], float (&U)[TT][V], Map (&m)[V],
                                     const typename Chan<DT, V>::raw (&xr)[TT], const typename Chan<DT, V>::raw (&gr)[TT],
                                     const Tile<TT, V>& k) {
#pragma unroll
  for (int i = 0; i < TT; ++i) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float g = Chan<DT, V>::get(gr[i], v), x = Chan<DT, V>::get(xr[i], v);
      if constexpr (MASKED) {
        const float2 p = gate_pair(g);
        const bool live = i < k.live;
        A[i][v] = live ? (k.reset(i) ? -1.0f : p.x) : 1.0f;
        U[i][v] = live ? p.y * x : 0.0f;
        m[v] = then(m[v], {A[i][v], U[i][v]});
      } else {
        const float2 p = gate_pair_small(g);
        A[i][v] = p.x;
        U[i][v] = p.y * x;
        m[v].A *= p.x;
        m[v].U = fmaf(p.x, m[v].U, U[i][v]);
      }
    }
  }
}

template <typename DT, int V, int TT>
__device__ __forceinline__ bool small_gates(const typename Chan<DT, V>::raw (&gr)[TT]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < TT; ++i) most = max(most, Chan<DT, V>::size(gr[i]));
  return __all(most <= __float_as_uint(kGateMost));  // NaN and infinity lie above
}

// waves: tiles of a segment; with one wave per segment the work-group holds
// blockDim / 64 channel groups instead.
template <typename DT, int V, int TT>
__global__ void __launch_bounds__(64 * kWaves) k_linrec(const LinrecArgs a, const Chain ch, int waves) {
  __shared__ Shared<V> sh;
  typedef Chan<DT, V> Ch;
  const int lane = threadIdx.x & 63;
  int w = uniform(threadIdx.x >> 6), seg;
  long group;
  place(&sh.order, ch, group, seg);
  if (waves == 1) group = group * (blockDim.x >> 6) + w, w = 0;
  const Tile<TT, V> k(group, (ch.seg0 + seg) * waves * TT + w * TT, a.T, a.B, a.H, a.resets, a.lengths);
  typename Ch::raw xr[TT], gr[TT];
  load_tile<DT, V, TT>(gr, a.gate, k);
  load_tile<DT, V, TT>(xr, a.x, k);
  float h[V];
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = w == 0 && ch.enter && k.on ? ch.enter[k.c + v] : 0.0f;
  float A[TT][V], U[TT][V];
  Map m[V];
#pragma unroll
  for (int v = 0; v < V; ++v) m[v] = {1.0f, 0.0f};
  const bool whole = k.whole() && small_gates<DT, V, TT>(gr);
  if (whole)
    fold<false, DT, V, TT>(A, U, m, xr, gr, k);
  else
    fold<true, DT, V, TT>(A, U, m, xr, gr, k);
  if (waves > 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      sh.tile[w][lane][v] = m[v];
      if (w == 0) sh.enter[lane][v] = h[v];  // read once, before anything of this row may be written
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = sh.enter[lane][v];
    if (ch.segs > 1) {
      Map e[V];
      before<V>(e, sh, ch, seg, group, waves, true);
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = apply(e[v], h[v]);
    }
    if (a.states && w == 0 && k.on)
#pragma unroll
      for (int v = 0; v < V; ++v) a.states[(long)(ch.seg0 + seg) * a.B * a.H + k.c + v] = h[v];
    for (int i = 0; i < w; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = apply(sh.tile[i][lane][v], h[v]);
  } else if (a.states && k.on) {
#pragma unroll
    for (int v = 0; v < V; ++v) a.states[k.c + v] = h[v];
  }
  At<DT, TT, V> y(a.y, (long)a.B * a.H, a.H, k);
  if (whole) {
#pragma unroll
    for (int i = 0; i < TT; ++i, y.p += y.step) {
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = fmaf(A[i][v], h[v], U[i][v]);
      Ch::put(y.p + y.off, h);
    }
  } else {
#pragma unroll
    for (int i = 0; i < TT; ++i, y.p += y.step) {
      float o[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[v] = apply({A[i][v], U[i][v]}, h[v]);
        o[v] = i < k.live ? h[v] : 0.0f;
      }
      if (i < k.nt && k.on) Ch::put(y.p + y.off, o);
    }
  }
  if (ch.leave && k.on && k.t0 + TT >= ch.t1 && k.t0 < max(ch.t1, 1))
#pragma unroll
    for (int v = 0; v < V; ++v) ch.leave[k.c + v] = h[v];
}

// The gradient's tile: a and 1 - a of its steps, the map of h and that of R,
//   R_out = sum_i (prod_{j <= i} a_j) dy_i + (prod a) R_in.
template <bool MASKED, typename DT, int V, int TT>
__device__ __forceinline__ void fold_grad(float (&A)[TT][V], float (&M)[TT][V], Map (&m)[V], Map (&r)[V],
                                          const typename Chan<DT, V>::raw (&xr)[TT],
                                          const typename Chan<DT, V>::raw (&gr)[TT],
                                          const typename Chan<DT, V>::raw (&dr)[TT], const Tile<TT, V>& k) {
#pragma unroll
  for (int i = 0; i < TT; ++i) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float g = Chan<DT, V>::get(gr[i], v), x = Chan<DT, V>::get(xr[i], v), d = Chan<DT, V>::get(dr[i], v);
      const float2 p = MASKED ? gate_pair(g) : gate_pair_small(g);
      A[i][v] = p.x;
      M[i][v] = p.y;
      if constexpr (MASKED) {
        if (i < k.live) {
          const bool cut = k.reset(i);
          m[v] = then(m[v], {cut ? -1.0f : p.x, p.y * x});
          if (cut) r[v].A = -1.0f;
          if (!(r[v].A < 0.0f)) {
            r[v].A *= p.x;
            r[v].U = fmaf(r[v].A, d, r[v].U);
          }
        }
      } else {
        m[v].A *= p.x;
        m[v].U = fmaf(p.x, m[v].U, p.y * x);
        r[v].U = fmaf(m[v].A, d, r[v].U);
      }
    }
  }
  if constexpr (!MASKED)
#pragma unroll
    for (int v = 0; v < V; ++v) r[v].A = m[v].A;
}

template <bool MASKED, typename DT, int V, int TT>
__device__ __forceinline__ void emit_grad(float (&A)[TT][V], float (&M)[TT][V], float (&h)[V], float (&R)[V],
                                          const typename Chan<DT, V>::raw (&xr)[TT],
                                          const typename Chan<DT, V>::raw (&dr)[TT], const Tile<TT, V>& k,
                                          const LinrecGradArgs& a) {
  typedef Chan<DT, V> Ch;
  // forward: what h_{t-1} puts into dgate
  float G[TT][V];
#pragma unroll
  for (int i = 0; i < TT; ++i) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float x = Ch::get(xr[i], v);
      if (MASKED && k.reset(i)) h[v] = 0.0f;
      G[i][v] = A[i][v] * M[i][v] * (h[v] - x);
      if (!MASKED || i < k.live) h[v] = fmaf(A[i][v], h[v], M[i][v] * x);
    }
  }
  At<DT, TT, V> dx(a.dx.p, a.dx.t, a.dx.b, k), dg(a.dgate.p, a.dgate.t, a.dgate.b, k);
  dx.p += (TT - 1) * dx.step;
  dg.p += (TT - 1) * dg.step;
#pragma unroll
  for (int i = TT - 1; i >= 0; --i, dx.p -= dx.step, dg.p -= dg.step) {
    float ox[V], og[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const bool live = !MASKED || i < k.live;
      const float D = R[v] + Ch::get(dr[i], v);
      ox[v] = live ? M[i][v] * D : 0.0f;
      og[v] = live ? G[i][v] * D : 0.0f;
      R[v] = live ? (MASKED && k.reset(i) ? 0.0f : A[i][v] * D) : R[v];
    }
    if (!MASKED || (i < k.nt && k.on)) {
      Ch::put(dx.p + dx.off, ox);
      Ch::put(dg.p + dg.off, og);
    }
  }
}

template <typename DT, int V, int TT>
__global__ void __launch_bounds__(64 * kWaves) k_linrec_grad(const LinrecGradArgs a, const Chain ch, int waves) {
  __shared__ Shared<V> sh;
  __shared__ Map fwd[kWaves][64][V];
  typedef Chan<DT, V> Ch;
  const int lane = threadIdx.x & 63;
  int w = uniform(threadIdx.x >> 6), order;
  long group;
  place(&sh.order, ch, group, order);
  const int seg = ch.seg0 + ch.segs - 1 - order;  // the chain runs from the last segment to the first
  if (waves == 1) group = group * (blockDim.x >> 6) + w, w = 0;
  const Tile<TT, V> k(group, seg * waves * TT + w * TT, a.T, a.B, a.H, a.resets, a.lengths);
  typename Ch::raw xr[TT], gr[TT], dr[TT];
  load_tile<DT, V, TT>(gr, a.gate, k);
  load_tile<DT, V, TT>(xr, a.x, k);
  load_tile<DT, V, TT>(dr, a.dy, k);
  float h[V], R[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    h[v] = k.on ? a.states[(long)seg * a.B * a.H + k.c + v] : 0.0f;
    R[v] = w == waves - 1 && ch.enter && k.on ? ch.enter[k.c + v] : 0.0f;
  }
  float A[TT][V], M[TT][V];  // a, 1 - a
  Map m[V], r[V];
#pragma unroll
  for (int v = 0; v < V; ++v) m[v] = r[v] = {1.0f, 0.0f};
  const bool whole = k.whole() && small_gates<DT, V, TT>(gr);
  if (whole)
    fold_grad<false, DT, V, TT>(A, M, m, r, xr, gr, dr, k);
  else
    fold_grad<true, DT, V, TT>(A, M, m, r, xr, gr, dr, k);
  if (waves > 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      fwd[w][lane][v] = m[v];
      sh.tile[w][lane][v] = r[v];
      if (w == waves - 1) sh.enter[lane][v] = R[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) R[v] = sh.enter[lane][v];
    if (ch.segs > 1) {
      Map e[V];
      before<V>(e, sh, ch, order, group, waves, false);
#pragma unroll
      for (int v = 0; v < V; ++v) R[v] = apply(e[v], R[v]);
    }
    for (int i = 0; i < w; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = apply(fwd[i][lane][v], h[v]);
    for (int i = waves - 1; i > w; --i)
#pragma unroll
      for (int v = 0; v < V; ++v) R[v] = apply(sh.tile[i][lane][v], R[v]);
  }
  if (whole)
    emit_grad<false, DT, V, TT>(A, M, h, R, xr, dr, k, a);
  else
    emit_grad<true, DT, V, TT>(A, M, h, R, xr, dr, k, a);
  if (ch.leave && k.on && k.t0 == ch.t0)
#pragma unroll
    for (int v = 0; v < V; ++v) ch.leave[k.c + v] = R[v];
}

// Empties the maps of a launch, and copies the state that enters it (which the
// last segment's result may overwrite); the first one clears the status words.
__global__ void __launch_bounds__(256) k_linrec_init(const Chain ch, long words, const float* from, long C, bool first) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, step = (long)gridDim.x * 256;
  if (i == 0) ch.head[0] = 0;
  if (first && i < 2) ch.head[kSyncErr + i] = 0;
  for (long j = i; j < words; j += step) ch.seg[j] = kEmpty;
  if (from)
    for (long j = i; j < C; j += step) const_cast<float*>(ch.enter)[j] = from[j];
}

// How a call of T steps is split: steps of a tile, tiles of a segment, segments.
struct Plan {
  int tt, waves;
  long segs;
};
Plan plan(int T) {
  if (T <= 1) return {1, 1, 1};
  const int tiles = (int)(((long)T + kTT - 1) / kTT);
  if (tiles <= kWaves) return {kTT, tiles, 1};
  return {kTT, kWaves, (tiles + kWaves - 1) / kWaves};
}

// The workspace of a call with several segments.
constexpr size_t kHeadBytes = kSyncWords * sizeof(unsigned);
long pad_channels(int B, int H) { return ((long)B * H + 127) / 128 * 128; }  // whole groups, of one or two channels a lane
long map_words(long segs, long channels) { return (segs + segs / kFan) * channels; }

// Runs go(Chain, first launch, last launch) for every launch of a call, in
// order; `from` is the state that enters the call, `to` the one that leaves it.
template <typename F>
hipError_t run_chain(int T, int B, int H, int V, const Plan& p, void* ws, const float* from, float* to, bool reverse,
                     hipStream_t s, F go) {
  const long C = (long)B * H, groups = (C + 64 * V - 1) / (64 * V);
  Chain ch{};
  ch.groups = groups;
  if (p.segs == 1) {
    ch.enter = from;
    ch.leave = to;
    ch.segs = 1;
    ch.t1 = T;
    return go(ch);
  }
  const long most = std::min<long>(p.segs, kMaxSegs), pad = pad_channels(B, H);
  char* base = reinterpret_cast<char*>(ws);
  ch.head = reinterpret_cast<unsigned*>(base);
  ch.seg = reinterpret_cast<unsigned long long*>(base + kHeadBytes);
  float* enter = reinterpret_cast<float*>(ch.seg + map_words(most, pad));
  float* carry = enter + pad;
  const long launches = (p.segs + kMaxSegs - 1) / kMaxSegs;
  for (long n = 0; n < launches; ++n) {
    const long s0 = (reverse ? launches - 1 - n : n) * kMaxSegs;
    ch.seg0 = (int)s0;
    ch.segs = (int)std::min<long>(kMaxSegs, p.segs - s0);
    ch.t0 = (int)(s0 * kSeg);
    ch.t1 = (int)std::min<long>(T, (s0 + ch.segs) * kSeg);
    ch.fan = ch.seg + ch.segs * groups * 64 * V;
    const float* f = n == 0 ? from : carry;
    ch.enter = f ? enter : nullptr;
    ch.leave = n == launches - 1 ? to : carry;
    const long words = map_words(ch.segs, groups * 64 * V);
    const unsigned grid = (unsigned)std::min<long>(1024, (std::max(words, C) + 255) / 256);
    hipError_t e = launch("linrec_init", k_linrec_init, dim3(grid), dim3(256), 0, s, ch, words, f, C, n == 0);
    if (e == hipSuccess) e = go(ch);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int V, typename K, typename A>
hipError_t run(const char* name, K tile, K step, const A& a, const float* from, float* to, bool reverse, hipStream_t s) {
  const Plan p = plan(a.T);
  return run_chain(a.T, a.B, a.H, V, p, a.ws, from, to, reverse, s, [&](const Chain& ch) {
    // a work-group of one tile per segment holds four channel groups
    const int per = p.waves == 1 ? 4 : 1;
    const long grid = (ch.groups + per - 1) / per * ch.segs;
    return launch(name, p.tt == 1 ? step : tile, dim3((unsigned)grid), dim3(64u * (p.waves == 1 ? per : p.waves)), 0, s, a,
                  ch, p.waves);
  });
}

}  // namespace

size_t linrec_states(int T, int B, int H) { return (size_t)plan(T).segs * B * H * sizeof(float); }

size_t linrec_workspace(int T, int B, int H) {
  const Plan p = plan(T);
  if (p.segs == 1) return 0;
  const long pad = pad_channels(B, H);
  return kHeadBytes + (size_t)map_words(std::min<long>(p.segs, kMaxSegs), pad) * 8 + (size_t)pad * 2 * sizeof(float);
}

hipError_t launch_linrec(int dtype, const LinrecArgs& a, hipStream_t s) {
  if (dtype == WM_FP32) return run<1>("linrec", k_linrec<float, 1, kTT>, k_linrec<float, 1, 1>, a, a.h0, a.h_T, false, s);
  if (a.H % 2 == 0)
    return run<2>("linrec", k_linrec<bf16_t, 2, kTT>, k_linrec<bf16_t, 2, 1>, a, a.h0, a.h_T, false, s);
  return run<1>("linrec", k_linrec<bf16_t, 1, kTT>, k_linrec<bf16_t, 1, 1>, a, a.h0, a.h_T, false, s);
}

hipError_t launch_linrec_grad(int dtype, const LinrecGradArgs& a, hipStream_t s) {
  if (dtype == WM_FP32)
    return run<1>("linrec_grad", k_linrec_grad<float, 1, kTT>, k_linrec_grad<float, 1, 1>, a, a.dh_T, a.dh0, true, s);
  return run<1>("linrec_grad", k_linrec_grad<bf16_t, 1, kTT>, k_linrec_grad<bf16_t, 1, 1>, a, a.dh_T, a.dh0, true, s);
}

}  // namespace wm
