// Gated linear recurrence over [T, B, H], each channel for itself:
//   a_t = sigmoid(gate_t),  h_t = a_t h_{t-1} + (1 - a_t) x_t,  y_t = h_t,
// where a reset step takes h_{t-1} = 0 and a step past the row's length keeps
// h and puts out 0.  Gradient, with R_t what the later steps add to dh_t:
//   D = dy_t + R_t, dx_t = (1 - a_t) D, dgate_t = a_t (1 - a_t) (h_{t-1} - x_t) D,
//   R_{t-1} = a_t D, or 0 at a reset.
//
// With enough channels to fill the device a wave walks its 64 channels through
// all steps, the state in a register (k_linrec_walk).  With fewer, the time
// axis is split (k_linrec_split): a run of steps is an affine map of the state
// that enters it, h -> U + A h, and maps compose.
//   - A wave owns a tile of kTT steps of 64 channels, loads it whole, and folds
//     it into the tile's map.
//   - The waves of a work-group own the tiles of one segment; their maps meet in
//     LDS.
//   - Sequences of more than kWide tiles take several segments of kWaves, each a
//     work-group of the same launch.  A work-group publishes its segment's map,
//     then composes the maps of the segments before it, and only then runs its
//     steps from the state that enters each tile.
// Either way inputs are read once and outputs written once, whatever T is.
// A segment waits only for maps, and a map is published before its segment
// waits for anything; the segments of 64 channels take their numbers from these
// channels' counter in the order in which they start, so every map that is
// waited for belongs to a work-group that already runs: no wait depends on what
// else occupies the device.  (The waits are bounded all the same; one that
// reached its bound would set the workspace's error word.)  The device adds to
// one address about every 4 ns: one counter for all channels held the 4096
// work-groups of 32768 steps by 1024 channels back by 18 us.
//
// The gradient recomputes h_{t-1} from the inputs and the fp32 state that
// entered each tile of kTT steps, which the forward call saves (4 / kTT bytes
// a value): in fp32, and without reading y.
//
// The walk is bound by memory: 128 steps of 262144 fp32 channels with padding
// 53 us forward and 97 us back, 5.1 TB/s over both.  The split waits: 32768 steps
// of 1024 bf16 channels 150 us in all, 2.7 TB/s; the kernels 54 and 82 us, and
// 5 us each way for emptying the maps.  Of 4096 work-groups the registers admit
// 768 at a time forward and 512 back, so that the wait for earlier segments' maps
// begins anew five to six times forward and eight times back.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_chain.h"
#include "wm_kernels.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

// Tiles of a segment at most, where there are several, and of a single one: a
// wide work-group leaves a CU fewer waves (16 of 24), but waits for no other and
// needs no maps.  Measured, 200 steps, forward and gradient, two segments against
// one: fp32 64 channels 22 and 14 us, 32768 59 and 51, 65536 103 and 97; bf16
// 32768 47 and 35, 81920 90 and 82.
constexpr int kWaves = 8, kWide = 16;
constexpr int kTT = 16;        // steps of a tile
constexpr int kSeg = kWaves * kTT;
constexpr int kMaxSegs = 1024; // segments of a launch; longer sequences take several
// Channel groups (of 64) from which a wave walks all steps.  Measured, forward
// and gradient of 500 steps, split against walked: fp32 1280 groups 258 and 268
// us, 1536 319 and 297; bf16 1536 groups 212 and 232 us, 2048 270 and 258.
constexpr long kWalk32 = 1536, kWalk16 = 2048;
constexpr int kNextPitch = 32;  // words from one counter to the next: lines of their own
constexpr unsigned kSpinLimit = 1u << 22;
constexpr unsigned long long kEmpty = ~0ull;  // a map not yet published (A's bits would be a NaN of this sign)

// One value at one step, as loaded; from a row's address, the same in every
// lane, and the lane's offset in it.
#define WM_GLOBAL __attribute__((address_space(1)))
template <typename DT> struct Chan;
template <> struct Chan<float> {
  typedef float raw;
  __device__ static raw load(uint64_t row, uint32_t off) { return *reinterpret_cast<const WM_GLOBAL float*>(row + off); }
  __device__ static float get(raw r) { return r; }
  template <bool STREAM>
  __device__ static void put(uint64_t row, uint32_t off, float v) {
    if constexpr (STREAM)  // past the caches
      __builtin_nontemporal_store(v, reinterpret_cast<WM_GLOBAL float*>(row + off));
    else
      *reinterpret_cast<WM_GLOBAL float*>(row + off) = v;
  }
};
template <> struct Chan<bf16_t> {
  typedef uint32_t raw;  // a register of its own: halves would make one load wait for another
  __device__ static raw load(uint64_t row, uint32_t off) { return *reinterpret_cast<const WM_GLOBAL bf16_t*>(row + off); }
  __device__ static float get(raw r) { return bf16_bits_to_f32(r); }
  template <bool STREAM>
  __device__ static void put(uint64_t row, uint32_t off, float v) {
    const bf16_t b = (bf16_t)f32_to_bf16_bits(v);
    if constexpr (STREAM)
      __builtin_nontemporal_store(b, reinterpret_cast<WM_GLOBAL bf16_t*>(row + off));
    else
      *reinterpret_cast<WM_GLOBAL bf16_t*>(row + off) = b;
  }
};
#undef WM_GLOBAL

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// e^-|g| beyond kGateMost.  Where that of a finite g leaves fp32's range it is
// held at the least positive number: only an infinite g makes a gate, or its
// complement, 0, which an infinite state or input would turn to NaN.
__device__ __forceinline__ float gate_exp_far(float g) {
  const float e = expf(-fabsf(g));
  return e == 0.0f && fabsf(g) < INFINITY ? __FLT_DENORM_MIN__ : e;
}
// e^-|g|: the long way too where some lane of the wave needs it (NaN and
// infinity lie beyond the bound), for that lane alone: a channel's bits do not
// depend on its neighbours.
__device__ __forceinline__ float gate_exp_any(float g) {
  return fabsf(g) <= kGateMost ? gate_exp_small(g) : gate_exp_far(g);
}
__device__ __forceinline__ float gate_exp(float g) {
  if (__builtin_expect(__any(!(fabsf(g) <= kGateMost)), 0)) return gate_exp_any(g);
  return gate_exp_small(g);
}

// The gates of any g, in the same bits as gate_pair_small where that may be used.
__device__ __forceinline__ float2 gate_pair_any(float g) {
  return fabsf(g) <= kGateMost ? gate_pair_small(g) : gate_pair_of(g, gate_exp_far(g));
}

// What a wave knows of its 64 channels.
struct Lanes {
  long c;        // the lane's channel (row b, column h)
  int b, h;
  int b0, b1;    // the wave's first and last row
  bool on;       // the channel exists
  int n;         // the row's length
  int most;      // the most of the wave's rows

  __device__ Lanes(long group, int T, int B, int H, const int32_t* lengths) {
    const long C = (long)B * H;
    c = group * 64 + (threadIdx.x & 63);
    on = c < C;
    const uint32_t cc = (uint32_t)(on ? c : C - 1);  // B H is below 2^31
    b = (int)(cc / (uint32_t)H);
    h = (int)(cc - (uint32_t)b * (uint32_t)H);
    b0 = uniform(b);
    b1 = __builtin_amdgcn_readlane(b, 63);
    n = most = T;
    if (lengths) {
      n = min(max(lengths[b], 0), T);
      most = 0;
      for (int r = b0; r <= b1; ++r) most = max(most, __builtin_amdgcn_readlane(n, uniform(lane_of(r, group, H))));
    }
    if (!on) n = 0;
  }
  // a lane of the wave that holds row r
  __device__ int lane_of(int r, long group, int H) const {
    return max((int)((long)r * H - group * 64), 0);
  }
};

// A [T, B, H] array as a wave goes through it: the present step's row of the
// wave's first lane as an address in scalar registers, the lane's place from
// there as a 32-bit offset (the call checks that the rows that a wave can reach
// lie within 2 GiB).
template <typename DT, bool STREAM = false>
struct Rows {
  uint64_t base, row;
  long st, b;    // bytes
  uint32_t off;
  __device__ Rows(const SeqView& v, const Lanes& l, int t) {
    constexpr long es = sizeof(DT);
    base = reinterpret_cast<uint64_t>(v.p) + (uint64_t)((long)l.b0 * v.b * es);
    st = v.t * es;
    off = (uint32_t)(((long)(l.b - l.b0) * v.b + l.h) * es);
    to(t);
  }
  __device__ void to(int t) { row = base + (uint64_t)((long)t * st); }
  // The empty asm keeps the rows' addresses from being computed all at once
  // (they would not fit the scalar registers), and the offset 32 bits wide.
  __device__ void move(long bytes) {
    row += (uint64_t)bytes;
    asm volatile("" : "+s"(row));
    asm volatile("" : "+v"(off));
  }
  __device__ typename Chan<DT>::raw load() const { return Chan<DT>::load(row, off); }
  __device__ void put(float v) const { Chan<DT>::template put<STREAM>(row, off, v); }
};

// The resets of TT steps from t0 on: one byte a lane holds 64 / TT rows by TT
// steps, handed round as ballots.
template <int TT>
struct Resets {
  static constexpr int kRows = 64 / TT;
  uint32_t byte;  // of the wave's first rows, requested ahead of its use
  __device__ static uint32_t flag(const uint8_t* resets, const Lanes& l, int r, int t0, int T, int B) {
    const int lane = threadIdx.x & 63, t = t0 + lane % TT, br = r + lane / TT;
    return t < T && br <= l.b1 ? resets[(long)t * B + br] : 0;
  }
  __device__ void ask(const uint8_t* resets, const Lanes& l, int t0, int T, int B) {
    byte = resets ? flag(resets, l, l.b0, t0, T, B) : 0;
  }
  // bit i: step t0 + i of the lane's row starts anew
  __device__ uint32_t bits(const uint8_t* resets, const Lanes& l, int t0, int T, int B) const {
    uint32_t rs = 0, f = byte;
    if (!resets) return 0;
    for (int r = l.b0; r <= l.b1; r += kRows) {
      if (r > l.b0) f = flag(resets, l, r, t0, T, B);
      const unsigned long long m = __ballot(f != 0);
      const int k = l.b - r;
      if (k >= 0 && k < kRows) rs = (uint32_t)(m >> (TT * k)) & (uint32_t)((1ull << TT) - 1);
    }
    return rs;
  }
};

// ---------------------------------------------------------------------------
// All steps in one wave
// ---------------------------------------------------------------------------

// One tile; LOAD: the next tile's value of each step is requested as soon as
// the present one's is used.  MASKED: some step is padding or starts anew.
template <bool LOAD, bool MASKED, typename DT, int TT, bool STREAM>
__device__ __forceinline__ float walk_tile(float h, typename Chan<DT>::raw (&gr)[TT], typename Chan<DT>::raw (&xr)[TT],
                                           Rows<DT>& g, Rows<DT>& x, Rows<DT, STREAM>& y, int steps, int ahead, int live,
                                           uint32_t rs, bool on) {
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    if (MASKED && i >= steps) continue;
    const float gv = Chan<DT>::get(gr[i]), xv = Chan<DT>::get(xr[i]);
    if (LOAD) {  // (past the last step: that one's place again)
      gr[i] = g.load();
      xr[i] = x.load();
      g.move(i + 1 < ahead ? g.st : 0);
      x.move(i + 1 < ahead ? x.st : 0);
    }
    const float2 p = gate_pair_of(gv, gate_exp(gv));
    if (MASKED) {
      const float from = (rs >> i) & 1u ? 0.0f : h;
      const float to = fmaf(p.x, from, p.y * xv);
      h = i < live ? to : h;
      if (on) y.put(i < live ? h : 0.0f);
    } else {
      h = fmaf(p.x, h, p.y * xv);
      y.put(h);
    }
    y.move(y.st);
  }
  return h;
}

// The status words of a workspace that a call does not use otherwise.
__device__ __forceinline__ void clear_status(void* ws) {
  if (ws && blockIdx.x == 0 && threadIdx.x < 2) reinterpret_cast<unsigned*>(ws)[kSyncErr + threadIdx.x] = 0;
}

template <typename DT, int TT, bool STREAM>
__global__ void __launch_bounds__(256) k_linrec_walk(const LinrecArgs a) {
  const long C = (long)a.B * a.H, group = (long)blockIdx.x * (blockDim.x >> 6) + uniform(threadIdx.x >> 6);
  clear_status(a.ws);
  if (group * 64 >= C) return;
  const Lanes l(group, a.T, a.B, a.H, a.lengths);
  Resets<TT> rb;
  rb.ask(a.resets, l, 0, l.most, a.B);
  Rows<DT> g(a.gate, l, 0), x(a.x, l, 0);
  Rows<DT, STREAM> y(SeqView{a.y, C, a.H}, l, 0);
  typename Chan<DT>::raw gr[TT], xr[TT];
  if (l.most > 0)
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      gr[i] = g.load();
      xr[i] = x.load();
      g.move(i + 1 < l.most ? g.st : 0);
      x.move(i + 1 < l.most ? x.st : 0);
    }
  float h = a.h0 && l.on ? a.h0[l.c] : 0.0f;
  for (int t0 = 0; t0 < l.most; t0 += TT) {
    const uint32_t rs = rb.bits(a.resets, l, t0, l.most, a.B);
    const int steps = min(l.most - t0, TT), live = min(max(l.n - t0, 0), TT), ahead = l.most - t0 - TT;
    const bool masked = !__all(live == TT && rs == 0);
    if (ahead > 0) rb.ask(a.resets, l, t0 + TT, l.most, a.B);
    if (a.states && l.on) a.states[(long)(t0 / kTT) * C + l.c] = h;
    if (ahead > 0)
      h = masked ? walk_tile<true, true, DT, TT, STREAM>(h, gr, xr, g, x, y, steps, ahead, live, rs, l.on)
                 : walk_tile<true, false, DT, TT, STREAM>(h, gr, xr, g, x, y, steps, ahead, live, rs, l.on);
    else
      h = masked ? walk_tile<false, true, DT, TT, STREAM>(h, gr, xr, g, x, y, steps, ahead, live, rs, l.on)
                 : walk_tile<false, false, DT, TT, STREAM>(h, gr, xr, g, x, y, steps, ahead, live, rs, l.on);
  }
  // padding of every row of the wave
  y.to(l.most);
  for (int t = l.most; t < a.T; ++t, y.move(y.st))
    if (l.on) y.put(0.0f);
  if (a.h_T && l.on) a.h_T[l.c] = h;
}

// From the last tile to the first; in each forward from the saved state, then
// backward.  Of each step e^-|gate| with the gate's sign and h_{t-1} - x stay in
// registers; the gates come from them again on the way back, which costs less
// than to keep them (half the waves).  Masks are looked at step by step: with a second loop for tiles
// without them the compiler loads both ways' next values ahead of the branch, 48
// registers too many, and selections in every step keep as many conditions in
// scalar registers.
template <typename DT, int TT, bool STREAM>
__global__ void __launch_bounds__(256, 4) k_linrec_grad_walk(const LinrecGradArgs a) {
  const long C = (long)a.B * a.H, group = (long)blockIdx.x * (blockDim.x >> 6) + uniform(threadIdx.x >> 6);
  clear_status(a.ws);
  if (group * 64 >= C) return;
  const Lanes l(group, a.T, a.B, a.H, a.lengths);
  Rows<DT, STREAM> dx(a.dx, l, l.most), dg(a.dgate, l, l.most);
  for (int t = l.most; t < a.T; ++t, dx.move(dx.st), dg.move(dg.st))
    if (l.on) {
      dx.put(0.0f);
      dg.put(0.0f);
    }
  float R = a.dh_T && l.on ? a.dh_T[l.c] : 0.0f;
  if (l.most > 0) {
    int t0 = (l.most - 1) / TT * TT;
    Resets<TT> rb;
    rb.ask(a.resets, l, t0, l.most, a.B);
    Rows<DT> g(a.gate, l, t0), x(a.x, l, t0), d(a.dy, l, t0);
    typename Chan<DT>::raw gr[TT], xr[TT], dr[TT];
    // the last tile, which may be short: a step past the end reads the last one's place
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      gr[i] = g.load();
      xr[i] = x.load();
      dr[i] = d.load();
      const bool more = t0 + i + 1 < l.most;
      g.move(more ? g.st : 0);
      x.move(more ? x.st : 0);
      d.move(more ? d.st : 0);
    }
    float s = l.on ? a.states[(long)(t0 / kTT) * C + l.c] : 0.0f;
    for (; t0 >= 0; t0 -= TT) {
      uint32_t rs = rb.bits(a.resets, l, t0, l.most, a.B);
      int live = min(max(l.n - t0, 0), TT), lim = l.on ? min(l.most - t0, TT) : 0;
      const bool masked = !__all(live == TT && rs == 0);
      // the tile before it (the first one reads its first step again, for nothing), dy from its end
      const int tb = max(t0 - TT, 0);
      rb.ask(a.resets, l, tb, l.most, a.B);
      const bool more = t0 > 0;
      g.to(tb);
      x.to(tb);
      d.to(max(t0 - 1, 0));
      const float before = l.on ? a.states[(long)(tb / kTT) * C + l.c] : 0.0f;
      float E[TT], K[TT];
#pragma unroll
      for (int i = 0; i < TT; ++i) {
        const float gv = Chan<DT>::get(gr[i]), xv = Chan<DT>::get(xr[i]);
        gr[i] = g.load();
        g.move(more ? g.st : 0);
        E[i] = copysignf(gate_exp(gv), gv);
        const float2 p = gate_pair_of(gv, fabsf(E[i]));
        if (masked) s = (rs >> i) & 1u ? 0.0f : s;
        K[i] = s - xv;
        float to = fmaf(p.x, s, p.y * xv);
        if (masked) to = i < live ? to : s;
        s = to;
        // the step ends here: drawn out over the tile, its parts would not fit the registers
        asm volatile("" : "+v"(s), "+v"(E[i]), "+v"(K[i]));
      }
      dx.to(t0 + TT - 1);
      dg.to(t0 + TT - 1);
      // the steps' conditions anew: kept from above they would fill the scalar registers
      asm volatile("" : "+v"(rs), "+v"(live), "+v"(lim));
#pragma unroll
      for (int i = TT - 1; i >= 0; --i) {
        const float2 p = gate_pair_of(E[i], fabsf(E[i]));
        const float D = R + Chan<DT>::get(dr[i]);
        dr[i] = d.load();
        d.move(more ? -d.st : 0);
        xr[TT - 1 - i] = x.load();  // (into what the steps done leave free)
        x.move(more ? x.st : 0);
        const float ox = p.y * D, og = p.x * K[i] * ox;
        if (masked) {
          const bool in = i < live;
          if (i < lim) {
            dx.put(in ? ox : 0.0f);
            dg.put(in ? og : 0.0f);
          }
          R = in ? ((rs >> i) & 1u ? 0.0f : p.x * D) : R;
        } else {
          dx.put(ox);
          dg.put(og);
          R = p.x * D;
        }
        dx.move(-dx.st);
        dg.move(-dg.st);
      }
      s = before;
    }
  }
  if (a.dh0 && l.on) a.dh0[l.c] = R;
}

// ---------------------------------------------------------------------------
// The time axis split
// ---------------------------------------------------------------------------

// A wave's tile: the masks of its steps.
struct Tile : Lanes {
  int t0, nt, some; // the tile's steps; those inside some row's length
  int live;         // those inside the lane's row
  uint32_t rs;      // bit i: step i starts anew
  __device__ Tile(long group, int t0_, int T, int B, int H, const int32_t* lengths)
      : Lanes(group, T, B, H, lengths), t0(t0_), rs(0) {
    nt = min(max(T - t0, 0), kTT);
    some = min(max(most - t0, 0), kTT);
    live = min(max(n - t0, 0), kTT);
  }
  __device__ bool reset(int i) const { return (rs >> i) & 1u; }
  // whether every step of every lane counts and none starts anew
  __device__ bool whole() const { return __all(live == kTT && rs == 0); }
};

template <typename DT>
__device__ __forceinline__ void load_tile(typename Chan<DT>::raw (&r)[kTT], const SeqView& v, const Tile& k) {
  Rows<DT> q(v, k, k.t0);
  if (k.some == kTT) {
#pragma unroll
    for (int i = 0; i < kTT; ++i, q.move(q.st)) r[i] = q.load();
  } else {
#pragma unroll
    for (int i = 0; i < kTT; ++i, q.move(q.st)) r[i] = i < k.some ? q.load() : typename Chan<DT>::raw(0);
  }
}

// The segment maps of a launch, in the workspace: the status words, then the
// counters, then [segments][channels] maps, then those of kFan segments each,
// then a copy of the state that enters the launch and the state between launches.
struct Chain {
  unsigned* head;  // [kSyncErr] the error word
  unsigned* next;  // [groups][kNextPitch] the segment that starts next
  unsigned long long *seg, *fan;
  const float* enter; // [channels] state that enters the launch, or null (0)
  float* leave;       // [channels] state that leaves it, or null
  int seg0, segs;     // first segment and segments of this launch
  int t0, t1;         // its steps
  long groups;        // channel groups of 64
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

// compose() over the published maps of a lane's channel, four of a fan's members in flight.
__device__ __forceinline__ Map published(const unsigned long long* seg, const unsigned long long* fan, int s, int s1,
                                         long stride, unsigned* head) {
  return compose(
      s, s1,
      [&](int i, Map& f) {
        const unsigned long long v = peek(fan + i / kFan * stride);
        if (!__all(v != kEmpty)) return false;
        f = await(fan, v, head);
        return true;
      },
      [&](int i, int e, auto take) {
#pragma unroll 1
        for (; i < e; i += 4) {
          unsigned long long v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = i + k < e ? peek(seg + (i + k) * stride) : 0;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + k < e) take(await(seg + (i + k) * stride, v[k], head));
        }
      });
}

// What the work-group's waves share: the tiles' maps, the parts of the
// composition over earlier segments, the state that enters the launch.
template <int W>
struct Shared {
  Map tile[W][64];
  Map part[W == kWaves ? W : 1][64];  // (W = kWide: a single segment)
  float enter[64];
  unsigned order;
};

// The map of everything before the segment that is `order`th in the chain
// (identity for the first), composed by all waves of the work-group; publishes
// the segment's own map first.  All kWaves waves of the work-group call it,
// after the barrier that completes sh.tile.
__device__ __forceinline__ Map before(Shared<kWaves>& sh, const Chain& ch, int order, long group, bool forward) {
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const long stride = ch.groups * 64, at = group * 64 + lane;
  const Map none{1.0f, 0.0f};
  // whole fans before it, then the segments of its own fan: dealt to the waves in runs
  const int fans = order / kFan, n = fans + order % kFan;
  const int i0 = n * w / kWaves, i1 = n * (w + 1) / kWaves;
  auto first = [&](int i) { return i < fans ? i * kFan : fans * (kFan - 1) + i; };
  Map own = none, p;
  bool fan = false;
  if (w == kWaves - 1) {  // the segment's map
#pragma unroll
    for (int i = 0; i < kWaves; ++i) own = then(own, sh.tile[forward ? i : kWaves - 1 - i][lane]);
    publish(ch.seg + order * stride + at, own);
    fan = order % kFan == kFan - 1;  // ... and that of its fan
  }
#pragma unroll 1
  for (;; fan = false) {
    p = published(ch.seg + at, ch.fan + at, fan ? order - (kFan - 1) : first(i0), fan ? order : first(i1), stride, ch.head);
    if (!fan) break;
    publish(ch.fan + order / kFan * stride + at, then(p, own));
  }
  sh.part[w][lane] = p;
  __syncthreads();
  Map m = none;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) m = then(m, sh.part[i][lane]);
  return m;
}

// The work-group's place: which channels, which segment in the chain's order.
template <int W>
__device__ __forceinline__ void place(unsigned* order, const Chain& ch, long& group, int& seg) {
  seg = 0;
  group = blockIdx.x;
  if (W == kWaves && ch.segs > 1) {
    group = blockIdx.x % (uint32_t)ch.groups;
    if (threadIdx.x == 0) *order = atomicAdd(ch.next + group * kNextPitch, 1u);
    __syncthreads();
    seg = uniform((int)*order);
  }
}

template <typename DT>
__device__ __forceinline__ bool small_gates(const typename Chan<DT>::raw (&gr)[kTT]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kTT; ++i) most = max(most, __float_as_uint(Chan<DT>::get(gr[i])) & 0x7fffffffu);
  return __all(most <= __float_as_uint(kGateMost));  // NaN and infinity lie above
}

// Folds the tile's steps into its map; keeps a and u = (1 - a) x of each.
// MASKED: some step is padding or starts anew, or some gate is beyond
// kGateMost.
template <bool MASKED, typename DT>
__device__ __forceinline__ Map fold(float (&A)[kTT], float (&U)[kTT], const typename Chan<DT>::raw (&xr)[kTT],
                                    const typename Chan<DT>::raw (&gr)[kTT], const Tile& k) {
  Map m{1.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kTT; ++i) {
    if (MASKED && i >= k.some) continue;
    const float g = Chan<DT>::get(gr[i]), x = Chan<DT>::get(xr[i]);
    if constexpr (MASKED) {
      const float2 p = gate_pair_any(g);
      const bool live = i < k.live;
      A[i] = live ? (k.reset(i) ? -1.0f : p.x) : 1.0f;
      U[i] = live ? p.y * x : 0.0f;
      m = then(m, {A[i], U[i]});
    } else {
      const float2 p = gate_pair_small(g);
      A[i] = p.x;
      U[i] = p.y * x;
      m.A *= p.x;
      m.U = fmaf(p.x, m.U, U[i]);
    }
  }
  if constexpr (!MASKED) m.A = both_positive(m.A, 1.0f);  // (a gate within kGateMost is not 0)
  return m;
}

template <typename DT, bool STREAM, int W>
__global__ void __launch_bounds__(64 * W, W == kWaves ? 6 : 4) k_linrec_split(const LinrecArgs a, const Chain ch, int waves) {
  __shared__ Shared<W> sh;
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const long C = (long)a.B * a.H;
  int seg;
  long group;
  place<W>(&sh.order, ch, group, seg);
  Tile k(group, ((ch.seg0 + seg) * waves + w) * kTT, a.T, a.B, a.H, a.lengths);
  Resets<kTT> rb;
  rb.ask(a.resets, k, k.t0, a.T, a.B);
  typename Chan<DT>::raw xr[kTT], gr[kTT];
  load_tile<DT>(gr, a.gate, k);
  load_tile<DT>(xr, a.x, k);
  k.rs = rb.bits(a.resets, k, k.t0, a.T, a.B);
  float h = w == 0 && ch.enter && k.on ? ch.enter[k.c] : 0.0f;
  float A[kTT], U[kTT];
  const bool whole = k.whole() && small_gates<DT>(gr);
  sh.tile[w][lane] = whole ? fold<false, DT>(A, U, xr, gr, k) : fold<true, DT>(A, U, xr, gr, k);
  if (w == 0) sh.enter[lane] = h;  // read once, before anything of this row may be written
  __syncthreads();
  h = sh.enter[lane];
  if constexpr (W == kWaves)
    if (ch.segs > 1) h = apply(before(sh, ch, seg, group, true), h);
#pragma unroll
  for (int i = 0; i < W - 1; ++i)
    if (i < w) h = apply(sh.tile[i][lane], h);
  if (a.states && k.on && k.nt > 0) a.states[(long)(k.t0 / kTT) * C + k.c] = h;
  Rows<DT, STREAM> y(SeqView{a.y, C, a.H}, k, k.t0);
  if (whole) {
#pragma unroll
    for (int i = 0; i < kTT; ++i, y.move(y.st)) {
      h = fmaf(A[i], h, U[i]);
      y.put(h);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kTT; ++i, y.move(y.st)) {
      if (i < k.some) h = apply({A[i], U[i]}, h);
      if (i < k.nt && k.on) y.put(i < k.live ? h : 0.0f);
    }
  }
  if (ch.leave && k.on && k.t0 < ch.t1 && ch.t1 - k.t0 <= kTT) ch.leave[k.c] = h;
}

// The gradient's tile: a and 1 - a of its steps, what h_{t-1} puts into dgate,
// and the map of R:
//   R_out = sum_i (prod_{j <= i} a_j) dy_i + (prod a) R_in.
template <bool MASKED, typename DT>
__device__ __forceinline__ Map fold_grad(float (&A)[kTT], float (&M)[kTT], float (&G)[kTT], float h,
                                         const typename Chan<DT>::raw (&xr)[kTT],
                                         const typename Chan<DT>::raw (&gr)[kTT],
                                         const typename Chan<DT>::raw (&dr)[kTT], const Tile& k) {
  Map r{1.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kTT; ++i) {
    if (MASKED && i >= k.some) continue;
    const float g = Chan<DT>::get(gr[i]), x = Chan<DT>::get(xr[i]), d = Chan<DT>::get(dr[i]);
    const float2 p = MASKED ? gate_pair_any(g) : gate_pair_small(g);
    A[i] = p.x;
    M[i] = p.y;
    if (MASKED && k.reset(i)) h = 0.0f;
    G[i] = p.x * p.y * (h - x);
    const float to = fmaf(p.x, h, p.y * x);
    if constexpr (MASKED) {
      if (i < k.live) {
        h = to;
        if (k.reset(i)) r.A = -1.0f;
        if (!(r.A < 0.0f)) {
          r.A = both(r.A, p.x);
          r.U = fmaf(r.A, d, r.U);
        }
      }
    } else {
      h = to;
      r.A = both_positive(r.A, p.x);
      r.U = fmaf(r.A, d, r.U);
    }
  }
  return r;
}

template <bool MASKED, typename DT, bool STREAM>
__device__ __forceinline__ float emit_grad(const float (&A)[kTT], const float (&M)[kTT], const float (&G)[kTT], float R,
                                           const typename Chan<DT>::raw (&dr)[kTT], const Tile& k,
                                           const LinrecGradArgs& a) {
  Rows<DT, STREAM> dx(a.dx, k, k.t0 + kTT - 1), dg(a.dgate, k, k.t0 + kTT - 1);
#pragma unroll
  for (int i = kTT - 1; i >= 0; --i, dx.move(-dx.st), dg.move(-dg.st)) {
    float ox = 0.0f, og = 0.0f;
    if (!MASKED || i < k.some) {
      const bool live = !MASKED || i < k.live;
      const float D = R + Chan<DT>::get(dr[i]);
      ox = live ? M[i] * D : 0.0f;
      og = live ? G[i] * D : 0.0f;
      R = live ? (MASKED && k.reset(i) ? 0.0f : A[i] * D) : R;
    }
    if (!MASKED || (i < k.nt && k.on)) {
      dx.put(ox);
      dg.put(og);
    }
  }
  return R;
}

template <typename DT, bool STREAM, int W>
__global__ void __launch_bounds__(64 * W, 4) k_linrec_grad_split(const LinrecGradArgs a, const Chain ch, int waves) {
  __shared__ Shared<W> sh;
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  int order;
  long group;
  place<W>(&sh.order, ch, group, order);
  const int seg = ch.seg0 + ch.segs - 1 - order;  // the chain runs from the last segment to the first
  Tile k(group, (seg * waves + w) * kTT, a.T, a.B, a.H, a.lengths);
  Resets<kTT> rb;
  rb.ask(a.resets, k, k.t0, a.T, a.B);
  typename Chan<DT>::raw xr[kTT], gr[kTT], dr[kTT];
  load_tile<DT>(gr, a.gate, k);
  load_tile<DT>(xr, a.x, k);
  load_tile<DT>(dr, a.dy, k);
  const float h = k.on && k.nt > 0 ? a.states[(long)(k.t0 / kTT) * a.B * a.H + k.c] : 0.0f;
  k.rs = rb.bits(a.resets, k, k.t0, a.T, a.B);
  float R = w == waves - 1 && ch.enter && k.on ? ch.enter[k.c] : 0.0f;
  float A[kTT], M[kTT], G[kTT];
  const bool whole = k.whole() && small_gates<DT>(gr);
  sh.tile[w][lane] = whole ? fold_grad<false, DT>(A, M, G, h, xr, gr, dr, k) : fold_grad<true, DT>(A, M, G, h, xr, gr, dr, k);
  if (w == waves - 1) sh.enter[lane] = R;  // read once, before anything of this row may be written
  __syncthreads();
  R = sh.enter[lane];
  if constexpr (W == kWaves)
    if (ch.segs > 1) R = apply(before(sh, ch, order, group, false), R);
#pragma unroll
  for (int i = W - 1; i > 0; --i)
    if (i > w && i < waves) R = apply(sh.tile[i][lane], R);
  R = whole ? emit_grad<false, DT, STREAM>(A, M, G, R, dr, k, a) : emit_grad<true, DT, STREAM>(A, M, G, R, dr, k, a);
  if (ch.leave && k.on && k.t0 == ch.t0) ch.leave[k.c] = R;
}

// Empties the maps of a launch, sets its counters to 0, and copies the state that enters it (which the
// last segment's result may overwrite); the first one clears the status words.
__global__ void __launch_bounds__(256) k_linrec_init(const Chain ch, long words, const float* from, long C, bool first) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, step = (long)gridDim.x * 256;
  if (first && i < 2) ch.head[kSyncErr + i] = 0;
  for (long j = i; j < ch.groups; j += step) ch.next[j * kNextPitch] = 0;
  for (long j = i; j < words; j += step) ch.seg[j] = kEmpty;
  if (from)
    for (long j = i; j < C; j += step) const_cast<float*>(ch.enter)[j] = from[j];
}

// How a call is split.  waves = 0: not at all.  A gradient of 2 to 16 steps is
// one tile a work-group whatever the channels (the walk requests a whole tile's
// values, the steps past the end too); the forward call walks these.  Measured,
// walk against one tile, gradient of 4 steps: 64 fp32 channels 6.2 and 4.9 us,
// 65536 7.9 and 5.6, 262144 bf16 ones 11.5 and 8.9; of 16 steps 5.8 and 4.1, 8.0
// and 5.6, 12.8 and 10.5; forward of 4 steps 3.4 and 4.2, 4.0 and 4.8, 5.6 and 7.1.
struct Plan {
  int waves;  // tiles of a segment
  long segs;
};
Plan plan(int dtype, int T, int B, int H, bool grad) {
  const long groups = ((long)B * H + 63) / 64, tiles = ((long)T + kTT - 1) / kTT;
  if (T <= 1 || (tiles == 1 && !grad)) return {0, 0};
  if (tiles > 1 && groups >= (dtype == WM_FP32 ? kWalk32 : kWalk16)) return {0, 0};
  if (tiles <= kWide) return {(int)tiles, 1};
  return {kWaves, (tiles + kWaves - 1) / kWaves};
}

// The workspace of a call with several segments.
constexpr size_t kHeadBytes = kSyncWords * sizeof(unsigned);
long pad_channels(int B, int H) { return ((long)B * H + 63) / 64 * 64; }  // whole groups
constexpr size_t kNextBytes = kNextPitch * sizeof(unsigned);  // a group's
long map_words(long segs, long channels) { return (segs + segs / kFan) * channels; }

// Runs go(Chain) for every launch of a call, in order; `from` is the state that enters the call, `to` the one that leaves it.
template <typename F>
hipError_t run_chain(int T, int B, int H, const Plan& p, void* ws, const float* from, float* to, bool reverse,
                     hipStream_t s, F go) {
  const long C = (long)B * H, pad = pad_channels(B, H);
  Chain ch{};
  ch.groups = pad / 64;
  if (p.segs == 1) {
    ch.enter = from;
    ch.leave = to;
    ch.segs = 1;
    ch.t1 = T;
    return go(ch);
  }
  const long most = std::min<long>(p.segs, kMaxSegs);
  char* base = reinterpret_cast<char*>(ws);
  ch.head = reinterpret_cast<unsigned*>(base);
  ch.next = reinterpret_cast<unsigned*>(base + kHeadBytes);
  ch.seg = reinterpret_cast<unsigned long long*>(base + kHeadBytes + ch.groups * kNextBytes);
  float* enter = reinterpret_cast<float*>(ch.seg + map_words(most, pad));
  float* carry = enter + pad;
  const long launches = (p.segs + kMaxSegs - 1) / kMaxSegs;
  for (long n = 0; n < launches; ++n) {
    const long s0 = (reverse ? launches - 1 - n : n) * kMaxSegs;
    ch.seg0 = (int)s0;
    ch.segs = (int)std::min<long>(kMaxSegs, p.segs - s0);
    ch.t0 = (int)(s0 * kSeg);
    ch.t1 = (int)std::min<long>(T, (s0 + ch.segs) * kSeg);
    ch.fan = ch.seg + ch.segs * pad;
    const float* f = n == 0 ? from : carry;
    ch.enter = f ? enter : nullptr;
    ch.leave = n == launches - 1 ? to : carry;
    const long words = map_words(ch.segs, pad);
    const unsigned grid = (unsigned)std::min<long>(1024, (std::max(words, C) + 255) / 256);
    hipError_t e = launch("linrec_init", k_linrec_init, dim3(grid), dim3(256), 0, s, ch, words, f, C, n == 0);
    if (e == hipSuccess) e = go(ch);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename W, typename S, typename A>
hipError_t run(const char* name, int dtype, W walk, W step, S split, S wide, A a, const float* from, float* to,
               bool reverse, hipStream_t s) {
  const Plan p = plan(dtype, a.T, a.B, a.H, reverse);
  if (linrec_workspace(a.T, a.B, a.H) == 0) a.ws = nullptr;
  if (p.waves == 0) {
    const long groups = ((long)a.B * a.H + 63) / 64;
    return launch(name, a.T <= 1 ? step : walk, dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, s, a);
  }
  return run_chain(a.T, a.B, a.H, p, a.ws, from, to, reverse, s, [&](const Chain& ch) {
    return launch(name, p.waves > kWaves ? wide : split, dim3((unsigned)(ch.groups * ch.segs)), dim3(64u * p.waves), 0, s, a, ch, p.waves);
  });
}

}  // namespace

size_t linrec_states(int T, int B, int H) { return ((size_t)T + kTT - 1) / kTT * B * H * sizeof(float); }

size_t linrec_workspace(int T, int B, int H) {
  const Plan p = plan(WM_BF16, T, B, H, false);  // (split wherever fp32 is, and beyond)
  if (p.segs <= 1) return 0;
  const long pad = pad_channels(B, H);
  return kHeadBytes + (size_t)pad / 64 * kNextBytes + (size_t)map_words(std::min<long>(p.segs, kMaxSegs), pad) * 8 +
         (size_t)pad * 2 * sizeof(float);
}

hipError_t launch_linrec(int dtype, const LinrecArgs& a, hipStream_t s) {
  auto go = [&](auto dt) {
    typedef decltype(dt) DT;
    const bool stream = (long)a.T * a.B * a.H * (long)sizeof(DT) >= kStreamBytes;
    return run("linrec", dtype, stream ? k_linrec_walk<DT, kTT, true> : k_linrec_walk<DT, kTT, false>,
               k_linrec_walk<DT, 1, false>,
               stream ? k_linrec_split<DT, true, kWaves> : k_linrec_split<DT, false, kWaves>,
               stream ? k_linrec_split<DT, true, kWide> : k_linrec_split<DT, false, kWide>, a, a.h0, a.h_T, false, s);
  };
  return dtype == WM_FP32 ? go(0.0f) : go(bf16_t());
}

hipError_t launch_linrec_grad(int dtype, const LinrecGradArgs& a, hipStream_t s) {
  auto go = [&](auto dt) {
    typedef decltype(dt) DT;
    const bool stream = 2L * a.T * a.B * a.H * (long)sizeof(DT) >= kStreamBytes;
    return run("linrec_grad", dtype, stream ? k_linrec_grad_walk<DT, kTT, true> : k_linrec_grad_walk<DT, kTT, false>,
               k_linrec_grad_walk<DT, 1, false>,
               stream ? k_linrec_grad_split<DT, true, kWaves> : k_linrec_grad_split<DT, false, kWaves>,
               stream ? k_linrec_grad_split<DT, true, kWide> : k_linrec_grad_split<DT, false, kWide>, a, a.dh_T, a.dh0, true,
               s);
  };
  return dtype == WM_FP32 ? go(0.0f) : go(bf16_t());
}

}  // namespace wm
