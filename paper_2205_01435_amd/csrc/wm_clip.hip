// The global norm of a list of gradient tensors, and the tensors scaled to it:
//   N = sqrt(sum over all tensors of sum g^2),  out = g (N > max ? max / N : 1).
// Squares are summed in 64 bits: fp32 squares overflow from |g| = 1.8e19 and
// vanish below 1e-23, and the sum runs over up to billions of terms (the 64-bit
// multiply-add costs less than the bytes it works on).  The tensors are cut
// into chunks of equal size, dealt to the work-groups in a fixed way; every
// work-group's sum has its place in the workspace, and each work-group of the
// second launch adds them all in one order, so that the result depends on the
// tensors alone.
//
// Bound by memory: the values are read twice (the second time from the
// last-level cache where the list fits it: from its end, which was read last)
// and written once.  Measured, 153 tensors, 270 MB: sum 45 us (6.0 TB/s, part of
// it from the cache), scale 88 us (6.2 TB/s).  Chunks in strides over the list keep
// the work-groups within some MB of each other; a range of the list for each took
// the sum from 70 to 86 us.  Arrays are aligned to their element only; the hardware
// takes 16-byte accesses at such addresses.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                       // 16-byte pieces of a thread
constexpr int kChunkBytes = kThreads * kPer * 16;
constexpr int kPerLaunch = 176;               // tensors whose table fits a launch's arguments
constexpr int kGroups = 2048;                 // work-groups of a launch: eight a CU, each over chunks in strides

typedef uint32_t __attribute__((ext_vector_type(4))) u32x4;
typedef u32x4 __attribute__((aligned(2))) u32x4_2;

// STREAM: past the caches.
template <bool STREAM>
__device__ __forceinline__ void put_piece(char* p, u32x4 v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_2*>(p));
  else
    *reinterpret_cast<u32x4_2*>(p) = v;
}

struct Table {
  int n;                        // tensors of this launch
  uint32_t part0;               // place of its first chunk's sum
  uint32_t first[kPerLaunch + 1]; // chunks before each tensor
  const void* in[kPerLaunch];
  void* out[kPerLaunch];
  uint16_t last[kPerLaunch];    // bytes of its last chunk, less one; the top bit: bf16
};
static_assert(sizeof(Table) + 24 <= 4096, "a launch's arguments");

// A chunk of a list: where, how many bytes.
struct Chunk {
  const char* in;
  char* out;
  int bytes;
  bool bf16;
  __device__ Chunk(const Table& t, uint32_t c) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (t.first[mid] <= c)
        lo = mid;
      else
        hi = mid;
    }
    const int64_t from = (int64_t)(c - t.first[lo]) * kChunkBytes;
    bf16 = t.last[lo] >> 15;
    bytes = c + 1 < t.first[lo + 1] ? kChunkBytes : (t.last[lo] & 0x7fff) + 1;
    in = static_cast<const char*>(t.in[lo]) + from;
    out = static_cast<char*>(t.out[lo]) + from;
  }
  __device__ bool whole() const { return bytes == kChunkBytes; }
  __device__ u32x4 load(int at) const { return *reinterpret_cast<const u32x4_2*>(in + at); }
  // the thread's pieces of a whole chunk
  __device__ void load(u32x4 (&r)[kPer]) const {
    if (whole())
#pragma unroll
      for (int k = 0; k < kPer; ++k) r[k] = load((k * kThreads + threadIdx.x) * 16);
  }
};
// The four waves' sums, in order.
__device__ __forceinline__ double group_sum(double v, double* sh) {
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

__device__ __forceinline__ double squares(u32x4 r, bool bf16, double s) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (bf16) {
      const double a = __uint_as_float(r[j] << 16), b = __uint_as_float(r[j] & 0xffff0000u);
      s = fma(a, a, s);
      s = fma(b, b, s);
    } else {
      const double a = __uint_as_float(r[j]);
      s = fma(a, a, s);
    }
  }
  return s;
}

__global__ void __launch_bounds__(kThreads) k_clip_sum(const Table t, double* part) {
  __shared__ double sh[4];
  const uint32_t all = t.first[t.n];
  double s = 0.0;
  Chunk next(t, blockIdx.x);
  u32x4 ahead[kPer];
  next.load(ahead);
  for (uint32_t i = blockIdx.x; i < all; i += gridDim.x) {
    const Chunk c = next;
    u32x4 r[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) r[k] = ahead[k];
    if (i + gridDim.x < all) {
      next = Chunk(t, i + gridDim.x);
      next.load(ahead);
    }
    if (c.whole()) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) s = squares(r[k], c.bf16, s);
    } else {
      int at = threadIdx.x * 16;
      for (; at + 16 <= c.bytes; at += kThreads * 16) s = squares(c.load(at), c.bf16, s);
      const int es = c.bf16 ? 2 : 4;  // the values beyond the last whole piece: one lane's
      for (; at < c.bytes; at += es) {
        const double g = c.bf16 ? DType<bf16_t>::load(reinterpret_cast<const bf16_t*>(c.in + at), 0)
                                : DType<float>::load(reinterpret_cast<const float*>(c.in + at), 0);
        s = fma(g, g, s);
      }
    }
  }
  s = group_sum(s, sh);
  if (threadIdx.x == 0) part[t.part0 + blockIdx.x] = s;
}

// The factor of every value.  Below fp32's normal numbers (values of 1e30 to a norm
// of 1e-10) it has too few bits there: the product is then one of 64 bits.
struct Factor {
  float f;
  double d;
  bool small;
  __device__ Factor(double v) : f((float)v), d(v), small(__any(v < 0x1p-126)) {}  // (the same in every lane)
  __device__ float of(float g) const {
    if (small) return (float)(d * (double)g);
    return f * g;
  }
  __device__ u32x4 of(u32x4 r, bool bf16) const {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      r[j] = bf16 ? pack2_bf16(of(__uint_as_float(r[j] << 16)), of(__uint_as_float(r[j] & 0xffff0000u)))
                  : __float_as_uint(of(__uint_as_float(r[j])));
    return r;
  }
};

template <bool STREAM>
__global__ void __launch_bounds__(kThreads) k_clip_scale(const Table t, const double* part, uint32_t parts, float max_norm,
                                                         float* norm) {
  __shared__ double sh[4];
  const uint32_t all = t.first[t.n];
  Chunk next(t, all - 1 - blockIdx.x);  // backwards: what was read last is read first
  u32x4 ahead[kPer];
  next.load(ahead);
  double s = 0.0;
#pragma unroll 8
  for (uint32_t k = threadIdx.x; k < parts; k += kThreads) s += part[k];
  const double N = sqrt(group_sum(s, sh));
  const float seen = (float)N;  // what the caller sees decides: infinite where fp32 cannot hold it
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = seen;
  const Factor by(N > (double)max_norm && seen < INFINITY ? (double)max_norm / N : 1.0);
  for (uint32_t i = blockIdx.x; i < all; i += gridDim.x) {
    const Chunk c = next;
    u32x4 r[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) r[k] = ahead[k];
    if (i + gridDim.x < all) {
      next = Chunk(t, all - 1 - (i + gridDim.x));
      if (by.f != 1.0f || next.in != next.out) next.load(ahead);
    }
    if (by.f == 1.0f && c.in == c.out) continue;  // in place, and within the limit
    if (c.whole()) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        put_piece<STREAM>(c.out + (k * kThreads + threadIdx.x) * 16, by.of(r[k], c.bf16));
    } else {
      int at = threadIdx.x * 16;
      for (; at + 16 <= c.bytes; at += kThreads * 16)
        *reinterpret_cast<u32x4_2*>(c.out + at) = by.of(c.load(at), c.bf16);
      const int es = c.bf16 ? 2 : 4;
      for (; at < c.bytes; at += es) {
        if (c.bf16)
          DType<bf16_t>::store(reinterpret_cast<bf16_t*>(c.out + at), 0,
                               by.of(DType<bf16_t>::load(reinterpret_cast<const bf16_t*>(c.in + at), 0)));
        else
          *reinterpret_cast<float*>(c.out + at) = by.of(*reinterpret_cast<const float*>(c.in + at));
      }
    }
  }
}

__global__ void k_clip_none(float* norm) { *norm = 0.0f; }

int64_t bytes_of(const wm_grad_tensor& t) { return t.n * (t.dtype == WM_FP32 ? 4 : 2); }
int64_t chunks_of(const wm_grad_tensor& t) { return (bytes_of(t) + kChunkBytes - 1) / kChunkBytes; }

// Runs f on the table and the work-groups of each launch; the sums of them all.
template <typename F>
hipError_t tables(int n, const wm_grad_tensor* t, uint32_t& part0, F f) {
  part0 = 0;
  for (int i = 0; i < n;) {
    Table tab;
    tab.n = 0;
    tab.part0 = part0;
    tab.first[0] = 0;
    for (; i < n && tab.n < kPerLaunch; ++i) {
      if (t[i].n == 0) continue;
      const int k = tab.n++;
      tab.in[k] = t[i].grad;
      tab.out[k] = t[i].out;
      tab.last[k] = (uint16_t)((bytes_of(t[i]) - 1) % kChunkBytes | (t[i].dtype == WM_FP32 ? 0 : 0x8000));
      tab.first[k + 1] = tab.first[k] + (uint32_t)chunks_of(t[i]);
    }
    if (tab.n == 0) break;
    const uint32_t groups = std::min<uint32_t>(tab.first[tab.n], kGroups);
    part0 += groups;
    const hipError_t e = f(tab, groups);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t clip_workspace(int n, const wm_grad_tensor* t) {
  uint32_t parts;
  (void)tables(n, t, parts, [](const Table&, uint32_t) { return hipSuccess; });
  return (size_t)parts * sizeof(double);
}

hipError_t launch_clip(int n, const wm_grad_tensor* t, float max_norm, float* norm, void* ws, hipStream_t s) {
  double* part = reinterpret_cast<double*>(ws);
  uint32_t parts;
  hipError_t e = tables(n, t, parts, [&](const Table& tab, uint32_t groups) {
    return launch("clip_sum", k_clip_sum, dim3(groups), dim3(kThreads), 0, s, tab, part);
  });
  if (e != hipSuccess) return e;
  if (parts == 0) return launch("clip_none", k_clip_none, dim3(1), dim3(1), 0, s, norm);
  int64_t bytes = 0;
  for (int i = 0; i < n; ++i) bytes += bytes_of(t[i]);
  uint32_t again;
  return tables(n, t, again, [&](const Table& tab, uint32_t groups) {
    return launch("clip_scale", bytes >= kStreamBytes ? k_clip_scale<true> : k_clip_scale<false>, dim3(groups),
                  dim3(kThreads), 0, s, tab, (const double*)part, parts, max_norm, tab.part0 == 0 ? norm : nullptr);
  });
}

}  // namespace wm
