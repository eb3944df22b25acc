// Rows of an action table for logged actions, scaled, and the table's
// gradient (the one-hot product of the world model's input as a gather, and
// its transpose).
//   y_i = s E[a_i], 0 where a_i is outside [0, V);  dE_v = s sum_{a_i = v} dy_i.
//
// The gradient of a small table (k_embed_scan) looks for each row's positions in
// the whole list, a part of it in every work-group, and adds the parts in order;
// that of few positions (k_embed_few) does so for the tokens that occur.
// Otherwise it sorts the positions by token (stably, by 8-bit digits, least
// first; codes outside the table sort behind it), so that a row's positions lie
// together, and cuts the sorted list into equal chunks whatever the tokens are:
// a row that every token names costs as much as one row each.  A wave sums the
// runs of equal tokens of its chunk, 16 bytes a lane, and writes the rows that
// lie inside the chunk; the first and the last run, which may go on in the
// neighbouring chunks, become partial sums.  The last launch adds a row's
// partial sums in order and clears the rows that no token names: every row of
// the gradient is written once, and the order of each sum is fixed.
// All of it is bound by memory: dy is read once, the gradient written once.
// Measured, 81920 positions of 57600 rows of 1024 bf16 values (690 MB both
// ways): rows 54 us; gradient sort 23, sums 79 (168 MB read, 230 MB written or
// cleared), join 23: 3.9 TB/s in all.  7224 positions of 50 rows of 367 fp32
// values: rows 5 us, gradient 12, launches and first loads.
#include <algorithm>

#include "../../include/wm.h"
#include "wm_seq.h"
#include "wm_profile.h"

namespace wm {
namespace {

typedef uint32_t __attribute__((ext_vector_type(4))) u32x4;
typedef u32x4 __attribute__((aligned(2))) u32x4_2;
typedef u32x4 __attribute__((aligned(4))) u32x4_4;

// Sixteen bytes of a row as fp32 values.  Rows are aligned to their element
// only: the hardware takes 16-byte accesses at such addresses.
template <typename DT> struct Piece;
template <> struct Piece<float> {
  static constexpr int V = 4;
  __device__ static u32x4 load(const float* p) { return *reinterpret_cast<const u32x4_4*>(p); }
  __device__ static void get(u32x4 r, float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(r[j]);
  }
  __device__ static void store(float* p, const float* v) {
    *reinterpret_cast<u32x4_4*>(p) =
        u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
template <> struct Piece<bf16_t> {
  static constexpr int V = 8;
  __device__ static u32x4 load(const bf16_t* p) { return *reinterpret_cast<const u32x4_2*>(p); }
  __device__ static void get(u32x4 r, float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(r[j] << 16);
      v[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
  }
  __device__ static void store(bf16_t* p, const float* v) {
    *reinterpret_cast<u32x4_2*>(p) =
        u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
  }
};

// A row's last, partial piece is read and written as the last 16 bytes of the
// row, over the end of the piece before it: both hold the same values.  A row
// narrower than a piece goes value by value.
template <typename DT>
__device__ __forceinline__ u32x4 load_piece(const DT* row, int col, int H) {
  if (H >= Piece<DT>::V) return Piece<DT>::load(row + col);
  u32x4 r = {0u, 0u, 0u, 0u};
  constexpr int k = 4 / sizeof(DT);  // values of a word
#pragma unroll
  for (int j = 0; j < Piece<DT>::V; ++j)
    if (j < H) r[j / k] |= __float_as_uint(DType<DT>::load(row, j)) >> (j % k == 0 && k == 2 ? 16 : 0);
  return r;
}
// N values to a row of type DT.
template <typename DT, int N>
__device__ __forceinline__ void store_values(DT* row, int col, int H, const float* v) {
  if (H >= N) {
#pragma unroll
    for (int j = 0; j < N; j += Piece<DT>::V) Piece<DT>::store(row + col + j, v + j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < H) DType<DT>::store(row, j, v[j]);
  }
}
template <typename DT>
__device__ __forceinline__ int column(int piece, int H) {
  return max(min(piece * Piece<DT>::V, H - Piece<DT>::V), 0);
}

// L lanes a row.
template <typename DT, int L>
__global__ void __launch_bounds__(256) k_embed(const EmbedArgs a) {
  constexpr int V = Piece<DT>::V;
  const DT* table = reinterpret_cast<const DT*>(a.table);
  DT* out = reinterpret_cast<DT*>(a.out);
  const int t = threadIdx.x % L;
  const long step = (long)gridDim.x * (256 / L);
  for (long i = (long)blockIdx.x * (256 / L) + threadIdx.x / L; i < a.n; i += step) {
    const int tok = a.tokens[i];
    const bool ok = tok >= 0 && tok < a.V;
    const DT* from = table + (long)(ok ? tok : 0) * a.H;
    DT* to = out + i * a.out_ld;
    for (int p = t; p * V < a.H; p += L) {
      const int c = column<DT>(p, a.H);
      float v[V];
      u32x4 r = {0u, 0u, 0u, 0u};
      if (ok) r = load_piece(from, c, a.H);
      Piece<DT>::get(r, v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = ok ? a.scale * v[j] : 0.0f;
      store_values<DT, V>(to, c, a.H, v);
    }
  }
}

// ---------------------------------------------------------------------------
// Sorting the positions by token
// ---------------------------------------------------------------------------

constexpr int kDigits = 256;
// Positions that one work-group sorts by itself (two lists in LDS).  Measured
// against counting and placing by many: 1000 positions 4.2 against 8.5 us, 4000
// of one pass 7.2 against 9.4 and of two 11.6 against 17.3; 8000 of one pass
// 10.9 against 9.8, of two 18.5 against 18.9.
constexpr int kOne = 4096;
constexpr int kMaxTiles = 256; // tiles of a longer list

__device__ __forceinline__ uint32_t key_of(int tok, int V) { return tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V; }

// Lanes of the wave with the same digit as this one, among those in `in`.
__device__ __forceinline__ unsigned long long same_digit(uint32_t d, unsigned long long in) {
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const bool bit = (d >> b) & 1u;
    const unsigned long long m = __ballot(bit);
    in &= bit ? m : ~m;
  }
  return in;
}

// Places the entries [begin, end) of a wave, in order: `at[digit]` holds where
// its next entry of that digit goes.  get(i) is entry i as (key, position).
template <typename Get, typename Put>
__device__ __forceinline__ void place_run(int begin, int end, int shift, uint32_t* at, Get get, Put put) {
  const int lane = threadIdx.x & 63;
  for (int i0 = begin; i0 < end; i0 += 64) {
    const int i = i0 + lane;
    const bool in = i < end;
    uint2 e = make_uint2(0u, 0u);
    if (in) e = get(i);
    const uint32_t d = (e.x >> shift) & (kDigits - 1);
    const unsigned long long peers = same_digit(d, __ballot(in));
    const uint32_t rank = __popcll(peers & ((1ull << lane) - 1ull));
    uint32_t to = 0;
    if (in) to = at[d] + rank;
    // (every lane has read before the last of each digit's lanes writes: they are one wave)
    if (in && (peers >> lane) == 1ull) at[d] = to + 1u;
    if (in) put(to, e);
  }
}

// Exclusive sums of 256 counts, one a thread of the first 256.
__device__ __forceinline__ uint32_t scan256(uint32_t v, uint32_t* sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t o = __shfl_up(s, k);
    if (lane >= k) s += o;
  }
  if (w < 4 && lane == 63) sh[w] = s;
  __syncthreads();
  for (int i = 0; i < w && i < 3; ++i) s += sh[i];
  __syncthreads();
  return s - v;
}

// All passes of a short list in one work-group of 16 waves.
__global__ void __launch_bounds__(1024) k_embed_sort(const int32_t* tokens, int n, int V, int passes, uint32_t* keys,
                                                     uint32_t* pos) {
  __shared__ uint2 list[2][kOne];
  __shared__ uint32_t at[16][kDigits];
  __shared__ uint32_t sh[4];
  const int w = threadIdx.x >> 6, run = ((n + 15) / 16 + 63) / 64 * 64;
  for (int i = threadIdx.x; i < n; i += 1024) list[0][i] = make_uint2(key_of(tokens[i], V), (uint32_t)i);
  for (int p = 0; p < passes; ++p) {
    for (int i = threadIdx.x; i < 16 * kDigits; i += 1024) at[i / kDigits][i % kDigits] = 0;
    __syncthreads();
    const uint2* from = list[p & 1];
    uint2* to = list[(p & 1) ^ 1];
    const int begin = min(w * run, n), end = min(begin + run, n);
    for (int i = begin + (threadIdx.x & 63); i < end; i += 64) atomicAdd(&at[w][(from[i].x >> 8 * p) & (kDigits - 1)], 1u);
    __syncthreads();
    uint32_t total = 0;
    if (threadIdx.x < kDigits)
      for (int k = 0; k < 16; ++k) total += at[k][threadIdx.x];
    uint32_t base = scan256(total, sh);
    if (threadIdx.x < kDigits)
      for (int k = 0; k < 16; ++k) {
        const uint32_t c = at[k][threadIdx.x];
        at[k][threadIdx.x] = base;
        base += c;
      }
    __syncthreads();
    place_run(begin, end, 8 * p, at[w], [&](int i) { return from[i]; }, [&](uint32_t i, uint2 e) { to[i] = e; });
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n; i += 1024) {
    const uint2 e = list[passes & 1][i];
    keys[i] = e.x;
    pos[i] = e.y;
  }
}

struct SortArgs {
  const int32_t* tokens;        // the first pass's entries: positions 0 .. n - 1
  const uint32_t *keys, *pos;   // the others'
  uint32_t *keys_to, *pos_to;
  uint32_t* hist;               // [tiles][256]
  int n, V, tile, tiles, pass;
};
__device__ __forceinline__ uint2 entry(const SortArgs& a, int i) {
  return a.pass == 0 ? make_uint2(key_of(a.tokens[i], a.V), (uint32_t)i) : make_uint2(a.keys[i], a.pos[i]);
}

// How often each digit occurs in each tile.
__global__ void __launch_bounds__(1024) k_embed_hist(const SortArgs a) {
  __shared__ uint32_t cnt[kDigits];
  if (threadIdx.x < kDigits) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int begin = blockIdx.x * a.tile, end = min(begin + a.tile, a.n);
  for (int i = begin + threadIdx.x; i < end; i += 1024) {
    const uint32_t key = a.pass == 0 ? key_of(a.tokens[i], a.V) : a.keys[i];
    atomicAdd(&cnt[(key >> 8 * a.pass) & (kDigits - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kDigits) a.hist[blockIdx.x * kDigits + threadIdx.x] = cnt[threadIdx.x];
}

// Places a tile's entries behind those of smaller digits and of earlier tiles.
__global__ void __launch_bounds__(1024) k_embed_scatter(const SortArgs a) {
  __shared__ uint32_t at[16][kDigits];
  __shared__ uint32_t part[2][4][kDigits];
  __shared__ uint32_t sh[4];
  const int w = threadIdx.x >> 6, d = threadIdx.x % kDigits, q = threadIdx.x / kDigits;
  const int begin0 = blockIdx.x * a.tile, run = a.tile / 16;
  const int begin = min(begin0 + w * run, a.n), end = min(begin + run, a.n);
  for (int i = threadIdx.x; i < 16 * kDigits; i += 1024) at[i / kDigits][i % kDigits] = 0;
  uint32_t all = 0, before = 0;
#pragma unroll 4
  for (int t = q; t < a.tiles; t += 4) {
    const uint32_t c = a.hist[t * kDigits + d];
    all += c;
    before += t < (int)blockIdx.x ? c : 0u;
  }
  part[0][q][d] = all;
  part[1][q][d] = before;
  __syncthreads();
  for (int i = begin + (threadIdx.x & 63); i < end; i += 64) {
    const uint32_t key = a.pass == 0 ? key_of(a.tokens[i], a.V) : a.keys[i];
    atomicAdd(&at[w][(key >> 8 * a.pass) & (kDigits - 1)], 1u);
  }
  all = part[0][0][d] + part[0][1][d] + part[0][2][d] + part[0][3][d];
  before = part[1][0][d] + part[1][1][d] + part[1][2][d] + part[1][3][d];
  uint32_t base = scan256(all, sh) + before;  // (its barriers complete the counts)
  if (threadIdx.x < kDigits)
    for (int k = 0; k < 16; ++k) {
      const uint32_t c = at[k][d];
      at[k][d] = base;
      base += c;
    }
  __syncthreads();
  place_run(begin, end, 8 * a.pass, at[w], [&](int i) { return entry(a, i); },
            [&](uint32_t i, uint2 e) {
              a.keys_to[i] = e.x;
              a.pos_to[i] = e.y;
            });
}

// ---------------------------------------------------------------------------
// Sums over runs of equal tokens
// ---------------------------------------------------------------------------

struct RowsArgs {
  EmbedGradArgs g;
  const uint32_t *keys, *pos;  // sorted
  float* part;                 // [chunks][2][H]
  int32_t* start;              // [V + 1] each row's first sorted position
  int chunk, chunks, groups;   // groups: work-groups over the chunks
};

// First sorted position whose token is at least v.
__device__ __forceinline__ int lower_bound(const uint32_t* keys, int n, uint32_t v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (keys[mid] < v)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo;
}

// The first `groups` work-groups of a column block: a wave's chunk of sorted
// positions, for 64 pieces of the columns, eight rows of dy in flight.  The run
// at the chunk's begin is a partial sum of slot 0 if it began before the chunk
// or goes on after it; another run that goes on after it is one of slot 1.  The
// work-groups behind them look up where each row of the table begins (a search
// in the sorted list, beside the loads of the others: inside the joining launch
// it took 208 us for 57600 rows).
template <typename DT>
__global__ void __launch_bounds__(256) k_embed_rows(const RowsArgs a) {
  constexpr int V = Piece<DT>::V, kAhead = 8;
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= a.groups) {
    const long step = (long)(gridDim.x - a.groups) * 256;
    if (blockIdx.y == 0)
      for (long v = (long)(blockIdx.x - a.groups) * 256 + threadIdx.x; v <= a.g.V; v += step)
        a.start[v] = lower_bound(a.keys, (int)a.g.n, (uint32_t)v);
    return;
  }
  const int chunk = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (chunk >= a.chunks) return;
  const int H = a.g.H, piece = blockIdx.y * 64 + lane, col = column<DT>(piece, H);
  const bool on = piece * V < H;
  const DT* dy = reinterpret_cast<const DT*>(a.g.dout);
  const int n = (int)a.g.n, begin = chunk * a.chunk, end = min(begin + a.chunk, n);
  float* const part = a.part + (long)chunk * 2 * H;
  const uint32_t before = begin > 0 ? a.keys[begin - 1] : ~0u, after = end < n ? a.keys[end] : ~0u;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.0f;
  uint32_t run = a.keys[begin];  // the run's token
  bool first = true;             // ... is the chunk's first
  auto flush = [&](bool last) {
    if (run >= (uint32_t)a.g.V) return;  // codes outside the table
    const bool shared = (first && run == before) || (last && run == after);
    if (!on) return;
    if (shared) {
      store_values<float, V>(part + (first ? 0 : H), col, H, sum);
    } else {
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = a.g.scale * sum[j];
      store_values<float, V>(a.g.dtable + (long)run * H, col, H, v);
    }
  };
  for (int i0 = begin; i0 < end; i0 += 64) {
    const int m = min(64, end - i0);
    const uint32_t key = lane < m ? a.keys[i0 + lane] : 0u, pos = lane < m ? a.pos[i0 + lane] : 0u;
    for (int k0 = 0; k0 < m; k0 += kAhead) {
      if ((uint32_t)__builtin_amdgcn_readlane((int)key, k0) >= (uint32_t)a.g.V) break;  // only codes from here on
      u32x4 r[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const long row = (uint32_t)__builtin_amdgcn_readlane((int)pos, min(k0 + k, m - 1));
        r[k] = load_piece(dy + row * a.g.dout_ld, col, H);  // (lanes past the row's end: its end)
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (k0 + k >= m) break;
        const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)key, k0 + k);
        if (t != run) {
          flush(false);
          run = t;
          first = false;
#pragma unroll
          for (int j = 0; j < V; ++j) sum[j] = 0.0f;
        }
        float v[V];
        Piece<DT>::get(r[k], v);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += v[j];
      }
    }
    const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)key, m - 1);
    if (t >= (uint32_t)a.g.V && run < (uint32_t)a.g.V) {  // the table's last run, before the codes
      flush(false);
      run = t;
      first = false;
    }
  }
  flush(true);
}

// The sum of the partial sums of a row, `count` from chunk c on: those of slot 0
// but the first one where the row does not begin its chunk.
__device__ __forceinline__ float4 join(const RowsArgs& a, int c, int i0, int i1, bool inside, int col) {
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    float v[4];
    Piece<float>::get(load_piece(a.part + ((long)(c + i) * 2 + (i == 0 && inside)) * a.g.H, col, a.g.H), v);
    s.x += v[0];
    s.y += v[1];
    s.z += v[2];
    s.w += v[3];
  }
  return s;
}
__device__ __forceinline__ void put_row(const RowsArgs& a, uint32_t row, int col, float4 s) {
  const float v[4] = {a.g.scale * s.x, a.g.scale * s.y, a.g.scale * s.z, a.g.scale * s.w};
  store_values<float, 4>(a.g.dtable + (long)row * a.g.H, col, a.g.H, v);
}

// 64 pieces of four columns.  The first `joins` work-groups: sixteen chunks
// each, a wave a chunk; the wave adds up the row that begins in its chunk and
// goes on after it, and if it lies in more than kAlone chunks all waves do, each
// a part of them (200000 positions of 5 rows of 64 values: 23 us, with one wave
// each 146; 2 chunks as the bound cost the rows of some chunks 1.5 us).  The
// others: 64 rows each, cleared where no token names them.
constexpr int kAlone = 16;
constexpr int kClear = 64;
__global__ void __launch_bounds__(1024) k_embed_join(const RowsArgs a, int joins) {
  __shared__ int4 wide[16];  // row, first chunk, chunks, whether it begins inside the chunk
  __shared__ float4 sums[16][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), H = a.g.H;
  const int piece = blockIdx.y * 64 + lane, col = column<float>(piece, H);
  const bool on = piece * 4 < H;
  if ((int)blockIdx.x >= joins) {
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const long step = (long)(gridDim.x - joins) * kClear;
    for (long r0 = (long)(blockIdx.x - joins) * kClear; r0 < a.g.V; r0 += step)
      for (long r = r0 + w; r < min(r0 + kClear, (long)a.g.V); r += 16)
        if (a.start[r] == a.start[r + 1] && on) store_values<float, 4>(a.g.dtable + r * H, col, H, zero);
    return;
  }
  const int c = blockIdx.x * 16 + w;
  int4 mine = make_int4(-1, 0, 0, 0);
  if (c < a.chunks) {
    const int begin = c * a.chunk, end = min(begin + a.chunk, (int)a.g.n);
    const uint32_t key = a.keys[end - 1];
    if (key < (uint32_t)a.g.V && end < a.g.n && a.keys[end] == key && a.start[key] >= begin)
      mine = make_int4((int)key, c, (a.start[key + 1] - 1) / a.chunk - c + 1, a.start[key] > begin);
  }
  if (mine.z > 0 && mine.z <= kAlone) {
    const float4 s = join(a, c, 0, mine.z, mine.w, col);
    if (on) put_row(a, (uint32_t)mine.x, col, s);
    mine.x = -1;
  }
  if (lane == 0) wide[w] = mine;
  __syncthreads();
  for (int k = 0; k < 16; ++k) {
    const int4 r = wide[k];
    if (r.x < 0) continue;
    const int i0 = (int)((long)r.z * w / 16), i1 = (int)((long)r.z * (w + 1) / 16);
    float4 s = join(a, r.y, i0, i1, r.w, col);
    sums[w][lane] = s;
    __syncthreads();
    if (w == 0 && on) {
#pragma unroll
      for (int i = 1; i < 16; ++i) {
        const float4 v = sums[i][lane];
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
      }
      put_row(a, (uint32_t)r.x, col, s);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Small tables: no sorting
// ---------------------------------------------------------------------------

constexpr int kScan = 512;  // positions that a work-group looks through

struct ScanArgs {
  EmbedGradArgs g;
  float* part;  // [parts][V][H]; not used by a single one
};

// Adds to `sum` the rows of dy whose positions among the 64 from `at` on have
// token v, a piece of each a lane.
template <typename DT>
__device__ __forceinline__ void add_rows(float (&sum)[Piece<DT>::V], const EmbedGradArgs& g, int v, int at, int col) {
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 63, n = (int)g.n;
  const DT* dy = reinterpret_cast<const DT*>(g.dout);
  unsigned long long m = __ballot(at + lane < n && g.tokens[min(at + lane, n - 1)] == v);
  while (m) {
    u32x4 r[kAhead];
    const int count = __popcll(m);
    int q = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      q = m ? __builtin_ctzll(m) : q;  // (past the last one: that one again)
      m &= m - 1;
      r[k] = load_piece(dy + (long)(at + q) * g.dout_ld, col, g.H);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k >= count) break;
      float x[Piece<DT>::V];
      Piece<DT>::get(r[k], x);
#pragma unroll
      for (int j = 0; j < Piece<DT>::V; ++j) sum[j] += x[j];
    }
  }
}

// The sums of the work-group's kScan / 64 waves, in order; the column and its
// total of a thread that has one.
template <int V>
__device__ __forceinline__ bool add_waves(float (*sums)[64 * V], const float (&sum)[V], int H, int& c, float& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int j = 0; j < V; ++j) sums[w][lane * V + j] = sum[j];
  __syncthreads();
  const int piece = blockIdx.y * 64 + threadIdx.x / V;
  c = max(min(piece * V, H - V), 0) + threadIdx.x % V;
  if (threadIdx.x >= 64 * V || piece * V >= H || c >= H) return false;
  total = 0.0f;
#pragma unroll
  for (int i = 0; i < kScan / 64; ++i) total += sums[i][threadIdx.x];
  return true;
}

// A row of the table, 64 pieces of its columns, kScan positions: every wave
// looks through 64 of them and adds up the rows of dy that belong to it; the
// waves' sums meet in LDS.  A row's parts are neighbouring work-groups: on
// different XCDs, where one token has all positions.
template <typename DT>
__global__ void __launch_bounds__(kScan) k_embed_scan(const ScanArgs a, int parts) {
  constexpr int V = Piece<DT>::V;
  __shared__ float sums[kScan / 64][64 * V];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), H = a.g.H;
  const int v = blockIdx.x / (unsigned)parts, part = blockIdx.x - v * parts, at = part * kScan + w * 64;
  const int col = column<DT>(blockIdx.y * 64 + lane, H);
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.0f;
  add_rows<DT>(sum, a.g, v, at, col);
  int c;
  float total;
  if (!add_waves<V>(sums, sum, H, c, total)) return;
  const long to = (long)v * H + c;
  if (parts == 1)
    a.g.dtable[to] = a.g.scale * total;
  else
    a.part[(long)part * a.g.V * H + to] = total;
}

// Adds the parts in order.
__global__ void __launch_bounds__(256) k_embed_parts(const ScanArgs a, int parts) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, size = (long)a.g.V * a.g.H;
  if (i >= size) return;
  float total = 0.0f;
#pragma unroll 8
  for (int p = 0; p < parts; ++p) total += a.part[p * size + i];
  a.g.dtable[i] = a.g.scale * total;
}

// Few positions of a larger table, in one launch.  The first n work-groups: a
// position each; if its token has not come earlier, all its positions' rows are
// summed, the waves taking 64 positions in turn, and their sums meet in LDS.
// The others: `rows` rows of the table each, cleared where no token names them.
template <typename DT>
__global__ void __launch_bounds__(kScan) k_embed_few(const EmbedGradArgs a, int rows) {
  constexpr int V = Piece<DT>::V;
  __shared__ float sums[kScan / 64][64 * V];
  const int H = a.H, n = (int)a.n, i = blockIdx.x;
  if (i >= n) {
    if (blockIdx.y > 0) return;
    uint32_t* named = reinterpret_cast<uint32_t*>(sums);
    const int r0 = (i - n) * rows, count = min(rows, a.V - r0);
    if ((int)threadIdx.x < count) named[threadIdx.x] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < n; j += kScan) {
      const uint32_t r = (uint32_t)a.tokens[j] - (uint32_t)r0;
      if (r < (uint32_t)count) named[r] = 1;
    }
    __syncthreads();
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t pieces = (uint32_t)(H + 3) / 4, all = pieces * count;
    for (uint32_t t = threadIdx.x; t < all; t += kScan) {
      const uint32_t r = t / pieces;
      if (!named[r])
        store_values<float, 4>(a.dtable + (long)(r0 + (int)r) * H, column<float>((int)(t - r * pieces), H), H, zero);
    }
    return;
  }
  const int v = a.tokens[i], col = column<DT>(blockIdx.y * 64 + (threadIdx.x & 63), H);
  if (v < 0 || v >= a.V) return;
  int earlier = 0;
  for (int j = threadIdx.x; j < i; j += kScan) earlier |= a.tokens[j] == v;
  if (__syncthreads_or(earlier)) return;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.0f;
  for (int at = threadIdx.x & ~63; at < n; at += kScan) add_rows<DT>(sum, a, v, __builtin_amdgcn_readfirstlane(at), col);
  int c;
  float total;
  if (add_waves<V>(sums, sum, H, c, total)) a.dtable[(long)v * H + c] = a.scale * total;
}

// The most work-groups (in columns of 256) of a gradient without sorting.
// Measured against sorting, with tokens that name all rows alike and one row
// only: 1024 rows of 64 from 500 positions (1024 work-groups) 3.8 and
// 9.3 against 14.5 and 14.0 us, 50 of 367 from 7224 (1500) 11.1 and 14.4 against
// 17.2 and 21.8, 128 of 64 from 16384 (4096) 13.8 and 14.0 against 17.4 and
// 26.3, 128 of 367 from 16384 (8192) 24.0 and 21.1 against 18.8 and 29.4, 128 of
// 64 from 40000 (10112) 28.5 and 19.7 against 19.4 and 45.2.
constexpr long kScanGroups = 4096;
constexpr long kScanParts = 64;  // ... and the most parts, which are added one after the other
// Positions up to which a larger table is done in one launch.  Measured against
// sorting, tokens that name all rows alike and one row only: 1000 positions of
// 4000 rows of 64 fp32 values 5.4 against 16.0 us, of 57600 of 512 bf16 ones 19.8
// against 29.9; 1500 of 4000 of 64 7.0 and 22.6 against 17.1 and 19.2, 3000 11.5
// and 42.2 against 19.6 and 25.1.
constexpr int kFew = 1024;

// How a call is cut.
struct Plan {
  int parts;                // without sorting; 0: with
  bool few;                 // one launch, no workspace
  int passes, tile, tiles;  // of the sort (tiles 0: one work-group)
  int chunk, chunks;
  size_t hist, start, part, total;  // workspace, after the keys and positions twice: counts, rows' begins, partial sums
};
Plan plan(long n, int V, int H) {
  Plan p{};
  const long columns = (H + 255) / 256;
  const long parts = (n + kScan - 1) / kScan, most_parts = std::min(kScanParts, kScanGroups / ((long)V * columns));
  if (n > 0 && parts <= most_parts) p.parts = (int)parts;
  p.few = n > 0 && p.parts == 0 && n <= kFew && n * columns <= kScanGroups;
  p.passes = 1;
  while (p.passes < 4 && (uint64_t)V >> (8 * p.passes)) ++p.passes;  // the keys are 0 .. V
  if (n > kOne) {
    p.tile = (int)(((n + kMaxTiles - 1) / kMaxTiles + 1023) / 1024 * 1024);
    p.tiles = (int)((n + p.tile - 1) / p.tile);
  }
  // about 16 waves for every CU, whole groups of loads
  const long blocks = (H + 255) / 256;
  p.chunk = (int)std::min<long>(128, std::max<long>(16, (n * blocks / 4096 + 7) / 8 * 8));
  p.chunks = (int)((n + p.chunk - 1) / p.chunk);
  // room for the chunks and tiles of this and every shorter list
  const long most = std::min<long>((n + 15) / 16, std::max<long>(8192 / blocks + 1, (n + 127) / 128));
  const auto up = [](size_t b) { return (b + 255) / 256 * 256; };
  const size_t list = up((size_t)n * 4);
  p.hist = 4 * list;
  p.start = p.hist + (n > kOne ? (size_t)kMaxTiles * kDigits * 4 : 0);
  p.part = p.start + up(((size_t)V + 1) * 4);
  p.total = std::max(p.part + up((size_t)most * 2 * H * sizeof(float)),
                     (size_t)std::min(parts, most_parts) * V * H * sizeof(float));
  return p;
}

}  // namespace

hipError_t launch_embed(int dtype, const EmbedArgs& a, hipStream_t s) {
  auto run = [&](auto dt) {
    typedef decltype(dt) DT;
    const int pieces = (a.H + Piece<DT>::V - 1) / Piece<DT>::V;
    auto go = [&](auto kernel, int L) {
      const long per = 256 / L, grid = std::min<long>((a.n + per - 1) / per, 8192);
      return launch("embed", kernel, dim3((unsigned)grid), dim3(256), 0, s, a);
    };
    // Measured: 200000 rows of 16 fp32 values with 4, 16 and 64 lanes a row 6, 11 and
    // 23 us, of 64 in 16 and 64 14 and 26; 100000 of 256 27 and 28; 81920 of 1024 bf16
    // ones 56 and 53.
    return pieces <= 4 ? go(k_embed<DT, 4>, 4) : pieces <= 64 ? go(k_embed<DT, 16>, 16) : go(k_embed<DT, 64>, 64);
  };
  return dtype == WM_FP32 ? run(0.0f) : run(bf16_t());
}

size_t embed_grad_workspace(long n, int V, int H) { return plan(n, V, H).total; }

hipError_t launch_embed_grad(int dtype, const EmbedGradArgs& a, hipStream_t s) {
  const Plan p = plan(a.n, a.V, a.H);
  char* ws = reinterpret_cast<char*>(a.ws);
  const int piece = dtype == WM_FP32 ? 4 : 8;
  const unsigned columns = (unsigned)(((a.H + piece - 1) / piece + 63) / 64);
  if (p.parts > 0) {
    const ScanArgs q{a, reinterpret_cast<float*>(ws)};
    const dim3 grid((unsigned)a.V * p.parts, columns);
    hipError_t e = dtype == WM_FP32 ? launch("embed_scan", k_embed_scan<float>, grid, dim3(kScan), 0, s, q, p.parts)
                                    : launch("embed_scan", k_embed_scan<bf16_t>, grid, dim3(kScan), 0, s, q, p.parts);
    if (e != hipSuccess || p.parts == 1) return e;
    const long size = (long)a.V * a.H;
    return launch("embed_parts", k_embed_parts, dim3((unsigned)((size + 255) / 256)), dim3(256), 0, s, q, p.parts);
  }
  if (p.few) {
    // 64 KB of the table a work-group, a flag for each row in LDS
    const int rows = std::min(kScan, std::max(1, 16384 / a.H));
    const dim3 grid((unsigned)(a.n + ((long)a.V + rows - 1) / rows), columns);
    return dtype == WM_FP32 ? launch("embed_few", k_embed_few<float>, grid, dim3(kScan), 0, s, a, rows)
                            : launch("embed_few", k_embed_few<bf16_t>, grid, dim3(kScan), 0, s, a, rows);
  }
  const size_t list = p.hist / 4;
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws), reinterpret_cast<uint32_t*>(ws + list)};
  uint32_t* pos[2] = {reinterpret_cast<uint32_t*>(ws + 2 * list), reinterpret_cast<uint32_t*>(ws + 3 * list)};
  int at = 0;
  hipError_t e = hipSuccess;
  if (a.n > 0 && p.tiles == 0) {
    e = launch("embed_sort", k_embed_sort, dim3(1), dim3(1024), 0, s, a.tokens, (int)a.n, a.V, p.passes, keys[0], pos[0]);
  } else {
    for (int k = 0; k < p.passes && a.n > 0 && e == hipSuccess; ++k) {
      const SortArgs q{a.tokens, keys[at], pos[at], keys[at ^ 1], pos[at ^ 1], reinterpret_cast<uint32_t*>(ws + p.hist),
                       (int)a.n, a.V, p.tile, p.tiles, k};
      e = launch("embed_hist", k_embed_hist, dim3(p.tiles), dim3(1024), 0, s, q);
      if (e == hipSuccess) e = launch("embed_scatter", k_embed_scatter, dim3(p.tiles), dim3(1024), 0, s, q);
      at ^= 1;
    }
  }
  if (e != hipSuccess) return e;
  const int groups = (p.chunks + 3) / 4, joins = (p.chunks + 15) / 16;
  const RowsArgs r{a, keys[at], pos[at], reinterpret_cast<float*>(ws + p.part), reinterpret_cast<int32_t*>(ws + p.start),
                   p.chunk, p.chunks, groups};
  const unsigned look = (unsigned)std::min<long>((long)a.V / 256 + 1, 4096);
  const dim3 grid(groups + look, columns);
  e = dtype == WM_FP32 ? launch("embed_rows", k_embed_rows<float>, grid, dim3(256), 0, s, r)
                       : launch("embed_rows", k_embed_rows<bf16_t>, grid, dim3(256), 0, s, r);
  if (e != hipSuccess) return e;
  const unsigned clear = (unsigned)std::min<long>(((long)a.V + kClear - 1) / kClear, 4096);
  return launch("embed_join", k_embed_join, dim3(joins + clear, ((a.H + 3) / 4 + 63) / 64), dim3(1024), 0, s, r, joins);
}

}  // namespace wm
