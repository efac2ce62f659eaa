// The matrix-core kernels of svf_chunk_attn: how their work is shared out, and how what was cut is joined.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>

#include "svf_chunk_device.h"

namespace svf {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short shortx4;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float floatx2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;

// Nothing but arithmetic is moved across this by the scheduler
#define SVF_IN_ORDER() __builtin_amdgcn_sched_barrier(0x6)

constexpr int kThreads = 512, kWaves = 8;
constexpr int kMostB = 4096;
constexpr int kXcds = 8;

__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const floatx2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// One item: R query rows (row r = query head r % G of new token r / G) of a (sequence, KV head) against the
// units of KEYS keys that they see.  Work is shared out by its cost: an item counts as many shares as it has units, and EXTRA in front of them for
// its beginning and end (reads in a chain, queries, a result), so that a range of many short items is no longer than one of a long one.
template <int R, int KEYS, int EXTRA>
struct Item {
  int row0, rows, first, last, unit0, units, shares;
  __device__ __forceinline__ Item(const ChunkParams& p, const ChunkSeq& s, int i) {
    const int M = s.n * p.G;
    row0 = i * R;
    rows = min(R, M - row0);
    const int j0 = row0 / p.G, j1 = (row0 + rows - 1) / p.G;
    first = p.window > 0 ? max(0, s.len + j0 + 1 - p.window) : 0;
    last = s.len + j1;
    unit0 = first / KEYS;
    units = last / KEYS + 1 - unit0;
    shares = units + EXTRA;
  }
};
template <int R>
__device__ __forceinline__ int items_of(const ChunkParams& p, const ChunkSeq& s) { return (s.n * p.G + R - 1) / R; }

// a value that all lanes hold, in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ ChunkSeq load_seq(const ChunkParams& p, int b) {
  return chunk_seq(p.seq_lens[b], p.new_rows[b], p.new_lens[b], p.max_seq_len, p.max_new, p.n_rows);
}

__device__ __forceinline__ int64_t shfl_up64(int64_t x, int d) {
  const int lo = __shfl_up((int)(x & 0xffffffff), d, 64), hi = __shfl_up((int)(x >> 32), d, 64);
  return ((int64_t)hi << 32) | (uint32_t)lo;
}
__device__ __forceinline__ int64_t lane64(int64_t x, int l) {
  const int lo = __builtin_amdgcn_readlane((int)(x & 0xffffffff), l), hi = __builtin_amdgcn_readlane((int)(x >> 32), l);
  return ((int64_t)hi << 32) | (uint32_t)lo;
}
__device__ __forceinline__ int64_t wave_scan64(int64_t x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t y = shfl_up64(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Shares of all items of one KV head of a sequence, by a wavefront.
template <int R, int KEYS, int EXTRA>
__device__ int64_t units_of_seq(const ChunkParams& p, const ChunkSeq& s, int lane) {
  const int n = items_of<R>(p, s);
  int64_t sum = 0;
  for (int i = lane; i < n; i += 64) sum += Item<R, KEYS, EXTRA>(p, s, i).shares;
  return lane64(wave_scan64(sum, lane), 63);
}

// How the work of a call is shared: all shares of all items in a row (sequence, KV head, item, share), cut into as many
// equal ranges as there are workgroups.
struct Cursor {
  int b, h, item;            // where a range begins
  int64_t skip;              // shares of that item in front of it
  int64_t total;
  ChunkSeq seq;              // sequence b
  int whole = 0;             // shares of the one item that the workgroup takes, where items aren't cut
};
// cum: [kMostB + 1] in LDS
template <int R, int KEYS, int EXTRA>
__device__ void units_before(const ChunkParams& p, int64_t* cum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = threadIdx.x; b < p.B; b += kThreads) {
    const ChunkSeq s = load_seq(p, b);
    const int n = items_of<R>(p, s);
    cum[b + 1] = n == 0 ? 0 : n == 1 ? Item<R, KEYS, EXTRA>(p, s, 0).shares : -1;
  }
  __syncthreads();
  for (int b = wave; b < p.B; b += kWaves) {
    if (cum[b + 1] >= 0) continue;
    const int64_t u = units_of_seq<R, KEYS, EXTRA>(p, load_seq(p, b), lane);
    if (lane == 0) cum[b + 1] = u;
  }
  __syncthreads();
  if (wave == 0) {
    int64_t run = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
      const int64_t x = wave_scan64(b0 + lane < p.B ? cum[b0 + lane + 1] * p.Hkv : 0, lane);
      if (b0 + lane < p.B) cum[b0 + lane + 1] = run + x;
      run += lane64(x, 63);
    }
    if (lane == 0) cum[0] = 0;
  }
  __syncthreads();
}
template <int R, int KEYS, int EXTRA>
__device__ Cursor cursor_at(const ChunkParams& p, const int64_t* cum, int64_t at) {
  const int lane = threadIdx.x & 63;
  Cursor c;
  int lo = 0, hi = p.B - 1;                              // the last sequence with cum[b] <= at that has units
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (cum[mid] <= at) lo = mid;
    else hi = mid - 1;
  }
  c.b = lo;
  const int64_t of_seq = (cum[lo + 1] - cum[lo]) / p.Hkv;
  int64_t rest = at - cum[lo];
  c.h = (int)(rest / of_seq);
  rest -= c.h * of_seq;
  const ChunkSeq s = load_seq(p, c.b);
  const int n = items_of<R>(p, s);
  c.item = 0;
  for (int i0 = 0;; i0 += 64) {
    const int64_t x = wave_scan64(i0 + lane < n ? Item<R, KEYS, EXTRA>(p, s, i0 + lane).shares : 0, lane);
    const uint64_t in = __ballot(rest < x);
    if (in) {
      const int l = __builtin_ctzll(in);
      c.item = i0 + l;
      if (l > 0) rest -= lane64(x, l - 1);
      break;
    }
    rest -= lane64(x, 63);
  }
  c.skip = rest;
  c.seq = s;
  return c;
}

// Scans over a wavefront's lanes by moves inside a row of sixteen and from row to row: no trips through LDS.
template <typename Join>
__device__ __forceinline__ int wave_scan(int x, Join&& join) {
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));     // row_shr:1, 2, 4, 8
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));    // row_bcast:15 -> rows 1, 3
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));    // row_bcast:31 -> rows 2, 3
  return x;
}

constexpr int kWorkgroups = 256;                         // one on each compute unit

// Sums of whole numbers of units.  T = R / G tokens of an item and KEYS are powers of two (shifts t and k).  Terms may pass 2^32 where the
// result doesn't (a million tokens in front, few tokens an item): everything is counted modulo 2^32.
// sum over x < n of (b + x T) / KEYS, rounded down
__device__ __forceinline__ uint32_t sum_of_units(uint32_t b, uint32_t n, int t, int k) {
  const auto pairs = [](uint32_t d) { return (d >> 1) * ((d - 1) | 1); };     // d (d - 1) / 2
  if (t >= k) return n * (b >> k) + (pairs(n) << (t - k));
  const int q = k - t;
  const uint32_t s = b >> t;                               // the same as of (s + x) / 2^q
  const auto upto = [&](uint32_t x) {
    const uint32_t d = x >> q;
    return (pairs(d) << q) + d * (x - (d << q));
  };
  return upto(s + n) - upto(s);
}
// Shares of the first i items of one KV head of a sequence.
template <int R, int KEYS, int EXTRA>
__device__ __forceinline__ int shares_upto(const ChunkParams& p, const ChunkSeq& s, int i) {
  constexpr int k = __builtin_ctz(KEYS);
  const int t = __builtin_ctz(R) - __builtin_ctz(p.G), T = 1 << t;
  const int items = items_of<R>(p, s), full = min(i, items - 1);         // (the last may have fewer rows)
  if (items == 0) return 0;
  uint32_t sum = full * (1 + EXTRA) + sum_of_units(s.len + T - 1, full, t, k);
  if (p.window > 0) {                                                    // less the units in front of the first tokens' windows
    const int c = s.len + 1 - p.window, x0 = c < 0 ? min(full, (-c + T - 1) >> t) : 0;
    sum -= sum_of_units(max(c + (x0 << t), 0), full - x0, t, k);
  }
  return (int)(i > full ? sum + Item<R, KEYS, EXTRA>(p, s, items - 1).shares : sum);
}

// The same without LDS and barriers, by every wavefront for itself, for up to 64 sequences (lane b has sequence b) and groups of a power of two
// of query heads, whose items' units have a sum in closed form (64 single tokens over 1000 57 us, 65 by the other way 61; one token over 8000 for groups of
// eight query heads 17.5 us, of seven 18.8; 2048 over 30k 1.16 and 1.10 PFLOP/s).  `begin` says where the range begins, given the total.  JOIN: shares that the end of an
// item costs if it was cut; where no more workgroups than there are have an item each, and the largest is within that of an equal range, they aren't
// cut (JOIN = 0: always); `take` says which, given how many there are.
template <int R, int KEYS, int EXTRA, int JOIN, typename Begin, typename Take>
__device__ bool cursor_of_few(const ChunkParams& p, Begin&& begin, Take&& take, Cursor& c) {
  if (p.B > 64 || p.share_bound >= (1 << 30) || (p.G & (p.G - 1)) != 0 || p.G > R) return false;
  const int lane = threadIdx.x & 63;
  const ChunkSeq s = load_seq(p, min(lane, p.B - 1));
  const int n = lane < p.B ? items_of<R>(p, s) : 0, of_seq = n > 0 ? shares_upto<R, KEYS, EXTRA>(p, s, n) : 0;
  const auto add = [](int x, int y) { return x + y; };
  const auto seq_at = [&](int b) {
    return ChunkSeq{__builtin_amdgcn_readlane(s.len, b), __builtin_amdgcn_readlane(s.row, b), __builtin_amdgcn_readlane(s.n, b)};
  };
  const int upto = wave_scan(of_seq * p.Hkv, add);
  c.total = __builtin_amdgcn_readlane(upto, 63);
  if constexpr (JOIN > 0) {
    int most = 0;
    if (n > 0) most = Item<R, KEYS, EXTRA>(p, s, n - 1).shares;          // (an item in front of the last has more where the last has fewer rows)
    if (n > 1) most = max(most, (int)Item<R, KEYS, EXTRA>(p, s, n - 2).shares);
    const int items_upto = wave_scan(n * p.Hkv, add), items = __builtin_amdgcn_readlane(items_upto, 63);
    most = __builtin_amdgcn_readlane(wave_scan(most, [](int x, int y) { return max(x, y); }), 63);       // (none is negative)
    if (items <= kWorkgroups && (int64_t)most * kWorkgroups <= c.total + JOIN * kWorkgroups) {
      const int mine = take(items);
      if (mine >= items) return true;
      c.b = __builtin_ctzll(__ballot(items_upto > mine));
      const int of_head = __builtin_amdgcn_readlane(n, c.b), rest = mine - (__builtin_amdgcn_readlane(items_upto, c.b) - of_head * p.Hkv);
      c.h = (int)((uint32_t)rest / (uint32_t)of_head);
      c.item = rest - c.h * of_head;
      c.skip = 0;
      c.seq = seq_at(c.b);
      c.whole = (int)Item<R, KEYS, EXTRA>(p, c.seq, c.item).shares;
      return true;
    }
  }
  const int64_t at = begin(c.total);
  if (at >= c.total) return true;                          // (nothing for this workgroup)
  c.b = __builtin_ctzll(__ballot((int64_t)upto > at));
  const int per_head = __builtin_amdgcn_readlane(of_seq, c.b);
  int rest = (int)at - (__builtin_amdgcn_readlane(upto, c.b) - per_head * p.Hkv);
  c.h = (int)((uint32_t)rest / (uint32_t)per_head);
  rest -= c.h * per_head;
  const ChunkSeq t = c.seq = seq_at(c.b);
  int lo = 0, hi = __builtin_amdgcn_readlane(n, c.b) - 1;  // the last item with no more than `rest` shares in front of it
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (shares_upto<R, KEYS, EXTRA>(p, t, mid) <= rest) lo = mid;
    else hi = mid - 1;
  }
  c.item = lo;
  c.skip = rest - shares_upto<R, KEYS, EXTRA>(p, t, lo);
  return true;
}

// Loads and stores of what workgroups on different XCDs exchange: at the scope of the device, past the L2s.
__device__ __forceinline__ void store_shared(float* p, floatx4 x) {
  const u32x4 w = __builtin_bit_cast(u32x4, x);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)w[1] << 32 | w[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p) + 1, (uint64_t)w[3] << 32 | w[2], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_shared(float2* p, float2 x) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)__float_as_uint(x.y) << 32 | __float_as_uint(x.x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t load_shared64(const void* p) {
  return __hip_atomic_load(static_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ floatx4 load_shared(const float* p) {
  const uint64_t a = load_shared64(p), b = load_shared64(p + 2);
  const u32x4 w = {(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
  return __builtin_bit_cast(floatx4, w);
}
__device__ __forceinline__ float2 load_shared(const float2* p) {
  const uint64_t a = load_shared64(p);
  return make_float2(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32)));
}

// Workgroup v of n takes shares [range_begin(v), range_begin(v + 1)); n is kWorkgroups, or the number of shares if that is less.
__device__ __forceinline__ int64_t range_begin(int64_t total, int n, int v) {
  return n == kWorkgroups ? (total * v) / kWorkgroups : (int64_t)v;
}
__device__ __forceinline__ int owner_of(int64_t total, int n, int64_t unit) {
  if (n != kWorkgroups) return (int)unit;
  // the largest v with total v / n <= unit, rounded down
  if (total < (1 << 22)) return (int)((uint32_t)((unit + 1) * kWorkgroups - 1) / (uint32_t)total);
  return (int)(((unit + 1) * kWorkgroups - 1) / total);
}

// The part of an item that shares [skip, skip + left) of it are: units [begin, end); it begins or ends the item, or is all of it.  `from`, `upto`: the
// workgroups that have the item's first and last unit.
struct Part {
  int taken, begin, end;
  bool begins, ends;
  template <int R, int KEYS, int EXTRA>
  __device__ __forceinline__ Part(const Item<R, KEYS, EXTRA>& it, int skip, int left) {
    taken = min(it.shares - skip, left);
    begin = max(skip - EXTRA, 0);
    end = max(skip + taken - EXTRA, 0);
    begins = begin == 0;
    ends = end == it.units;
  }
};

// The workspace: for every workgroup two partial results of R rows (0: of the item its range begins inside of, 1: of the one
// its range ends inside of) and what the second launch joins.
template <int D, int R>
struct Parts {
  float* o;                  // [N][2][R][D], relative to the maximum
  float2* ml;                // [N][2][R] maximum (log2 units), denominator
  int4* join;                // [N] of the item that begins in a range and ends behind it: b, KV head, item, last workgroup; b < 0: none
  uint32_t* arrived;         // [N] the same, where the last of an item's workgroups joins its parts: how many are there; zero between calls
  __host__ __device__ Parts(char* ws, int n) {
    arrived = reinterpret_cast<uint32_t*>(ws);
    static_assert(kWorkgroups * sizeof(uint32_t) <= kChunkCounters, "");
    ws += kChunkCounters;
    o = reinterpret_cast<float*>(ws);
    ml = reinterpret_cast<float2*>(ws + (size_t)n * 2 * R * D * sizeof(float));
    join = reinterpret_cast<int4*>(ws + (size_t)n * 2 * R * (D * sizeof(float) + sizeof(float2)));
  }
  static size_t bytes(int n) { return kChunkCounters + (size_t)n * (2 * R * (D * sizeof(float) + sizeof(float2)) + sizeof(int4)); }
};

// Joins the parts of the items that were cut: workgroup (v, y) rows 32 y .. 32 y + 31 of the item that begins in range v.  A thread adds up four
// channels of a row; where rows are few, several threads take the parts in turn.
template <int D, int R, int KEYS, int EXTRA>
__global__ __launch_bounds__(kThreads) void chunk_merge_kernel(ChunkParams p) {
  __shared__ floatx4 others[kThreads];
  __shared__ float2 others_ml[kThreads];
  const int N = gridDim.x, me = blockIdx.x, tid = threadIdx.x;
  const Parts<D, R> parts(p.ws, N);
  const int4 join = parts.join[me];
  if (join.x < 0) return;
  const ChunkSeq s = load_seq(p, join.x);
  const Item<R, KEYS, EXTRA> it(p, s, join.z);
  const int r0 = 32 * blockIdx.y, rows = min(32, it.rows - r0);
  if (rows <= 0) return;
  const int cells = rows * (D / 4);
  // threads of a cell; consecutive threads have consecutive cells, so that what a wavefront asks for at once lies side by side
  const int takers = cells < kThreads ? min(kThreads / cells, 16) : 1, step = takers > 1 ? cells : kThreads;
  const int n = join.w - me + 1;
  for (int c0 = 0; c0 < cells; c0 += step) {
    const int first = tid / step, cell = first < takers ? c0 + tid - first * step : cells;
    const bool live = cell < cells;
    const int r = r0 + (live ? cell : 0) / (D / 4), ch = 4 * (cell % (D / 4));
    float top = -INFINITY, den = 0.f;
    floatx4 x = {};
    for (int i0 = first; i0 < n; i0 += 4 * takers) {
      float2 ml[4];
      floatx4 y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = min(i0 + k * takers, n - 1);
        const int64_t at = (int64_t)(2 * (me + i) + (i == 0 ? 1 : 0)) * R + r;
        ml[k] = parts.ml[at];
        y[k] = *reinterpret_cast<const floatx4*>(parts.o + at * D + ch);
      }
      float now = top;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i0 + k * takers >= n) ml[k].x = -INFINITY;
        now = fmaxf(now, ml[k].x);
      }
      const float use = now == -INFINITY ? 0.f : now, f0 = __builtin_amdgcn_exp2f(top - use);
      den *= f0;
      x *= f0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float f = __builtin_amdgcn_exp2f(ml[k].x - use);
        if (i0 + k * takers < n) {
          den += f * ml[k].y;
          x += f * y[k];
        }
      }
      top = now;
    }
    if (takers > 1) {
      __syncthreads();
      others[tid] = x;
      others_ml[tid] = make_float2(top, den);
      __syncthreads();
      if (first == 0) {
        for (int k = 1; k < takers; ++k) top = fmaxf(top, others_ml[tid + k * step].x);
        den = 0.f;
        x = floatx4{};
        for (int k = 0; k < takers; ++k) {
          const float2 ml = others_ml[tid + k * step];
          const float f = __builtin_amdgcn_exp2f(ml.x - top);
          den += f * ml.y;
          x += f * others[tid + k * step];
        }
      }
    }
    if (!live || first != 0) continue;
    const int row = it.row0 + r, j = row / p.G, head = join.y * p.G + row - j * p.G;
    const float inv = 1.0f / den;
    const u32x2 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
    *reinterpret_cast<u32x2*>(static_cast<char*>(p.out) + 2 * ((int64_t)(s.row + j) * p.out_stride + (int64_t)head * D + ch)) = w;
    if (ch == 0 && p.lse) p.lse[(int64_t)(s.row + j) * p.Hq + head] = (top + log2f(den)) * 0.69314718055994530942f;
  }
}

}  // namespace

}  // namespace svf
