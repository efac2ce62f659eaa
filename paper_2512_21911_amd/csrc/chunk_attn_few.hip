// Attention of new tokens over the cache (svf_chunk_attn), 32 query rows of a (sequence, KV head) at a time: bf16 with up to 32 of them, as for
// single tokens, and everything in fp32.
//   S = scale Q K^T, a running maximum m and sum l of each row:  O <- O 2^(m - m') + 2^(S - m') V,  l likewise,  out = O / l.
//
// The eight wavefronts of a workgroup have nothing to do with one another until the end of an item: each takes every eighth unit of 32 keys, the
// next unit's loads on their way while one is worked on, and keeps its own maximum, sum and output.  Then the eight are joined through LDS, and where an
// item was cut, the last of its workgroups joins the parts.
//   bf16  bound by memory, the cache goes by once, 128 KB in flight on a compute unit at d = 128: 537 MB for four tokens over 32k in 111 us,
//         4.8 TB/s (one token over 8k, 34 MB: 17 us, of which launch, first tiles and join are 10).  The matrix cores still do both products (32 rows
//         at a time, whatever of them is used), and have the time for weights of sixteen bits (two bf16 terms): what is left of a weight behind
//         its first term is rounded to bf16 too, 2^-16 of the weight.
//   fp32  bound by the fp32 matrix instructions (v_mfma_f32_32x32x2_f32: 64 cycles per 4096 operations, 157 TFLOP/s over the chip; 32 keys in
//         0.58 us at d = 64, 1.1 at d = 128, 0.43 and 0.85 at that rate).  S^T = K Q^T leaves a query row in lane mod 32 with sixteen of
//         the unit's keys per lane, which is the operand that O^T += V^T P^T takes, one register per step: the weights never leave their lanes.
//         K goes from memory into operand registers, V straight into LDS once the unit before has been read there (through registers there were
//         too few of them: 1024 tokens, 8 heads, d = 128 109 us instead of 54), the queries, the same for all wavefronts, wait in LDS.
#include "chunk_share.h"

namespace svf {

namespace {

constexpr int kFewRows = 32;
constexpr int kFewKeys = 32;                             // keys of a unit

// What a lane looks a unit's tokens up for: where its rows' chunks are.
template <int N> struct Places { uint32_t page[N], slot[N]; };
template <int N, int EXTRA>
__device__ __forceinline__ void look_up_places(const ChunkParams& p, const int32_t* table, int b, const Item<kFewRows, kFewKeys, EXTRA>& it, int key0,
                                               int t_lane, int step, Places<N>& to) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // (places outside what the item's rows see are read as the nearest one inside)
    const uint32_t t = (uint32_t)min(max(key0 + t_lane + i * step, it.first), it.last);
    const uint32_t np = p.page.of(t);
    to.slot[i] = t - np * (uint32_t)p.kv.page_size;
    to.page[i] = p.kv.page_size == 0 ? (uint32_t)b : (uint32_t)table[np];
  }
}
__device__ __forceinline__ uint32_t inside(const ChunkParams& p, uint32_t page) { return page < (uint32_t)p.n_pages ? page : 0; }

// The scores of a unit into exponents' base and weights: x[i] becomes the weight of key 8 (i / 4) + 4 (lane / 32) + i mod 4.  m, l: maximum (log2
// units) and sum so far; o follows the maximum.
template <int D>
__device__ __forceinline__ void few_weights(floatx16& x, float scale_log2, bool masked, int most, int least, float& m, float& l,
                                            floatx16 (&o)[D / 32]) {
  if (masked) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i / 4) + i % 4;
      if (key > most || key < least) x[i] = -INFINITY;
    }
  }
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
  top = halves_max(top) * scale_log2;
  if (__ballot(top > m)) {
    const float now = fmaxf(m, top), f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
    m = now;
    l *= f;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb) o[cb] *= f;
  }
  const float use = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale_log2, -use));
    l += x[i];
  }
}

// bf16: a wavefront's part of LDS holds a unit's K, then its V.
template <int D>
struct FewBf16 {
  typedef __bf16 Element;
  static constexpr int kRowBytes = 2 * D, kChunks = D / 8, kTileBytes = kFewKeys * kRowBytes;
  static constexpr int kOwn = 2 * kTileBytes;
  static constexpr int kLanesRows = 64 / kChunks, kPasses = kFewKeys / kLanesRows;      // rows that a wavefront loads at once
  static constexpr int kQueries = 16;                    // (bytes of LDS for the queries: none)
  // What cutting costs.  Cut and not, us, by the shares that the largest item has above the mean (32 and 31 tokens, 8 KV heads over 3300 .. 4700):
  // d = 128 4: 107, 103; 15: 107, 106; 19: 106, 102; 22: 109, 110; 26: 106, 104; d = 64 4: 58, 54; 15: 57, 55; 19: 56, 52; 22: 56, 57; 26: 55, 53.
  static constexpr int kJoin = 20;
  static constexpr int kExtra = 4;                       // an item's beginning and end, 3 us, in units of 0.8 us
  // (where a chunk of a row sits: as in the kernel for many rows)
  static __device__ __forceinline__ uint32_t k_at(int t, int c) {
    return t * kRowBytes + ((c ^ (D == 128 ? t & 15 : (t >> 1) & 7)) << 4);
  }
  static __device__ __forceinline__ uint32_t v_at(int t, int c) {
    return t * kRowBytes + ((c ^ (D == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1))) << 4);
  }
  bf16x8 q[D / 16];
  u32x4 k[kPasses], v[kPasses];
  Places<kPasses> at;

  __device__ __forceinline__ void queries(const char* row, char*, int lane) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) q[ks] = *reinterpret_cast<const bf16x8*>(row + 32 * ks + 16 * (lane >> 5));
  }
  template <int EXTRA>
  __device__ __forceinline__ void look_up(const ChunkParams& p, const int32_t* table, int b, const Item<kFewRows, kFewKeys, EXTRA>& it, int key0,
                                          int lane) {
    look_up_places(p, table, b, it, key0, lane / kChunks, kLanesRows, at);
  }
  __device__ __forceinline__ void request(const ChunkParams& p, const char* K, const char* V, int lane) {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const uint64_t off = 16 * ((uint64_t)at.slot[i] * p.tok16 + (uint64_t)inside(p, at.page[i]) * p.page16 + lane % kChunks);
      k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(K + off));
      v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(V + off));
    }
  }
  __device__ __forceinline__ void send(const char*, char*, int) {}
  // `next`: puts the next unit on its way, once this one's registers are free
  template <typename Next>
  __device__ __forceinline__ void work(char* own, const char*, int lane, float scale_log2, bool masked, int most, int least, float& m, float& l,
                                       floatx16 (&o)[D / 32], Next&& next) {
    const int r32 = lane & 31, hh = lane >> 5;
    char* const vs = own + kTileBytes;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int t = lane / kChunks + i * kLanesRows;
      *reinterpret_cast<u32x4*>(own + k_at(t, lane % kChunks)) = k[i];
      *reinterpret_cast<u32x4*>(vs + v_at(t, lane % kChunks)) = v[i];
    }
    next();
    floatx16 x = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(own + k_at(r32, 2 * ks + hh)), q[ks], x, 0, 0, 0);
    few_weights<D>(x, scale_log2, masked, most, least, m, l, o);
    bf16x8 high[2], low[2];
#pragma unroll
    for (int b8 = 0; b8 < 2; ++b8) {
      u32x4 wh, wl;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = x[8 * b8 + 2 * i], b = x[8 * b8 + 2 * i + 1];
        wh[i] = pack_bf16(a, b);
        wl[i] = pack_bf16(a - __uint_as_float(wh[i] << 16), b - __uint_as_float(wh[i] & 0xffff0000u));
      }
      high[b8] = __builtin_bit_cast(bf16x8, wh);
      low[b8] = __builtin_bit_cast(bf16x8, wl);
    }
    const int vt = 4 * hh + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vb = 8 * (lane & 1);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) {
        shortx4 y[2];
#pragma unroll
        for (int z = 0; z < 2; ++z)
          y[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) shortx4*)(vs + v_at(16 * kb + 8 * z + vt, 4 * cb + vc) + vb));
        const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(y[0], y[1], 0, 1, 2, 3, 4, 5, 6, 7));
        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, high[kb], o[cb], 0, 0, 0);
        o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, low[kb], o[cb], 0, 0, 0);
      }
  }
  static __device__ __forceinline__ void write(char* to, floatx4 y) {
    *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
  }
};

// fp32: a wavefront's part of LDS holds a unit's V, channel c of key t at c ^ 32 (t / 4 mod 2), since the halves of the wavefront read keys four
// apart (a load to LDS writes lane after lane: the lanes' sources are exchanged instead).  A lane's K is half of the 16-byte chunks of one key.
template <int D>
struct FewF32 {
  typedef float Element;
  static constexpr int kRowBytes = 4 * D, kChunks = D / 4;
  static constexpr int kOwn = kFewKeys * kRowBytes;
  static constexpr int kLanesRows = 64 / kChunks, kPasses = kFewKeys / kLanesRows;
  static constexpr int kQueries = kFewRows * kRowBytes;
  // What cutting costs.  Cut and not, us (8 x 128 tokens over 100 .. 1300, and one prompt of 800 and 900 over 1000): d = 128 5: 73, 55; 15: 76, 64;
  // 20: 91, 87; 21: 77, 73; 24: 81, 85; d = 64 5: 34, 27; 15: 34, 31; 20: 44, 42; 21: 34, 35; 24: 39, 42.
  static constexpr int kJoin = 22;
  static constexpr int kExtra = 8;                       // ... in units of 0.6 us (d = 64) and 1.1 us
  floatx4 k[D / 8];
  Places<1> at;                                          // (of key lane mod 32)
  int64_t off;                                           // of that key's row of the unit that was requested last

  // chunk c of row r at c ^ (r mod 16): sixteen lanes read the same chunk of sixteen rows
  static __device__ __forceinline__ int q_at(int r, int c) { return r * kRowBytes + 16 * (c ^ (r & 15)); }
  __device__ __forceinline__ void queries(const char* row, char* shared, int lane) {
    if (threadIdx.x >= 64) return;                       // (one wavefront for all)
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
      const int at_c = 2 * c + (lane >> 5);
      *reinterpret_cast<floatx4*>(shared + q_at(lane & 31, at_c)) = *reinterpret_cast<const floatx4*>(row + 16 * at_c);
    }
  }
  template <int EXTRA>
  __device__ __forceinline__ void look_up(const ChunkParams& p, const int32_t* table, int b, const Item<kFewRows, kFewKeys, EXTRA>& it, int key0,
                                          int lane) {
    look_up_places(p, table, b, it, key0, lane & 31, 0, at);
  }
  __device__ __forceinline__ void request(const ChunkParams& p, const char* K, const char* V, int lane) {
    off = 4 * ((int64_t)at.slot[0] * p.kv.stride_tok + (int64_t)inside(p, at.page[0]) * p.kv.stride_page);
#pragma unroll
    for (int c = 0; c < D / 8; ++c) k[c] = *reinterpret_cast<const floatx4*>(K + off + 16 * (2 * c + (lane >> 5)));
  }
  // the values of the unit that was requested, straight into LDS, where those of the unit before have been read
  __device__ __forceinline__ void send(const char* V, char* own, int lane) {
    const int t_lane = lane / kChunks, c = lane % kChunks;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int t = t_lane + i * kLanesRows;
      const int64_t row = __shfl((long long)off, t, 64);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(V + row + 16 * (c ^ (8 * ((t >> 2) & 1)))),
                                       (__attribute__((address_space(3))) uint32_t*)(own + i * 1024), 16, 0, 0);
    }
  }
  template <typename Next>
  __device__ __forceinline__ void work(char* own, const char* shared, int lane, float scale_log2, bool masked, int most, int least, float& m,
                                       float& l, floatx16 (&o)[D / 32], Next&& next) {
    const int r32 = lane & 31, hh = lane >> 5;
    float* const vs = reinterpret_cast<float*>(own);
    floatx16 s[2] = {};                                  // (two chains)
    // (operands are read out of LDS a group of products ahead, and not all at once, for which there are no registers)
    floatx4 q[2][2];
    const auto q_read = [&](int g) {
#pragma unroll
      for (int c = 0; c < 2; ++c) q[g & 1][c] = *reinterpret_cast<const floatx4*>(shared + q_at(r32, 2 * (2 * g + c) + hh));
    };
    q_read(0);
#pragma unroll
    for (int g = 0; g < D / 16; ++g) {
      if (g + 1 < D / 16) q_read(g + 1);
      SVF_IN_ORDER();
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[2 * g + c][e], q[g & 1][c][e], s[e & 1], 0, 0, 0);
      SVF_IN_ORDER();
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): the unit's values are in LDS
    floatx16 x = s[0] + s[1];
    SVF_IN_ORDER();
    next();
    few_weights<D>(x, scale_log2, masked, most, least, m, l, o);
    float w[2][2][D / 32];
    const auto v_read = [&](int g) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
          w[g & 1][i][n] = vs[(8 * ((2 * g + i) / 4) + 4 * hh + (2 * g + i) % 4) * D + ((32 * n + r32) ^ (32 * hh))];
    };
    v_read(0);
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      if (g + 1 < 8) v_read(g + 1);
      SVF_IN_ORDER();
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < D / 32; ++n) o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[g & 1][i][n], x[2 * g + i], o[n], 0, 0, 0);
      SVF_IN_ORDER();
    }
  }
  static __device__ __forceinline__ void write(char* to, floatx4 y) { *reinterpret_cast<floatx4*>(to) = y; }
};

template <int D, typename Unit>
__global__ __launch_bounds__(kThreads, 2) void chunk_attn_few_kernel(ChunkParams p) {
  constexpr int R = kFewRows, E = sizeof(typename Unit::Element), kOwn = Unit::kOwn, kExtra = Unit::kExtra;
  // the wavefronts' parts; at the end of an item each holds its wavefront's output, as many bytes
  static_assert(kOwn == kFewRows * D * 4 && (kMostB + 1) * 8 <= kWaves * kOwn, "");
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kOwn];
  __shared__ __attribute__((aligned(16))) char shared_q[Unit::kQueries];
  __shared__ float2 joint[kWaves][kFewRows];
  __shared__ bool joins;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), hh = lane >> 5, r32 = lane & 31;
  const Parts<D, R> parts(p.ws, gridDim.x);
  // where this workgroup's range begins
  int64_t total = 0, at = 0, end = 0;
  int N = 0, me = 0;
  const auto take = [&](int n) {
    N = n;
    // Consecutive ranges, which read the same keys, go to one XCD and its L2: workgroups are dealt to the eight in turn
    return me = N == kWorkgroups ? (int)(blockIdx.x % kXcds * (kWorkgroups / kXcds) + blockIdx.x / kXcds) : (int)blockIdx.x;
  };
  const auto begin = [&](int64_t all) {
    total = all;
    take((int)min((int64_t)kWorkgroups, total));           // workgroups with work: one unit at least
    at = me < N ? range_begin(total, N, me) : total;
    end = me < N ? range_begin(total, N, me + 1) : total;
    return at;
  };
  Cursor c;
  if (!cursor_of_few<R, kFewKeys, kExtra, Unit::kJoin>(p, begin, take, c)) {
    int64_t* const cum = reinterpret_cast<int64_t*>(lds);
    units_before<R, kFewKeys, kExtra>(p, cum);
    begin(cum[p.B]);
    if (me < N) c = cursor_at<R, kFewKeys, kExtra>(p, cum, at);
    __syncthreads();
  }
  if (me >= N) return;
  c.b = uniform(c.b);
  c.h = uniform(c.h);
  c.item = uniform(c.item);
  int skip = uniform((int)c.skip), left = uniform(c.whole > 0 ? c.whole : (int)(end - at));

  char* const mine = lds + wave * kOwn;
  while (skip + left > kExtra) {                             // (else the range ends in front of an item's units)
    const ChunkSeq s{uniform(c.seq.len), uniform(c.seq.row), uniform(c.seq.n)};
    const Item<R, kFewKeys, kExtra> it(p, s, c.item);
    const Part part(it, skip, left);
    const int n = part.end - part.begin, unit0 = it.unit0 + part.begin;
    const int64_t first_unit = end - left - skip + kExtra;   // (counted in shares) of the item
    const char* const K = static_cast<const char*>(p.K) + E * (int64_t)c.h * p.kv.stride_head;
    const char* const V = static_cast<const char*>(p.V) + E * (int64_t)c.h * p.kv.stride_head;
    const int32_t* const table = p.table + (int64_t)c.b * p.kv.max_pages;
    Unit unit;
    const auto look_up = [&](int u) { unit.look_up(p, table, c.b, it, (unit0 + u) * kFewKeys, lane); };
    if (wave < n) {
      look_up(wave);
      unit.request(p, K, V, lane);
      unit.send(V, mine, lane);
      if (wave + kWaves < n) look_up(wave + kWaves);
    }
    // this lane's row
    const int row = it.row0 + min(r32, it.rows - 1), row_j = row / p.G;
    const int hi = s.len + row_j, lo = p.window > 0 ? hi + 1 - p.window : 0;
    unit.queries(static_cast<const char*>(p.q) +
                     E * ((int64_t)(s.row + row_j) * p.q_stride + (int64_t)(c.h * p.G + row - row_j * p.G) * D), shared_q, lane);
    if (E == 4) __syncthreads();
    floatx16 o[D / 32] = {};
    float m = -INFINITY, l = 0.f;
    const int hi_all = s.len + it.row0 / p.G, lo_all = p.window > 0 ? it.last + 1 - p.window : 0;
    for (int u = wave; u < n; u += kWaves) {
      const int key0 = (unit0 + u) * kFewKeys;
      unit.work(mine, shared_q, lane, p.scale_log2, key0 + kFewKeys - 1 > hi_all || key0 < lo_all, hi - key0 - 4 * hh, lo - key0 - 4 * hh, m, l,
                o, [&]() {
                  if (u + kWaves < n) {
                    unit.request(p, K, V, lane);
                    if (u + 2 * kWaves < n) look_up(u + 2 * kWaves);
                  }
                });
      if (u + kWaves < n) unit.send(V, mine, lane);
    }

    // the wavefronts' results joined: each leaves its own in its part of LDS
    l = halves_sum(l);
    if (r32 < it.rows) {
      float* to = reinterpret_cast<float*>(mine) + r32 * D + 4 * hh;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const floatx4 y = {o[cb][4 * g], o[cb][4 * g + 1], o[cb][4 * g + 2], o[cb][4 * g + 3]};
          *reinterpret_cast<floatx4*>(to + 32 * cb + 8 * g) = y;
        }
      if (hh == 0) joint[wave][r32] = make_float2(m, l);
    }
    __syncthreads();
    const bool whole = part.begins && part.ends;
    const int from = whole ? me : owner_of(total, N, first_unit), upto = whole ? me : owner_of(total, N, first_unit + it.units - 1);
    const auto write = [&](int r, int ch, float top, float den, floatx4 y) {
      const float inv = 1.0f / den;
      const int at_row = it.row0 + r, j = at_row / p.G, head = c.h * p.G + at_row - j * p.G;
      Unit::write(static_cast<char*>(p.out) + E * ((int64_t)(s.row + j) * p.out_stride + (int64_t)head * D + ch), y * inv);
      if (ch == 0 && p.lse) p.lse[(int64_t)(s.row + j) * p.Hq + head] = (top + log2f(den)) * 0.69314718055994530942f;
    };
    const int cells = it.rows * (D / 4);
    for (int i = tid; i < cells; i += kThreads) {
      const int r = i / (D / 4), ch = 4 * (i % (D / 4));
      float top = joint[0][r].x;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, joint[w][r].x);
      const float use = top == -INFINITY ? 0.f : top;
      float den = 0.f;
      floatx4 y = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 ml = joint[w][r];
        const float f = __builtin_amdgcn_exp2f(ml.x - use);
        den += f * ml.y;
        y += f * *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(lds + w * kOwn) + r * D + ch);
      }
      if (whole) {
        write(r, ch, top, den, y);
      } else {
        const int64_t at_part = (int64_t)(2 * me + (me == from ? 1 : 0)) * R + r;
        store_shared(parts.o + at_part * D + ch, y);
        if (ch == 0) store_shared(&parts.ml[at_part], make_float2(top, den));
      }
    }
    if (!whole) {
      // The workgroup that comes last joins the parts, in their order: the sum does not depend on which one it is
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0): this thread's stores are where the others read
      __syncthreads();
      if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(&parts.arrived[from], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        joins = before == (uint32_t)(upto - from);
        if (joins) __hip_atomic_store(&parts.arrived[from], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      if (joins) {
        constexpr int kTogether = 12;                       // a trip to memory, some 2 us from another XCD, for as many parts at once
        // (consecutive threads have consecutive cells: what a wavefront asks for at once lies side by side)
        const int takers = cells < kThreads ? min(kThreads / cells, 16) : 1, step = takers > 1 ? cells : kThreads;
        floatx4* const others = reinterpret_cast<floatx4*>(lds);
        float2* const others_ml = reinterpret_cast<float2*>(lds + kThreads * sizeof(floatx4));
        const int parts_n = upto - from + 1;
        for (int c0 = 0; c0 < cells; c0 += step) {
          const int first = tid / step, cell = first < takers ? c0 + tid - first * step : cells;
          const int r = (cell < cells ? cell : 0) / (D / 4), ch = 4 * (cell % (D / 4));
          float top = -INFINITY, den = 0.f;
          floatx4 y = {};
          for (int i0 = first; i0 < parts_n; i0 += kTogether * takers) {
            float2 ml[kTogether];
            floatx4 z[kTogether];
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
              const int i = min(i0 + k * takers, parts_n - 1);
              const int64_t at_part = (int64_t)(2 * (from + i) + (i == 0 ? 1 : 0)) * R + r;
              ml[k] = load_shared(&parts.ml[at_part]);
              z[k] = load_shared(parts.o + at_part * D + ch);
            }
            float now = top;
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
              if (i0 + k * takers >= parts_n) ml[k].x = -INFINITY;
              now = fmaxf(now, ml[k].x);
            }
            const float use = now == -INFINITY ? 0.f : now, f0 = __builtin_amdgcn_exp2f(top - use);
            den *= f0;
            y *= f0;
#pragma unroll
            for (int k = 0; k < kTogether; ++k)
              if (i0 + k * takers < parts_n) {
                const float f = __builtin_amdgcn_exp2f(ml[k].x - use);
                den += f * ml[k].y;
                y += f * z[k];
              }
            top = now;
          }
          if (takers > 1) {
            others[tid] = y;
            others_ml[tid] = make_float2(top, den);
            __syncthreads();
            if (first == 0) {
              for (int k = 1; k < takers; ++k) top = fmaxf(top, others_ml[tid + k * step].x);
              den = 0.f;
              y = floatx4{};
              for (int k = 0; k < takers; ++k) {
                const float2 ml = others_ml[tid + k * step];
                const float f = __builtin_amdgcn_exp2f(ml.x - top);
                den += f * ml.y;
                y += f * others[tid + k * step];
              }
            }
            __syncthreads();
          }
          if (cell < cells && first == 0) write(r, ch, top, den, y);
        }
      }
    }
    __syncthreads();

    // the next item
    left -= part.taken;
    skip = 0;
    if (++c.item == items_of<R>(p, s)) {
      c.item = 0;
      if (++c.h == p.Hkv) {
        c.h = 0;
        if (left > 0) {
          do c.seq = load_seq(p, ++c.b); while (c.seq.n == 0);             // (there is one with shares: some are left)
        }
      }
    }
  }
}

}  // namespace

bool chunk_attn_is_few(int G, int max_new) { return (int64_t)G * max_new <= kFewRows; }

size_t chunk_attn_few_workspace(int d) {
  return d == 128 ? Parts<128, kFewRows>::bytes(kWorkgroups) : Parts<64, kFewRows>::bytes(kWorkgroups);
}

hipError_t launch_chunk_attn_few(const ChunkParams& p, bool f32, hipStream_t st) {
  const dim3 grid(kWorkgroups), block(kThreads);
  if (p.d == 128) {
    if (f32) hipLaunchKernelGGL((chunk_attn_few_kernel<128, FewF32<128>>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((chunk_attn_few_kernel<128, FewBf16<128>>), grid, block, 0, st, p);
  } else {
    if (f32) hipLaunchKernelGGL((chunk_attn_few_kernel<64, FewF32<64>>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((chunk_attn_few_kernel<64, FewBf16<64>>), grid, block, 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace svf
