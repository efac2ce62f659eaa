// Attention of new tokens over the cache in bf16 (svf_chunk_attn), many query rows of a (sequence, KV head) at a time.
//   S = scale Q K^T, weights 2^(S - m) relative to a running m of each row, l their sum:  out = sum 2^(S - m) V / l.
//
// An item is 256 query rows (32 for each of eight wavefronts, in the order token, head of the group, so that all heads of a group share
// the keys in LDS); its keys go by in units of 64, the next three of them in LDS or on their way there.  S^T = K Q^T and O^T = V^T P^T leave a query row in
// lane mod 32: row statistics are a lane's own but for one exchange of halves, and the weights, rounded to bf16, are the second
// product's operand where they are.  The rounding is the size of the output's own, 2^-8 of a weight at most, and l is summed from the unrounded ones.
//
// 2048 tokens over 32k, 32 heads, d = 128: 921 to 977 us, 1.09 to 1.15 PFLOP/s, where a bf16 product of 8192^3 in the library reaches 1.27.  Matrix cores and vector
// units are busy 63 and 62 % of the cycles, and the clock gives way to them.  At d = 64 there are two weights to work out for every four products: 0.91 PFLOP/s
// for 2048 over 30k; with windows of 1024 (288 items, 350 TFLOP/s) they are busy 25 and 50 %, and the beginnings and ends of items are
// the rest.  What it took for the first, from 1461 us with all wavefronts in step: two of a SIMD a phase apart, one multiplies
// while the other works out weights (1220), operands read four products ahead, places without divisions, a head's ranges on one XCD (1163), no
// maximum per unit (1116), loading between the two products (1017), ranges by cost and masks by one comparison (960), items not cut where each has a
// workgroup (943 then).
#include <algorithm>

#include "chunk_share.h"

namespace svf {

namespace {

constexpr int kKeys = 64;                                // keys of a unit: 2 us
constexpr int kExtra = 4;                                // an item's beginning and end: 8 us

template <int D>
struct Kernel {
  static constexpr int R = kWaves * 32;                  // rows of an item
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kChunks = D / 8;                  // sixteen-byte chunks of a row
  static constexpr int kTileBytes = kKeys * kRowBytes;   // K or V of a unit
  static constexpr int kRowsPerPass = kThreads / kChunks;
  static constexpr int kPasses = kKeys / kRowsPerPass;
  static constexpr int kLds = 8 * kTileBytes;            // four units; at first the sums over the sequences
  // What cutting costs, a second beginning and the merge.  Cut and not, us, by the shares that the largest of 256 items has above the mean (8 x 256 tokens
  // over 1000 .. 7000, 32 heads): d = 128 10: 169, 147; 25: 168, 161; 33: 169, 170; 49: 174, 188; d = 64 10: 101, 95; 18: 102, 104; 25: 101, 111.  One
  // prompt of 2048 over 30k, 16: 940, 928 and 573, 590; of 1024 over nothing, 128 items, 14: 48, 39 and 33, 28.
  static constexpr int kJoin = D == 128 ? 24 : 14;
  static_assert((kMostB + 1) * 8 <= kLds, "");

  // K chunk c of key t at c ^ (t mod 16) (d = 64, two rows to a line of banks: c ^ (t / 2 mod 8)): sixteen lanes that read the same chunk of
  // sixteen keys hit all banks.
  static __device__ __forceinline__ uint32_t k_at(int t, int c) {
    return t * kRowBytes + ((c ^ (D == 128 ? t & 15 : (t >> 1) & 7)) << 4);
  }
  // V chunk c of key t at c ^ 4 (t mod 4) (d = 64: c ^ 4 (t / 2 mod 2) ): the four keys that sixteen lanes of a transposing read address
  // lie in different banks.
  static __device__ __forceinline__ uint32_t v_at(int t, int c) {
    return t * kRowBytes + ((c ^ (D == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1))) << 4);
  }
};

template <int D>
__global__ __launch_bounds__(kThreads, 2) void chunk_attn_kernel(ChunkParams p) {
  typedef Kernel<D> C;
  constexpr int R = C::R;
  __shared__ __attribute__((aligned(16))) char lds[C::kLds];
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
  if (!cursor_of_few<R, kKeys, kExtra, C::kJoin>(p, begin, take, c)) {
    int64_t* const cum = reinterpret_cast<int64_t*>(lds);
    units_before<R, kKeys, kExtra>(p, cum);
    begin(cum[p.B]);
    if (me < N) c = cursor_at<R, kKeys, kExtra>(p, cum, at);
    __syncthreads();
  }
  if (tid == 0) parts.join[me] = make_int4(-1, 0, 0, 0);
  if (me >= N) return;
  c.b = uniform(c.b);
  c.h = uniform(c.h);
  c.item = uniform(c.item);
  int skip = uniform((int)c.skip), left = uniform(c.whole > 0 ? c.whole : (int)(end - at));      // shares of the item in front of the range; shares to do

  const int c_lane = tid % C::kChunks, t_lane = tid / C::kChunks;
  const bool second = wave >= kWaves / 2;
  while (skip + left > kExtra) {                             // (else the range ends in front of an item's units)
    const ChunkSeq s{uniform(c.seq.len), uniform(c.seq.row), uniform(c.seq.n)};
    const Item<R, kKeys, kExtra> it(p, s, c.item);
    const Part part(it, skip, left);
    const int n = part.end - part.begin, unit0 = it.unit0 + part.begin;
    const int64_t first_unit = end - left - skip + kExtra;   // (counted in shares) of the item
    const char* const K = static_cast<const char*>(p.K) + 2 * (int64_t)c.h * p.kv.stride_head + 16 * c_lane;
    const char* const V = static_cast<const char*>(p.V) + 2 * (int64_t)c.h * p.kv.stride_head + 16 * c_lane;

    // A thread's chunks of a unit: looked up in the page table one unit ahead of their request, requested one unit ahead of their way
    // into LDS.  Places outside what the item's rows see are read as the nearest one inside.
    const int32_t* const table = p.table + (int64_t)c.b * p.kv.max_pages;
    struct Places { uint32_t page[C::kPasses], slot[C::kPasses]; };
    struct Chunks { u32x4 k[C::kPasses], v[C::kPasses]; };
    const auto look_up = [&](int u, Places& at) {
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const uint32_t t = (uint32_t)min(max((unit0 + u) * kKeys + t_lane + i * C::kRowsPerPass, it.first), it.last);
        const uint32_t np = p.page.of(t);
        at.slot[i] = t - np * (uint32_t)p.kv.page_size;
        at.page[i] = p.kv.page_size == 0 ? (uint32_t)c.b : (uint32_t)table[np];
      }
    };
    const auto request = [&](const Places& at, Chunks& x) {
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const uint32_t pg = at.page[i] < (uint32_t)p.n_pages ? at.page[i] : 0;
        const uint64_t off = (uint64_t)at.slot[i] * p.tok16 + (uint64_t)pg * p.page16;
        x.k[i] = *reinterpret_cast<const u32x4*>(K + 16 * off);
        x.v[i] = *reinterpret_cast<const u32x4*>(V + 16 * off);
      }
    };
    const auto put = [&](int buf, const Chunks& x) {
      char* const k = lds + buf * 2 * C::kTileBytes;
      char* const v = k + C::kTileBytes;
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const int t = t_lane + i * C::kRowsPerPass;
        *reinterpret_cast<u32x4*>(k + C::k_at(t, c_lane)) = x.k[i];
        *reinterpret_cast<u32x4*>(v + C::v_at(t, c_lane)) = x.v[i];
      }
    };
    Places at;
    Chunks on_way;
    Chunks begin[2];
    {
      Places a[3];
      look_up(0, a[0]);
      if (n > 1) look_up(1, a[1]);
      if (n > 2) look_up(2, a[2]);
      if (n > 3) look_up(3, at);
      request(a[0], begin[0]);
      if (n > 1) request(a[1], begin[1]);
      if (n > 2) request(a[2], on_way);
    }

    // this lane's row
    bf16x8 qf[D / 16];
    floatx16 o[D / 32] = {};
    const int row = it.row0 + min(wave * 32 + r32, it.rows - 1), row_j = row / p.G;
    const int hi = s.len + row_j, lo = p.window > 0 ? hi + 1 - p.window : 0;
    {
      const char* qr = static_cast<const char*>(p.q) +
                       2 * ((int64_t)(s.row + row_j) * p.q_stride + (int64_t)(c.h * p.G + row - row_j * p.G) * D) + 16 * hh;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qr + 32 * ks);
    }
    float m = -INFINITY, l = 0.f;
    // units whose keys every row of the item sees need no mask
    const int hi_all = s.len + it.row0 / p.G, lo_all = p.window > 0 ? it.last + 1 - p.window : 0;

    floatx16 sc[2];
    bf16x8 pf[4];
    // The two products of a unit, K Q^T (scores) and V^T P^T (outputs), kProducts instructions each.  Behind every instruction the
    // operand of the one four further on is read, into registers that were used four before: the scheduler, left alone, puts every read right
    // in front of its product and waits a trip to LDS for each.  V^T operands: lane 16 g + 4 j + x of a transposing read addresses channels
    // 16 (g mod 2) + 4 x .. + 3 of key j of the four keys of its half, and receives channel lane mod 16 of those keys.
    constexpr int kProducts = D / 8;
    const int vt = 4 * hh + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vb = 8 * (lane & 1);
    const auto k_operand = [&](int buf, int i) {
      return *reinterpret_cast<const bf16x8*>(lds + buf * 2 * C::kTileBytes + C::k_at(32 * (i & 1) + r32, 2 * (i / 2) + hh));
    };
    const auto v_operand = [&](int buf, int i) {
      const char* const v = lds + buf * 2 * C::kTileBytes + C::kTileBytes;
      shortx4 h[2];
#pragma unroll
      for (int z = 0; z < 2; ++z)
        h[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(
            v + C::v_at(16 * (i / (D / 32)) + 8 * z + vt, 4 * (i % (D / 32)) + vc) + vb));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const auto k_multiply = [&](int i, bf16x8 a) {
      sc[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[i / 2], i < 2 ? floatx16{} : sc[i & 1], 0, 0, 0);
    };
    const auto v_multiply = [&](int i, bf16x8 a) {
      const int cb = i % (D / 32);
      o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf[i / (D / 32)], o[cb], 0, 0, 0);
    };
    bf16x8 x[4], y[4];                                     // operands, in turn; x: of the next four products
    const auto scores = [&](int buf) {
#pragma unroll
      for (int g = 0; g < kProducts; g += 8) {
#pragma unroll
        for (int i = g; i < g + 4; ++i) {
          k_multiply(i, x[i - g]);
          y[i - g] = k_operand(buf, i + 4);
          SVF_IN_ORDER();
        }
#pragma unroll
        for (int i = g + 4; i < g + 8; ++i) {
          k_multiply(i, y[i - g - 4]);
          if (i + 4 < kProducts) x[i - g - 4] = k_operand(buf, i + 4);
          SVF_IN_ORDER();
        }
      }
    };
    const auto outputs = [&](int u) {                      // (and the scores' first operands)
#pragma unroll
      for (int g = 0; g < kProducts; g += 8) {
#pragma unroll
        for (int i = g; i < g + 4; ++i) {
          v_multiply(i, x[i - g]);
          y[i - g] = v_operand(u & 3, i + 4);
          SVF_IN_ORDER();
        }
#pragma unroll
        for (int i = g + 4; i < g + 8; ++i) {
          v_multiply(i, y[i - g - 4]);
          x[i - g - 4] = i + 4 < kProducts ? v_operand(u & 3, i + 4) : k_operand((u + 1) & 3, i + 4 - kProducts);
          SVF_IN_ORDER();
        }
      }
    };
    const auto phase_ends = [&]() {
      __builtin_amdgcn_sched_barrier(0);
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
    };
    // A unit's scores into weights, 2^(score - m), and their sum into l.  m need not be the maximum: weights, sums and outputs are
    // floating point, and good as long as nothing overflows.  So the maximum of the first unit that a row sees serves until a lane's weights of
    // a unit sum to more than 2^8 (the sums are there anyway; looking for the maximum of every unit cost a tenth of the time),
    // and then the unit is done again with the maximum it has.  A key weighs no more than 8 on average: values have nearly the range that weights of at
    // most one leave them.
    const auto exponents = [&](float use) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kk][i] = __builtin_fmaf(sc[kk][i], p.scale_log2, -use);
    };
    const auto exponentials = [&]() {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int b8 = 0; b8 < 2; ++b8) {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = __builtin_amdgcn_exp2f(sc[kk][8 * b8 + 2 * i]), y = __builtin_amdgcn_exp2f(sc[kk][8 * b8 + 2 * i + 1]);
            sum[i & 1] += x;
            sum[2 + (i & 1)] += y;
            w[i] = pack_bf16(x, y);
          }
          pf[2 * kk + b8] = __builtin_bit_cast(bf16x8, w);
        }
      return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    // (sc: exponents relative to m, or to 0 for a row that has seen nothing)
    const auto rebase = [&]() {
      float top = fmaxf(sc[0][0], sc[1][0]);
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(fmaxf(top, sc[0][i]), sc[1][i]);
      top = halves_max(top);
      float up = 0.f, f = 1.f;                             // (a row whose keys so far are all masked keeps -inf and weights of zero)
      if (top > -INFINITY) {
        if (m == -INFINITY) {                              // l and o are zero, and 2^-up may be infinite
          up = m = top;
        } else {
          up = fmaxf(top, 0.f);
          m += up;
          f = __builtin_amdgcn_exp2f(-up);
        }
      }
      l *= f;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) o[cb] *= f;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kk][i] -= up;
    };
    bool unseen = true;                                    // some row has seen nothing yet
    const auto weights = [&](int u) {
      const int key0 = (unit0 + u) * kKeys;
      if (key0 + kKeys - 1 > hi_all) {
        const int most = hi - key0 - 4 * hh;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * kk + 8 * (i / 4) + i % 4 > most) sc[kk][i] = -INFINITY;
      }
      if (key0 < lo_all) {
        const int least = lo - key0 - 4 * hh;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * kk + 8 * (i / 4) + i % 4 < least) sc[kk][i] = -INFINITY;
      }
      exponents(m == -INFINITY ? 0.f : m);
      if (unseen) {
        rebase();
        unseen = __ballot(m == -INFINITY) != 0;
      }
      float sum = exponentials();
      if (__ballot(sum > 0x1p8f)) {
        rebase();
        sum = exponentials();
      }
      l += sum;
    };
    put(0, begin[0]);
    if (n > 1) put(1, begin[1]);
    if (n > 2) put(2, on_way);
    if (n > 3) {
      request(at, on_way);
      if (n > 4) look_up(4, at);
    }
    __syncthreads();
    // The first four wavefronts and the second four, one of each on a SIMD, are a phase apart: while the ones multiply (the outputs of a unit
    // and the scores of the next) the others work out weights.
    if (second) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = k_operand(0, i);
    scores(0);
    phase_ends();
    for (int u = 0; u < n; ++u) {
      weights(u);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v_operand(u & 3, i);
      phase_ends();
      __builtin_amdgcn_s_setprio(2);                       // (the matrix cores first: 3 %)
      outputs(u);
      if (u + 3 < n) {
        // Loading, in the products' shadow: unit u + 3 into LDS (both have multiplied by the values of unit u - 1, which were there), u + 4
        // on its way, u + 5 looked up.  (One place for all three: 957 us then for 2048 tokens over 32k; among the first products 977, spread
        // over the outputs 1179, while the weights are worked out 1116.)
        put((u + 3) & 3, on_way);
        if (u + 4 < n) {
          request(at, on_way);
          if (u + 5 < n) look_up(u + 5, at);
        }
      }
      scores((u + 1) & 3);                                 // (of nothing behind the last unit)
      __builtin_amdgcn_s_setprio(0);
      phase_ends();
    }
    if (!second) __syncthreads();

    // this item's result, whole or a part
    if (part.begins && !part.ends && tid == 0)
      parts.join[me] = make_int4(c.b, c.h, c.item, owner_of(total, N, first_unit + it.units - 1));
    const int r = wave * 32 + r32;
    const float den = halves_sum(l);
    if (r < it.rows) {
      if (part.begins && part.ends) {
        const int head = c.h * p.G + row - row_j * p.G;
        const float inv = 1.0f / den;
        char* to = static_cast<char*>(p.out) + 2 * ((int64_t)(s.row + row_j) * p.out_stride + (int64_t)head * D) + 8 * hh;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const u32x2 w = {pack_bf16(o[cb][4 * g] * inv, o[cb][4 * g + 1] * inv),
                             pack_bf16(o[cb][4 * g + 2] * inv, o[cb][4 * g + 3] * inv)};
            *reinterpret_cast<u32x2*>(to + 64 * cb + 16 * g) = w;
          }
        if (p.lse && hh == 0) p.lse[(int64_t)(s.row + row_j) * p.Hq + head] = (m + log2f(den)) * 0.69314718055994530942f;
      } else {
        const int64_t at_part = (int64_t)(2 * me + (part.begins ? 1 : 0)) * R + r;
        float* to = parts.o + at_part * D + 4 * hh;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const floatx4 x = {o[cb][4 * g], o[cb][4 * g + 1], o[cb][4 * g + 2], o[cb][4 * g + 3]};
            *reinterpret_cast<floatx4*>(to + 32 * cb + 8 * g) = x;
          }
        if (hh == 0) parts.ml[at_part] = make_float2(m, den);
      }
    }

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

template <int D>
hipError_t launch_d(const ChunkParams& p, hipStream_t st) {
  typedef Kernel<D> C;
  hipLaunchKernelGGL(chunk_attn_kernel<D>, dim3(kWorkgroups), dim3(kThreads), 0, st, p);
  hipLaunchKernelGGL((chunk_merge_kernel<D, C::R, kKeys, kExtra>), dim3(kWorkgroups, (unsigned)std::min<int64_t>(C::R / 32, ((int64_t)p.max_new * p.G + 31) / 32)),
                     dim3(kThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace

size_t chunk_attn_workspace(int d) {
  return d == 128 ? Parts<128, Kernel<128>::R>::bytes(kWorkgroups) : Parts<64, Kernel<64>::R>::bytes(kWorkgroups);
}

hipError_t launch_chunk_attn(const ChunkParams& p, hipStream_t st) {
  return p.d == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace svf
