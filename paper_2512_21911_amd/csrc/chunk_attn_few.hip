// Attention of a few new tokens over the cache in bf16 (svf_chunk_attn): up to 32 query rows per (sequence, KV head), as
// for single tokens.
//
// Bound: the cache goes by once, so the kernel is there to keep memory busy.  The matrix cores still do both products (32 rows at a time,
// whatever of them is used).  The eight wavefronts of a workgroup have nothing to do with one another until the end of an item: each takes
// every eighth unit of 32 keys, brings it into LDS of its own through registers - sixteen 16-byte loads of a lane, the next unit's on their way
// while one is worked on, 128 KB in flight on a compute unit - and keeps its own maximum, sum and output.  Then the eight are joined through LDS.
// Weights keep sixteen bits (two bf16 terms): the matrix cores have the time.
#include "chunk_share.h"

namespace svf {

namespace {

constexpr int kFewRows = 32;
constexpr int kFewKeys = 32;                             // keys of a unit

template <int D>
struct Few {
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kChunks = D / 8;
  static constexpr int kTileBytes = kFewKeys * kRowBytes;
  static constexpr int kLanesRows = 64 / kChunks;        // rows that a wavefront loads at once
  static constexpr int kPasses = kFewKeys / kLanesRows;
  // (where a chunk of a row sits: as in the kernel for many rows)
  static __device__ __forceinline__ uint32_t k_at(int t, int c) {
    return t * kRowBytes + ((c ^ (D == 128 ? t & 15 : (t >> 1) & 7)) << 4);
  }
  static __device__ __forceinline__ uint32_t v_at(int t, int c) {
    return t * kRowBytes + ((c ^ (D == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1))) << 4);
  }
};

template <int D>
__global__ __launch_bounds__(kThreads, 2) void chunk_attn_few_kernel(ChunkParams p) {
  typedef Few<D> C;
  constexpr int R = kFewRows;
  constexpr int kOwn = 2 * C::kTileBytes;                // a wavefront's K and V; at the end its output, as many bytes
  static_assert(kOwn == kFewRows * D * 4, "");
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kOwn];
  __shared__ float2 joint[kWaves][kFewRows];
  __shared__ bool joins;
  static_assert((kMostB + 1) * 8 <= kWaves * kOwn, "");
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), hh = lane >> 5, r32 = lane & 31;
  const Parts<D, R> parts(p.ws, gridDim.x);

  // where this workgroup's range begins
  int64_t total = 0, at = 0, end = 0;
  int N = 0, me = 0;
  const auto begin = [&](int64_t all) {
    total = all;
    N = (int)min((int64_t)kWorkgroups, total);             // workgroups with work: one unit at least
    // Consecutive ranges, which read the same keys, go to one XCD and its L2: workgroups are dealt to the eight in turn
    me = N == kWorkgroups ? (int)(blockIdx.x % kXcds * (kWorkgroups / kXcds) + blockIdx.x / kXcds) : (int)blockIdx.x;
    at = me < N ? range_begin(total, N, me) : total;
    end = me < N ? range_begin(total, N, me + 1) : total;
    return at;
  };
  Cursor c;
  if (!cursor_of_few<R, kFewKeys, true>(p, begin, c)) {
    int64_t* const cum = reinterpret_cast<int64_t*>(lds);
    units_before<R, kFewKeys>(p, cum);
    begin(cum[p.B]);
    if (me < N) c = cursor_at<R, kFewKeys>(p, cum, at);
    __syncthreads();
  }
  if (me >= N) return;
  c.b = uniform(c.b);
  c.h = uniform(c.h);
  int skip = uniform((int)c.skip), left = uniform((int)(end - at));

  char* const mine = lds + wave * kOwn;
  const int c_lane = lane % C::kChunks, t_lane = lane / C::kChunks;
  while (left > 0) {
    ChunkSeq s = load_seq(p, c.b);
    s = {uniform(s.len), uniform(s.row), uniform(s.n)};
    const Item<R, kFewKeys> it(p, s, 0);                 // (one item per KV head: all its rows)
    const int n = min(it.units - skip, left);
    const int unit0 = it.unit0 + skip;
    const char* const K = static_cast<const char*>(p.K) + 2 * (int64_t)c.h * p.kv.stride_head + 16 * c_lane;
    const char* const V = static_cast<const char*>(p.V) + 2 * (int64_t)c.h * p.kv.stride_head + 16 * c_lane;
    const int32_t* const table = p.table + (int64_t)c.b * p.kv.max_pages;
    struct Places { uint32_t page[C::kPasses], slot[C::kPasses]; };
    struct Chunks { u32x4 k[C::kPasses], v[C::kPasses]; };
    const auto look_up = [&](int u, Places& to) {
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const uint32_t t = (uint32_t)min(max((unit0 + u) * kFewKeys + t_lane + i * C::kLanesRows, it.first), it.last);
        const uint32_t np = p.page.of(t);
        to.slot[i] = t - np * (uint32_t)p.kv.page_size;
        to.page[i] = p.kv.page_size == 0 ? (uint32_t)c.b : (uint32_t)table[np];
      }
    };
    const auto request = [&](const Places& from, Chunks& x) {
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const uint32_t pg = from.page[i] < (uint32_t)p.n_pages ? from.page[i] : 0;
        const uint64_t off = (uint64_t)from.slot[i] * p.tok16 + (uint64_t)pg * p.page16;
        x.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(K + 16 * off));
        x.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(V + 16 * off));
      }
    };
    Places places;
    Chunks x;
    if (wave < n) {
      look_up(wave, places);
      request(places, x);
      if (wave + kWaves < n) look_up(wave + kWaves, places);
    }

    bf16x8 qf[D / 16];
    const int row = it.row0 + min(r32, it.rows - 1), row_j = row / p.G;
    const int hi = s.len + row_j, lo = p.window > 0 ? hi + 1 - p.window : 0;
    {
      const char* qr = static_cast<const char*>(p.q) +
                       2 * ((int64_t)(s.row + row_j) * p.q_stride + (int64_t)(c.h * p.G + row - row_j * p.G) * D) + 16 * hh;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qr + 32 * ks);
    }
    floatx16 o[D / 32] = {};
    float m = -INFINITY, l = 0.f;
    const int hi_all = s.len, lo_all = p.window > 0 ? it.last + 1 - p.window : 0;
    const int vt = 4 * hh + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vb = 8 * (lane & 1);
    for (int u = wave; u < n; u += kWaves) {
      char* const k = mine;
      char* const v = mine + C::kTileBytes;
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const int t = t_lane + i * C::kLanesRows;
        *reinterpret_cast<u32x4*>(k + C::k_at(t, c_lane)) = x.k[i];
        *reinterpret_cast<u32x4*>(v + C::v_at(t, c_lane)) = x.v[i];
      }
      if (u + kWaves < n) {
        request(places, x);
        if (u + 2 * kWaves < n) look_up(u + 2 * kWaves, places);
      }
      floatx16 sc = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(k + C::k_at(r32, 2 * ks + hh)), qf[ks], sc, 0, 0, 0);
      const int key0 = (unit0 + u) * kFewKeys;
      if (key0 + kFewKeys - 1 > hi_all || key0 < lo_all) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 8 * (i / 4) + 4 * hh + i % 4;
          if (key > hi || key < lo) sc[i] = -INFINITY;
        }
      }
      float top = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
      top = halves_max(top) * p.scale_log2;
      if (__ballot(top > m)) {
        const float now = fmaxf(m, top), f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= f;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) o[cb] *= f;
      }
      const float use = m == -INFINITY ? 0.f : m;
      bf16x8 high[2], low[2];
#pragma unroll
      for (int b8 = 0; b8 < 2; ++b8) {
        u32x4 wh, wl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * b8 + 2 * i], p.scale_log2, -use));
          const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[8 * b8 + 2 * i + 1], p.scale_log2, -use));
          l += a + b;
          wh[i] = pack_bf16(a, b);
          wl[i] = pack_bf16(a - __uint_as_float(wh[i] << 16), b - __uint_as_float(wh[i] & 0xffff0000u));
        }
        high[b8] = __builtin_bit_cast(bf16x8, wh);
        low[b8] = __builtin_bit_cast(bf16x8, wl);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) {
          shortx4 y[2];
#pragma unroll
          for (int z = 0; z < 2; ++z)
            y[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) shortx4*)(v + C::v_at(16 * kb + 8 * z + vt, 4 * cb + vc) + vb));
          const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(y[0], y[1], 0, 1, 2, 3, 4, 5, 6, 7));
          o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, high[kb], o[cb], 0, 0, 0);
          o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, low[kb], o[cb], 0, 0, 0);
        }
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
    const bool whole = skip == 0 && n == it.units;
    const int64_t first_unit = end - left - skip;           // of the item
    const int from = whole ? me : owner_of(total, N, first_unit), upto = whole ? me : owner_of(total, N, first_unit + it.units - 1);
    const auto write = [&](int r, int ch, float top, float den, floatx4 y) {
      const int j = r / p.G, head = c.h * p.G + r - j * p.G;
      const float inv = 1.0f / den;
      const u32x2 w = {pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv)};
      *reinterpret_cast<u32x2*>(static_cast<char*>(p.out) + 2 * ((int64_t)(s.row + j) * p.out_stride + (int64_t)head * D + ch)) = w;
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

    left -= n;
    skip = 0;
    if (++c.h == p.Hkv) {
      c.h = 0;
      ++c.b;
      while (left > 0 && load_seq(p, c.b).n == 0) ++c.b;
    }
  }
}

template <int D>
hipError_t launch_few_d(const ChunkParams& p, hipStream_t st) {
  hipLaunchKernelGGL(chunk_attn_few_kernel<D>, dim3(kWorkgroups), dim3(kThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace

bool chunk_attn_is_few(int G, int max_new) { return (int64_t)G * max_new <= kFewRows; }

size_t chunk_attn_few_workspace(int d) {
  return d == 128 ? Parts<128, kFewRows>::bytes(kWorkgroups) : Parts<64, kFewRows>::bytes(kWorkgroups);
}

hipError_t launch_chunk_attn_few(const ChunkParams& p, hipStream_t st) {
  return p.d == 128 ? launch_few_d<128>(p, st) : launch_few_d<64>(p, st);
}

}  // namespace svf
