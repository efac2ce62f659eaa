// Attention of new tokens over the cache in fp32 (svf_chunk_attn).
//
// A workgroup of four wavefronts takes 32 query rows of one (sequence, KV head) - row r is query head r % G of
// new token r / G - and a share of the 32-token tiles they see; its wavefronts take the tiles in turn, each with a
// running maximum and denominator of its own, and are joined through LDS.  Both products run on the
// fp32 matrix instructions (v_mfma_f32_32x32x2_f32): S^T = K Q^T leaves a query row in lane mod 32 with sixteen of the
// tile's keys per lane, which is the operand that O^T += V^T P^T takes, one register per step; so the
// weights never leave their lanes, and K and V go from memory into operand registers (a K row's
// 16-byte chunks alternate between the wavefront's halves, as do the query's).
// Bound: 64 cycles per 4096 operations, 157 TFLOP/s over the chip.  Where rows are few the tiles are cut into
// splits, joined by a second launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "svf_chunk_device.h"

namespace svf {

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;

constexpr int kThreads = 256, kWaves = 4, kRows = 32, kTile = 32;
constexpr int kMostSplits = 64;
constexpr int kFill = 1024;                              // workgroups that fill the chip

int64_t row_tiles(int max_new, int G) { return ((int64_t)max_new * G + kRows - 1) / kRows; }

int splits_of(int B, int Hkv, int G, int max_new, int max_seq_len, int window) {
  const int64_t items = (int64_t)B * Hkv * row_tiles(max_new, G);
  // (a split has eight tiles at least: two for each wavefront)
  const int64_t keys = window > 0 ? std::min<int64_t>(max_seq_len, (int64_t)window + max_new) : max_seq_len;
  const int64_t most = std::min<int64_t>(kMostSplits, (keys + 8 * kTile - 1) / (8 * kTile));
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, kFill / items));
}

__device__ __forceinline__ float halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a workgroup does: rows row0 .. row0 + rows - 1 of (sequence b, KV head h), tiles [tile0, tile1)
struct Work {
  ChunkSeq s;
  int b, h, row0, rows, split, first, last;              // first, last + 1: the places its rows see
  int tile0, tile1;
};
__device__ __forceinline__ bool work_of(const ChunkParams& p, int64_t item, int n_splits, int64_t tiles, Work& w) {
  w.split = (int)(item % n_splits);
  item /= n_splits;
  const int64_t rt = item % tiles;
  const int pair = (int)(item / tiles);
  w.b = pair / p.Hkv;
  w.h = pair - w.b * p.Hkv;
  w.s = chunk_seq(p.seq_lens[w.b], p.new_rows[w.b], p.new_lens[w.b], p.max_seq_len, p.max_new, p.n_rows);
  const int64_t M = (int64_t)w.s.n * p.G;
  if (rt * kRows >= M) return false;
  w.row0 = (int)(rt * kRows);
  w.rows = (int)min((int64_t)kRows, M - rt * kRows);
  const int j0 = w.row0 / p.G, j1 = (w.row0 + w.rows - 1) / p.G;
  w.first = p.window > 0 ? max(0, w.s.len + j0 + 1 - p.window) : 0;
  w.last = w.s.len + j1;
  const int t0 = w.first / kTile, t1 = w.last / kTile + 1, n = t1 - t0;
  w.tile0 = t0 + (int)((int64_t)n * w.split / n_splits);
  w.tile1 = t0 + (int)((int64_t)n * (w.split + 1) / n_splits);
  return true;
}

// element offset of a token, with its page kept inside the pool
__device__ __forceinline__ int64_t place_of(const ChunkParams& p, int b, int t) {
  if (p.kv.page_size == 0) return (int64_t)b * p.kv.stride_page + (int64_t)t * p.kv.stride_tok;
  const int n = p.kv.page_shift >= 0 ? t >> p.kv.page_shift : t / p.kv.page_size;
  int page = p.table[(int64_t)b * p.kv.max_pages + n];
  if ((uint32_t)page >= (uint32_t)p.n_pages) page = 0;
  return (int64_t)page * p.kv.stride_page + (int64_t)(t - n * p.kv.page_size) * p.kv.stride_tok;
}

// partials: [item][32 rows][D] outputs relative to the maximum, then [item][32] (maximum, denominator)
template <int D>
__global__ __launch_bounds__(kThreads) void chunk_attn_f32_kernel(ChunkParams p, int n_splits, int64_t tiles, int64_t items,
                                                                  float* part_o, float2* part_ml) {
  __shared__ float so[kWaves][kRows][D + 4];
  __shared__ float sm[kWaves][kRows], sl[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hh = lane >> 5, r32 = lane & 31;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    Work w;
    if (!work_of(p, item, n_splits, tiles, w)) continue;
    const float* const q = static_cast<const float*>(p.q);
    const float* const K = static_cast<const float*>(p.K) + (int64_t)w.h * p.kv.stride_head;
    const float* const V = static_cast<const float*>(p.V) + (int64_t)w.h * p.kv.stride_head;
    const int row = w.row0 + min(r32, w.rows - 1), j = row / p.G;
    const float* qr = q + (int64_t)(w.s.row + j) * p.q_stride + (int64_t)(w.h * p.G + row - j * p.G) * D;
    floatx4 qf[D / 8];
#pragma unroll
    for (int c = 0; c < D / 8; ++c) qf[c] = *reinterpret_cast<const floatx4*>(qr + 4 * (2 * c + hh));
    const int hi = w.s.len + j, lo = p.window > 0 ? hi + 1 - p.window : 0;
    float m = -INFINITY, l = 0.f;
    floatx16 o[D / 32] = {};
    for (int t = w.tile0 + wave; t < w.tile1; t += kWaves) {
      // (places outside what the workgroup's rows see are read as the nearest one inside)
      const int base = t * kTile;
      const float* kr = K + place_of(p, w.b, min(max(base + r32, w.first), w.last));
      floatx16 s = {};
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        const floatx4 kf = *reinterpret_cast<const floatx4*>(kr + 4 * (2 * c + hh));
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[c][e], s, 0, 0, 0);
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = base + 8 * (i / 4) + 4 * hh + i % 4;
        if (key > hi || key < lo) s[i] = -INFINITY;
        top = fmaxf(top, s[i]);
      }
      const float now = fmaxf(m, halves_max(top) * p.scale_log2);
      const float use = now == -INFINITY ? 0.f : now;
      const float scale = __builtin_amdgcn_exp2f(m - use);
      m = now;
      l *= scale;
#pragma unroll
      for (int n = 0; n < D / 32; ++n) o[n] *= scale;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], p.scale_log2, -use));
        l += s[i];
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = base + 8 * (i / 4) + 4 * hh + i % 4;
        const float* vr = V + place_of(p, w.b, min(max(key, w.first), w.last));
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
          o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[32 * n + r32], s[i], o[n], 0, 0, 0);
      }
    }
    l = halves_sum(l);
    __syncthreads();                                     // (the item before has been read)
    if (hh == 0) {
      sm[wave][r32] = m;
      sl[wave][r32] = l;
    }
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4 x = {o[n][4 * g], o[n][4 * g + 1], o[n][4 * g + 2], o[n][4 * g + 3]};
        *reinterpret_cast<floatx4*>(&so[wave][r32][32 * n + 8 * g + 4 * hh]) = x;
      }
    __syncthreads();
    for (int i = tid; i < w.rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c = 4 * (i % (D / 4));
      float top = sm[0][r];
#pragma unroll
      for (int k = 1; k < kWaves; ++k) top = fmaxf(top, sm[k][r]);
      const float use = top == -INFINITY ? 0.f : top;
      floatx4 x = {};
      float den = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float f = __builtin_amdgcn_exp2f(sm[k][r] - use);
        den += f * sl[k][r];
        x += f * *reinterpret_cast<const floatx4*>(&so[k][r][c]);
      }
      if (n_splits > 1) {
        *reinterpret_cast<floatx4*>(part_o + (item * kRows + r) * D + c) = x;
        if (c == 0) part_ml[item * kRows + r] = make_float2(top, den);
      } else {
        const int rr = w.row0 + r, jj = rr / p.G, head = w.h * p.G + rr - jj * p.G;
        *reinterpret_cast<floatx4*>(static_cast<float*>(p.out) + (int64_t)(w.s.row + jj) * p.out_stride + (int64_t)head * D + c) =
            x / den;
        if (c == 0 && p.lse) p.lse[(int64_t)(w.s.row + jj) * p.Hq + head] = (top + log2f(den)) * 0.69314718055994530942f;
      }
    }
  }
}

// grid: one workgroup per (sequence, KV head, 32 rows)
template <int D>
__global__ __launch_bounds__(kThreads) void chunk_merge_f32_kernel(ChunkParams p, int n_splits, int64_t tiles, int64_t groups,
                                                                   const float* part_o, const float2* part_ml) {
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
    Work w;
    if (!work_of(p, group * n_splits, n_splits, tiles, w)) continue;
    for (int i = threadIdx.x; i < w.rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c = 4 * (i % (D / 4));
      float top = -INFINITY;
      for (int k = 0; k < n_splits; ++k) top = fmaxf(top, part_ml[((group * n_splits + k) * kRows) + r].x);
      floatx4 x = {};
      float den = 0.f;
      for (int k = 0; k < n_splits; ++k) {
        const int64_t at = (group * n_splits + k) * kRows + r;
        const float2 ml = part_ml[at];
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        den += f * ml.y;
        x += f * *reinterpret_cast<const floatx4*>(part_o + at * D + c);
      }
      const int rr = w.row0 + r, jj = rr / p.G, head = w.h * p.G + rr - jj * p.G;
      *reinterpret_cast<floatx4*>(static_cast<float*>(p.out) + (int64_t)(w.s.row + jj) * p.out_stride + (int64_t)head * D + c) =
          x / den;
      if (c == 0 && p.lse) p.lse[(int64_t)(w.s.row + jj) * p.Hq + head] = (top + log2f(den)) * 0.69314718055994530942f;
    }
  }
}

template <int D>
void launch_d(const ChunkParams& p, hipStream_t st) {
  const int n_splits = splits_of(p.B, p.Hkv, p.G, p.max_new, p.max_seq_len, p.window);
  const int64_t tiles = row_tiles(p.max_new, p.G), groups = (int64_t)p.B * p.Hkv * tiles, items = groups * n_splits;
  float* part_o = reinterpret_cast<float*>(p.ws + kChunkCounters);
  float2* part_ml = reinterpret_cast<float2*>(p.ws + kChunkCounters + (n_splits > 1 ? items * kRows * D * sizeof(float) : 0));
  hipLaunchKernelGGL(chunk_attn_f32_kernel<D>, dim3((unsigned)std::min<int64_t>(items, 1 << 20)), dim3(kThreads), 0, st, p,
                     n_splits, tiles, items, part_o, part_ml);
  if (n_splits > 1)
    hipLaunchKernelGGL(chunk_merge_f32_kernel<D>, dim3((unsigned)groups), dim3(kThreads), 0, st, p, n_splits, tiles, groups,
                       part_o, part_ml);
}

}  // namespace

size_t chunk_attn_f32_workspace(const svf_chunk_shape_t& s) {
  const int G = s.Hq / s.Hkv, n = splits_of(s.B, s.Hkv, G, s.max_new, s.max_seq_len, s.window);
  if (n == 1) return kChunkCounters;
  return kChunkCounters + (size_t)((int64_t)s.B * s.Hkv * row_tiles(s.max_new, G) * n) * kRows * (s.d * sizeof(float) + sizeof(float2));
}

hipError_t launch_chunk_attn_f32(const ChunkParams& p, hipStream_t st) {
  if (p.d == 64) launch_d<64>(p, st);
  else launch_d<128>(p, st);
  return hipGetLastError();
}

}  // namespace svf
