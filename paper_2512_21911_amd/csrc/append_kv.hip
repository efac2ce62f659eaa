// Appending new tokens to the cache, with the position rotation on the way (svf_append_kv).
//
// A workgroup takes one row.  What a row belongs to (sequence, place, page) is a chain of
// two reads, so the row's own data, whose addresses follow from the row alone, is requested before it:
// by the time the place is known the data is there.  The unit of work is a pair of 16-byte chunks of one
// head: the two halves of eight (bf16) or four (fp32) rotated pairs, or, where pairs are neighbours or
// nothing is rotated, two neighbouring chunks.  A token's sines and cosines serve all its heads: each is
// worked out once, by one thread, and handed over through LDS.
// The angle is reduced in fp64 (position times turns per position, minus the nearest whole number): the phase is
// then good to 2^-53 of the angle, and its sine and cosine are fp32 functions of a number in [-1/2, 1/2].
// Bound by memory: 8200 tokens of 32 + 2 x 8 heads of 128 in bf16, 202 MB read and written, in 45 us, 4.5 TB/s (a copy of 1 GiB: 5.5); a step of 64
// tokens 3.9 us, of which the launch is 2 and the chain of reads the rest.  (Four rows to a workgroup, whose sines and cosines share a pass: 6.0
// instead of 3.6 us for 64 rows, 43.1 instead of 42.3 for 8192.)
#include <algorithm>

#include "svf_chunk_device.h"

namespace svf {

namespace {

constexpr int kAppendThreads = 256;
constexpr double kTurnsPerRadian = 0.15915494309189533576888376337251436;

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

template <typename T> struct Chunk;                      // the sixteen bytes of a chunk as floats
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(u32x4 w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
    return w;
  }
};
template <> struct Chunk<__hip_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    typedef __attribute__((__vector_size__(2 * sizeof(float)))) float floatx2;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx2 f = {x[2 * i], x[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
    }
    return w;
  }
};

template <typename T, int D>
__global__ __launch_bounds__(kAppendThreads) void append_kv_kernel(AppendParams p) {
  constexpr int N = Chunk<T>::N;
  constexpr int kUnits = D / (2 * N);                    // units of a head
  constexpr int kStep = kAppendThreads / kUnits;         // heads that the workgroup takes at once
  constexpr int kAhead = 3;                              // units of a thread on their way together
  __shared__ float2 turn[D / 2];                         // (cosine, sine) of the pairs
  // what each wavefront found: whether the row belongs to a sequence, element offset of the token in the pools (-1: not written), position
  constexpr int kWaves = kAppendThreads / 64;
  __shared__ int64_t places[kWaves];
  __shared__ int owned[kWaves], positions[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = (int)(blockIdx.y * gridDim.x + blockIdx.x);
  if (row >= p.n_rows) return;
  const int heads = p.Hq + 2 * p.Hkv, half = p.rotary_dim / 2;
  const int u = tid & (kUnits - 1), h0 = tid / kUnits;

  // the two chunks of a unit: partners of a rotation, or neighbours
  const int rotated = p.interleaved ? 0 : half / N;      // units whose chunks are half a rotation apart
  const int c0 = u < rotated ? u : 2 * u, c1 = u < rotated ? u + rotated : 2 * u + 1;

  const T* const q = static_cast<const T*>(p.q);
  const T* const kn = static_cast<const T*>(p.k_new);
  const T* const vn = static_cast<const T*>(p.v_new);
  // head numbers of a token: its query heads, then keys, then values
  const auto source = [&](int h) -> const T* {
    if (h < p.Hq) return q + (int64_t)row * p.q_stride + (int64_t)h * D;
    if (h < p.Hq + p.Hkv) return kn + (int64_t)row * p.k_stride + (int64_t)(h - p.Hq) * D;
    return vn + (int64_t)row * p.v_stride + (int64_t)(h - p.Hq - p.Hkv) * D;
  };
  u32x4 a[kAhead], b[kAhead];
  const auto request = [&](int at) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const T* s = source(min(at + i * kStep, heads - 1));
      a[i] = *reinterpret_cast<const u32x4*>(s + c0 * N);
      b[i] = *reinterpret_cast<const u32x4*>(s + c1 * N);
    }
  };
  request(h0);

  // which sequence has the row: each wavefront looks at 64 in turn
  {
    int who = -1, j = 0, len = 0;
    for (int s0 = 64 * wave; s0 < p.B && who < 0; s0 += kAppendThreads) {
      const int s = min(s0 + lane, p.B - 1);
      const ChunkSeq c = chunk_seq(p.seq_lens[s], p.new_rows[s], p.new_lens[s], p.max_seq_len, p.max_new, p.n_rows);
      const uint64_t has = __ballot(s0 + lane < p.B && row >= c.row && row - c.row < c.n);
      if (has) {
        const int l = __builtin_ctzll(has);
        who = s0 + l;
        j = row - __builtin_amdgcn_readlane(c.row, l);
        len = __builtin_amdgcn_readlane(c.len, l);
      }
    }
    if (lane == 0) {
      int64_t at = -1;
      if (who >= 0) {
        const int tok = len + j;
        int page = who, slot = tok;
        if (p.kv.page_size > 0) {
          const int n = p.kv.page_shift >= 0 ? tok >> p.kv.page_shift : tok / p.kv.page_size;
          slot = tok - n * p.kv.page_size;
          page = p.table[(int64_t)who * p.kv.max_pages + n];
        }
        if (page >= 0 && page < p.n_pages) at = (int64_t)page * p.kv.stride_page + (int64_t)slot * p.kv.stride_tok;
        positions[wave] = p.positions ? p.positions[row] : tok;
      }
      places[wave] = at;
      owned[wave] = who >= 0;
    }
  }
  __syncthreads();
  int by = 0;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) by = owned[w] ? w : by;
  if (!owned[by]) return;
  const int64_t place = places[by];
  if (half > 0) {
    if (tid < half) {
      double turns = (double)positions[by] * (p.inv_freq[tid] * kTurnsPerRadian);
      turns -= rint(turns);
      float s, c;
      sincospif(2.0f * (float)turns, &s, &c);
      turn[tid] = make_float2(c * p.rotary_scale, s * p.rotary_scale);
    }
    __syncthreads();
  }

  for (int at = h0; at < heads; at += kAhead * kStep) {
    if (at != h0) request(at);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = at + i * kStep;
      if (h >= heads) continue;
      u32x4 wa = a[i], wb = b[i];
      if (h < p.Hq + p.Hkv && c0 * N < p.rotary_dim) {
        float x[N], y[N], rx[N], ry[N];
        Chunk<T>::unpack(wa, x);
        Chunk<T>::unpack(wb, y);
        if (p.interleaved) {
          // (two chunks of neighbours; rotary_dim is a multiple of sixteen, so both are rotated)
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            const float2 m = turn[c0 * (N / 2) + e], n2 = turn[c1 * (N / 2) + e];
            rx[2 * e] = x[2 * e] * m.x - x[2 * e + 1] * m.y;
            rx[2 * e + 1] = x[2 * e + 1] * m.x + x[2 * e] * m.y;
            ry[2 * e] = y[2 * e] * n2.x - y[2 * e + 1] * n2.y;
            ry[2 * e + 1] = y[2 * e + 1] * n2.x + y[2 * e] * n2.y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 m = turn[c0 * N + e];
            rx[e] = x[e] * m.x - y[e] * m.y;
            ry[e] = y[e] * m.x + x[e] * m.y;
          }
        }
        wa = Chunk<T>::pack(rx);
        wb = Chunk<T>::pack(ry);
      }
      T* to;
      if (h < p.Hq) {
        to = static_cast<T*>(p.q_out) + (int64_t)row * p.q_stride + (int64_t)h * D;
      } else {
        if (place < 0) continue;
        const bool key = h < p.Hq + p.Hkv;
        to = static_cast<T*>(key ? p.K : p.V) + place + (int64_t)(h - p.Hq - (key ? 0 : p.Hkv)) * p.kv.stride_head;
      }
      *reinterpret_cast<u32x4*>(to + c0 * N) = wa;
      *reinterpret_cast<u32x4*>(to + c1 * N) = wb;
    }
  }
}

template <typename T, int D>
void launch_typed(const AppendParams& p, hipStream_t st) {
  constexpr int kMostX = 1 << 22;                        // (a grid's threads in x are a 32-bit number)
  const int x = std::min(p.n_rows, kMostX);
  hipLaunchKernelGGL((append_kv_kernel<T, D>), dim3((unsigned)x, (unsigned)((p.n_rows + x - 1) / x)), dim3(kAppendThreads), 0, st, p);
}

}  // namespace

hipError_t launch_append_kv(const AppendParams& p, int dtype, hipStream_t st) {
  if (dtype == SVF_F32) {
    if (p.d == 64) launch_typed<float, 64>(p, st);
    else launch_typed<float, 128>(p, st);
  } else {
    if (p.d == 64) launch_typed<__hip_bfloat16, 64>(p, st);
    else launch_typed<__hip_bfloat16, 128>(p, st);
  }
  return hipGetLastError();
}

}  // namespace svf
