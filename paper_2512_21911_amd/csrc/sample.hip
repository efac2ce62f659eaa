// Sampling from logits (svf_sample): temperature, top-k, top-p, min-p, and the draw by inversion.
//
// All three filters keep a prefix of the tokens in descending order of their logits (ties by index), so what a row keeps is
// one number: the key of the last kept logit and how many of the tokens with that key stay.  It is found
// by radix selection over the logits' bit patterns, by count (top-k) and by weight (top-p).  Equal logits have equal weights, so
// the ties at the border need no sorting.  Weights are added in fixed point: sums do not depend on their order.
#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>

#include "svf_device.h"
#include "svf_rules.h"

namespace svf {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kFraction = 43;                            // bits of a weight behind the point; 2^19 weights of one fit 63 bits
constexpr uint32_t kLowestKey = 0x007fffffu;             // of -inf

struct SampleParams {
  const void* logits;
  int64_t stride;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* tokens;
  float* probs;
  int32_t rows, V;
};

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__hip_bfloat16 x) { return __bfloat162float(x); }
// (NaN counts as -inf)
template <typename T>
__device__ __forceinline__ float logit(const T* x, int v) {
  const float f = as_float(x[v]);
  return f == f ? f : -INFINITY;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

struct Row {
  float top;                 // the largest logit
  double to_log2;            // log2(e) / temperature
  __device__ __forceinline__ double log2_weight(float x) const { return x == top ? 0.0 : ((double)x - (double)top) * to_log2; }
  __device__ __forceinline__ uint64_t weight(float x) const {
    return (uint64_t)(exp2(log2_weight(x)) * (double)(1ull << kFraction) + 0.5);
  }
};

__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) x += __shfl_xor((unsigned long long)x, d, 64);
  return x;
}
__device__ __forceinline__ uint64_t block_sum64(uint64_t x, uint64_t* sh) {
  x = wave_sum64(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  uint64_t s = 0;
  for (int w = 0; w < kWaves; ++w) s += sh[w];
  return s;
}

// The largest key such that the tokens with keys above it have less than `limit` (of count, or weight) and those with it and above have
// at least that; `before`: what those above have.  (All threads return the same.)
template <typename T, bool WEIGHT>
__device__ uint32_t select_key(const T* x, int V, const Row& row, uint64_t limit, unsigned long long* hist, uint64_t* sh,
                               uint64_t& before) {
  uint32_t prefix = 0;
  before = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t hi_mask = shift == 24 ? 0u : (0xffffffffu << (shift + 8));
    for (int v = threadIdx.x; v < V; v += kThreads) {
      const float f = logit(x, v);
      const uint32_t key = score_key(f);
      if ((key & hi_mask) == prefix) atomicAdd(&hist[(key >> shift) & 255], WEIGHT ? (unsigned long long)row.weight(f) : 1ull);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint64_t sum = before;
      int bin = 255;
      for (; bin > 0; --bin) {
        if (sum + hist[bin] >= limit) break;
        sum += hist[bin];
      }
      sh[0] = sum;
      sh[1] = prefix | ((uint32_t)bin << shift);
    }
    __syncthreads();
    before = sh[0];
    prefix = (uint32_t)sh[1];
    __syncthreads();
  }
  return prefix;
}

// grid: (rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p) {
  __shared__ unsigned long long hist[256];
  __shared__ uint64_t sh[kWaves];
  __shared__ float shf[kWaves];
  __shared__ int shi[kWaves];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = p.V;
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  Row row;
  row.top = -INFINITY;
  for (int v = tid; v < V; v += kThreads) row.top = fmaxf(row.top, logit(x, v));
#pragma unroll
  for (int d = 32; d > 0; d /= 2) row.top = fmaxf(row.top, __shfl_xor(row.top, d, 64));
  if (lane == 0) shf[wave] = row.top;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) row.top = fmaxf(row.top, shf[w]);
  float* const probs = p.probs ? p.probs + (int64_t)r * V : nullptr;
  if (row.top == -INFINITY) {
    if (probs)
      for (int v = tid; v < V; v += kThreads) probs[v] = 0.f;
    if (tid == 0 && p.tokens) p.tokens[r] = -1;
    return;
  }
  float temperature = p.temperature ? p.temperature[r] : 1.f;
  int k = p.top_k ? p.top_k[r] : 0;
  if (!(temperature > 0.f)) {
    temperature = 1.f;
    k = 1;
  }
  row.to_log2 = 1.4426950408889634074 / (double)temperature;
  // what is kept: keys above `key`, and the first `ties` tokens with it
  uint32_t key = kLowestKey;
  uint64_t ties = (uint64_t)V, before;
  if (k > 0 && k < V) {
    key = select_key<T, false>(x, V, row, (uint64_t)k, hist, sh, before);
    ties = (uint64_t)k - before;
  }
  const float top_p = p.top_p ? p.top_p[r] : 1.f;
  if (top_p < 1.f) {
    uint64_t mass = 0, same = 0;
    for (int v = tid; v < V; v += kThreads) {
      const float f = logit(x, v);
      const uint32_t kf = score_key(f);
      if (kf > key) mass += row.weight(f);
      same += kf == key;
    }
    mass = block_sum64(mass, sh);
    same = block_sum64(same, sh);
    mass += min(ties, same) * row.weight(key_logit(key));
    const double share = ceil((double)top_p * (double)mass);
    const uint64_t limit = share < 1.0 ? 1 : (uint64_t)share;
    const uint32_t at = select_key<T, true>(x, V, row, limit, hist, sh, before);
    const uint64_t w = row.weight(key_logit(at));
    const uint64_t n = w == 0 ? (uint64_t)V : (limit - before + w - 1) / w;
    if (at > key) {
      key = at;
      ties = n;
    } else {
      ties = min(ties, n);
    }
  }
  const float min_p = p.min_p ? p.min_p[r] : 0.f;
  if (min_p > 0.f) {
    const double least = (double)row.top + (double)temperature * log((double)min_p);
    float f = (float)least;
    if ((double)f < least) f = nextafterf(f, INFINITY);
    const uint32_t at = score_key(fminf(f, row.top));
    if (at > key) {
      key = at;
      ties = (uint64_t)V;
    }
  }
  // the wavefronts' shares, consecutive tokens each
  const int share = (V + kWaves * 64 - 1) / (kWaves * 64) * 64, v0 = min(wave * share, V), v1 = min(v0 + share, V);
  int same = 0;
  uint64_t mass = 0;
  for (int v = v0 + lane; v < v1; v += 64) {
    const float f = logit(x, v);
    const uint32_t kf = score_key(f);
    same += kf == key;
    if (kf > key) mass += row.weight(f);
  }
#pragma unroll
  for (int d = 32; d > 0; d /= 2) same += __shfl_xor(same, d, 64);
  if (lane == 0) shi[wave] = same;
  __syncthreads();
  uint64_t seen = 0;                                      // ties in front of this wavefront's share
  for (int w = 0; w < wave; ++w) seen += shi[w];
  const uint64_t wkey = row.weight(key_logit(key));
  mass = wave_sum64(mass) + wkey * (seen >= ties ? 0 : min((uint64_t)same, ties - seen));
  __syncthreads();
  if (lane == 0) sh[wave] = mass;
  __syncthreads();
  uint64_t total = 0, front = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) front = total;
    total += sh[w];
  }
  uint64_t target = ~0ull;
  if (p.tokens) {
    const double t = (double)p.u[r] * (double)total;
    target = t > 0.0 ? (uint64_t)t : 0;
    target = min(target, total - 1);
  }
  const bool holds = p.tokens && target >= front && target < front + mass;
  if (!probs && !holds) return;
  const double inv = 1.0 / ((double)total / (double)(1ull << kFraction));
  uint64_t run = front;
  bool found = false;
  for (int v = v0; v < v1; v += 64) {
    const float f = v + lane < v1 ? logit(x, v + lane) : -INFINITY;
    const uint32_t kf = score_key(f);
    const uint64_t tied = __ballot(v + lane < v1 && kf == key);
    const uint64_t rank = seen + __popcll(tied & ((1ull << lane) - 1));
    const bool kept = v + lane < v1 && f != -INFINITY && (kf > key || (kf == key && rank < ties));
    seen += __popcll(tied);
    if (probs && v + lane < v1) probs[v + lane] = kept ? (float)(exp2(row.log2_weight(f)) * inv) : 0.f;
    if (holds && !found) {
      uint64_t s = kept ? row.weight(f) : 0;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up((unsigned long long)s, d, 64);
        if (lane >= d) s += o;
      }
      const uint64_t hit = __ballot(run + s > target);
      if (hit) {
        found = true;
        if (lane == 0) p.tokens[r] = v + __builtin_ctzll(hit);
      }
      run += __shfl((unsigned long long)s, 63, 64);
    }
  }
}

}  // namespace

}  // namespace svf

extern "C" {

size_t svf_sample_workspace_bytes(int32_t rows, int32_t V) {
  if (rows < 1 || V < 1 || V > 524288) return 0;
  return 256;
}

int svf_sample(const void* logits, int32_t dtype, int64_t logits_stride, int32_t rows, int32_t V,
               const float* temperature_or_null, const int32_t* top_k_or_null, const float* top_p_or_null,
               const float* min_p_or_null, const float* u_or_null, int32_t* tokens_or_null, float* probs_or_null,
               void* ws, size_t ws_bytes, void* stream) {
  if (dtype != SVF_F32 && dtype != SVF_BF16) return SVF_ERR_DTYPE;
  if (!logits || (u_or_null == nullptr) != (tokens_or_null == nullptr) || (!tokens_or_null && !probs_or_null)) return SVF_ERR_NULL;
  if (rows < 1 || V < 1 || V > 524288 || (logits_stride != 0 && logits_stride < V)) return SVF_ERR_SHAPE;
  const auto misaligned = [](const void* q, uintptr_t to) { return reinterpret_cast<uintptr_t>(q) % to != 0; };
  if (misaligned(logits, dtype == SVF_F32 ? 4 : 2) || misaligned(temperature_or_null, 4) || misaligned(top_k_or_null, 4) ||
      misaligned(top_p_or_null, 4) || misaligned(min_p_or_null, 4) || misaligned(u_or_null, 4) || misaligned(tokens_or_null, 4) ||
      misaligned(probs_or_null, 4))
    return SVF_ERR_SHAPE;
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < svf_sample_workspace_bytes(rows, V)) return SVF_ERR_WORKSPACE;
  svf::SampleParams p;
  p.logits = logits;
  p.stride = logits_stride ? logits_stride : V;
  p.temperature = temperature_or_null;
  p.top_k = top_k_or_null;
  p.top_p = top_p_or_null;
  p.min_p = min_p_or_null;
  p.u = u_or_null;
  p.tokens = tokens_or_null;
  p.probs = probs_or_null;
  p.rows = rows;
  p.V = V;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == SVF_F32) hipLaunchKernelGGL(svf::sample_kernel<float>, dim3(rows), dim3(svf::kThreads), 0, st, p);
  else hipLaunchKernelGGL(svf::sample_kernel<__hip_bfloat16>, dim3(rows), dim3(svf::kThreads), 0, st, p);
  return hipGetLastError() == hipSuccess ? SVF_OK : SVF_ERR_HIP;
}

}  // extern "C"
