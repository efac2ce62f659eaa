// Sampling from logits (svf_sample): temperature, top-k, top-p, min-p, and the draw by inversion.
//
// All three filters keep a prefix of the tokens in descending order of their logits (ties by index), so what a row keeps
// is two numbers, a border: the key of the last kept logit and the index of the last kept token with it.  Nothing is sorted
// but the few tokens around it.  A row is cut into slices, and three launches find border and token:
//   stats    a workgroup per slice reads its logits once, into registers: their maximum, the sum of their weights, and, if the row has a
//            filter, a histogram of counts and weights over 1023 bins of logits below the maximum (and one for the rest).
//   gather   every workgroup adds up the row's histograms for itself and knows the bin the border is in; it reads its slice again only if
//            it has tokens there, and writes those to the row's list (top-k: all from the top on, so that
//            the mass that top-p takes its share of is at hand).
//   draw     a workgroup per row sorts the list, walks it to the border, adds up what every slice keeps, and walks the one slice the
//            target falls in.
// and a fourth, with a workgroup per slice again, writes the probabilities where they are asked for.
// A row whose border bin has more tokens than the list (many equal logits, a top-k of thousands) is settled in the third launch by
// radix selection over the whole row.
//
// Weights are fixed-point numbers relative to their slice's maximum, so that sums do not depend on their order; slices are brought to the row's
// maximum by one factor each.  2^t is a table of 64 entries in 64 bits times a cubic: good to 2^-30, which an fp32 exponential (2^-23) is
// not, and a hundred thousand borders of tokens wait for the target in between.
// Bound: the logits, once from memory and, where the border's bin is gathered and the slice walked, again from the caches.
#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "svf_device.h"
#include "svf_rules.h"

namespace svf {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kFraction = 43;                            // bits of a weight behind the point; 2^19 weights of one fit 63 bits
constexpr int kBins = 1024;                              // the last: everything below the others
constexpr int kList = 4096;                              // tokens around the border that are sorted
constexpr int kTable = 64;
constexpr double kLog2e = 1.4426950408889634074;

struct SliceStats {
  float top;                 // largest logit; -inf: the slice has none above that
  int32_t n;                 // logits above -inf (rows with a filter)
  uint64_t total;            // sum of the weights, relative to top
  uint64_t above;            // of the tokens in bins above the list's
};
enum { kEverything, kFromList, kSlow };                  // how the border is found
struct RowPlan {
  float top;
  int32_t how, listed, k;    // k: top-k, 0 if it drops nothing
  uint64_t limit, above;     // without top-k: the weight (relative to top) that the kept tokens reach, and what is above the list's bin
};
struct Border { uint32_t key; int32_t index; double inv_total; };     // inv_total: 1 / total weight of the kept tokens

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
  int32_t rows, V, slice, slices;
  SliceStats* stats;         // [rows][slices]
  uint64_t* mass;            // [rows][slices][kBins]
  uint32_t* count;           // [rows][slices][kBins]
  uint64_t* list;            // [rows][kList]: ~key in the high half, index in the low one
  RowPlan* plan;             // [rows]
  Border* border;            // [rows]
};

// ---- logits ----------------------------------------------------------------------------------------

// NaN counts as -inf; +inf as the largest finite number, so that differences are numbers
__device__ __forceinline__ float clean(float x) { return x == x ? fminf(x, 3.402823466e38f) : -INFINITY; }

// Four consecutive logits on the element type's own boundary (rows of odd length start on no better one).
typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t uint2_u __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ float4 load4(const float* p) {
  const float4_u x = *reinterpret_cast<const float4_u*>(p);
  return make_float4(x.x, x.y, x.z, x.w);
}
__device__ __forceinline__ float4 load4(const __hip_bfloat16* p) {
  const uint2_u x = *reinterpret_cast<const uint2_u*>(p);
  return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                     __uint_as_float(x.y & 0xffff0000u));
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __hip_bfloat16* p) { return __bfloat162float(*p); }
// tokens v .. v + 3, -inf past the end
template <typename T>
__device__ __forceinline__ float4 logits4(const T* x, int v, int end) {
  float4 f = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
  if (v + 3 < end) {
    f = load4(x + v);
  } else {
    if (v < end) f.x = load1(x + v);
    if (v + 1 < end) f.y = load1(x + v + 1);
    if (v + 2 < end) f.z = load1(x + v + 2);
  }
  return make_float4(clean(f.x), clean(f.y), clean(f.z), clean(f.w));
}
__device__ __forceinline__ float get(const float4& f, int i) { return i == 0 ? f.x : i == 1 ? f.y : i == 2 ? f.z : f.w; }
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

// ---- a row's settings ------------------------------------------------------------------------------

struct Settings {
  double to_log2;            // log2(e) / temperature
  float temperature, top_p, min_p, per_bin;              // per_bin: bins to a unit of the logits, a power of two
  int k;
  __device__ __forceinline__ Settings(const SampleParams& p, int r) {
    temperature = p.temperature ? p.temperature[r] : 1.f;
    k = p.top_k ? p.top_k[r] : 0;
    top_p = p.top_p ? p.top_p[r] : 1.f;
    min_p = p.min_p ? p.min_p[r] : 0.f;
    if (!(temperature > 0.f)) {
      temperature = 1.f;
      k = 1;
    }
    if (k >= p.V || k < 0) k = 0;
    if (!(top_p < 1.f)) top_p = 1.f;
    if (!(min_p > 0.f)) min_p = 0.f;
    to_log2 = kLog2e / (double)temperature;
    // a bin is 1/32 of a logit wide, and of the temperature's power of two if that is lower (down to 2^-20): the 1023 bins reach 32
    // logits, or 32 to 64 temperatures' worth, below the maximum
    const int e = min(0, max(-15, (int)((__float_as_uint(temperature) >> 23) & 255) - 127));
    per_bin = __uint_as_float((uint32_t)(127 + 5 - e) << 23);
  }
  __device__ __forceinline__ bool filtered() const { return k > 0 || top_p < 1.f || min_p > 0.f; }
  // monotone, exact: a whole number
  __device__ __forceinline__ float bin_of(float x) const { return floorf(fminf(fmaxf(x, -1e30f), 1e30f) * per_bin); }
  __device__ __forceinline__ uint32_t least_key(float top) const {
    if (min_p == 0.f) return 0;
    const double least = (double)top + (double)temperature * log((double)min_p);
    float f = (float)least;
    if ((double)f < least) f = nextafterf(f, INFINITY);
    return score_key(fminf(f, top));
  }
};

// ---- weights ---------------------------------------------------------------------------------------

// table[i] = 2^(i / 64) 2^43
__device__ __forceinline__ void fill_table(double* table) {
  if (threadIdx.x < kTable) table[threadIdx.x] = exp2((double)threadIdx.x / kTable + kFraction);
}
// 2^((x - top) to_log2), times 2^43, as a number whose rounding is left to the caller
__device__ __forceinline__ double weight_real(float x, double top, double to_log2, const double* table) {
  const double t = fmax(((double)x - top) * to_log2, -1200.0);
  const double n = rint(t * kTable);
  const float r = (float)(t - n * (1.0 / kTable)) * 0.69314718055994530942f;
  const float q = r * (1.f + r * (0.5f + r * (1.f / 6.f)));
  const int k = (int)n;
  const double w = table[k & (kTable - 1)];
  return ldexp(__builtin_fma(w, (double)q, w), k >> 6);
}
__device__ __forceinline__ uint64_t weight(float x, double top, double to_log2, const double* table) {
  constexpr double kShift = 4503599627370496.0;          // 2^52: the sum's low bits are the rounded whole number
  const double w = weight_real(x, top, to_log2, table) + kShift;
  return __builtin_bit_cast(uint64_t, w) - __builtin_bit_cast(uint64_t, kShift);
}
// from a slice's maximum to the row's
__device__ __forceinline__ double factor_of(float top, float row_top, double to_log2) {
  return top == -INFINITY ? 0.0 : exp2(fmax(((double)top - (double)row_top) * to_log2, -1000.0));
}
__device__ __forceinline__ uint64_t scaled(uint64_t mass, double factor) { return (uint64_t)((double)mass * factor); }
// the weight that the kept tokens reach, of `mass`
__device__ __forceinline__ uint64_t limit_of(float top_p, uint64_t mass) {
  const double share = ceil((double)top_p * (double)mass);
  return share < 1.0 ? 1 : (uint64_t)share;
}

// ---- sums over a wavefront and a workgroup ---------------------------------------------------------

__device__ __forceinline__ uint64_t shfl_up64(uint64_t x, int d) { return __shfl_up((unsigned long long)x, d, 64); }
__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) x += __shfl_xor((unsigned long long)x, d, 64);
  return x;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t y = shfl_up64(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
// inclusive; every thread also gets the total.  sh: kWaves words, free when the call begins
__device__ __forceinline__ uint64_t block_scan64(uint64_t x, uint64_t* sh, uint64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_scan64(x, lane);
  if (lane == 63) sh[wave] = x;
  __syncthreads();
  uint64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = total;
    total += sh[w];
  }
  __syncthreads();
  return before + x;
}
__device__ __forceinline__ float block_max(float x, float* sh) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) x = fmaxf(x, __shfl_xor(x, d, 64));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x = fmaxf(x, sh[w]);
  __syncthreads();
  return x;
}

// ---- stats -----------------------------------------------------------------------------------------

// grid: (slices, rows).  EPT: logits of a thread, four at a time
template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void sample_stats_kernel(SampleParams p) {
  __shared__ unsigned long long mass[kBins];
  __shared__ uint32_t count[kBins];
  __shared__ double table[kTable];
  __shared__ float shf[kWaves];
  __shared__ uint64_t sh[kWaves];
  const int tid = threadIdx.x, s = blockIdx.x, r = blockIdx.y;
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  const int v0 = s * p.slice, end = min(v0 + p.slice, p.V);
  float4 f[EPT / 4];
#pragma unroll
  for (int i = 0; i < EPT / 4; ++i) f[i] = logits4(x, v0 + 4 * (i * kThreads + tid), end);
  const Settings set(p, r);
  fill_table(table);
  mass[tid] = 0;
  count[tid] = 0;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < EPT / 4; ++i) top = fmaxf(top, fmaxf(fmaxf(f[i].x, f[i].y), fmaxf(f[i].z, f[i].w)));
  top = block_max(top, shf);
  const int64_t at = (int64_t)r * p.slices + s;
  uint64_t total = 0;
  uint32_t n = 0;
  const bool filtered = set.filtered();
  if (top > -INFINITY) {
    const float first = set.bin_of(top);
    uint64_t rest = 0;
#pragma unroll
    for (int i = 0; i < EPT / 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float l = get(f[i], e);
        if (l == -INFINITY) continue;
        const uint64_t w = weight(l, (double)top, set.to_log2, table);
        const float b = first - set.bin_of(l);
        if (filtered && b < kBins - 1) {
          atomicAdd(&mass[(int)b], (unsigned long long)w);
          atomicAdd(&count[(int)b], 1u);
        } else {
          rest += w;
          ++n;
        }
      }
    if (filtered) {
      rest = wave_sum64(rest);
#pragma unroll
      for (int d = 32; d > 0; d /= 2) n += __shfl_xor(n, d, 64);
      if ((tid & 63) == 0) {
        atomicAdd(&mass[kBins - 1], (unsigned long long)rest);
        atomicAdd(&count[kBins - 1], n);
      }
      __syncthreads();
      rest = mass[tid];
      n = count[tid];
    }
    block_scan64(rest, sh, total);
  }
  if (filtered) {
    p.mass[at * kBins + tid] = top > -INFINITY ? mass[tid] : 0;
    p.count[at * kBins + tid] = n;
    uint64_t all;
    block_scan64(n, sh, all);
    n = (uint32_t)all;
  }
  if (tid == 0) {
    p.stats[at].top = top;
    p.stats[at].n = (int)n;
    p.stats[at].total = total;
  }
}

// ---- gather ----------------------------------------------------------------------------------------

constexpr int kMostSlices = 128;

// Bins of the row, counted from its maximum's bin: `shift` bins of a slice further down than the slice's own.
__device__ __forceinline__ int shift_of(const Settings& set, float top, float row_top) {
  return top == -INFINITY ? kBins : (int)fminf(set.bin_of(row_top) - set.bin_of(top), (float)kBins);
}

// grid: (slices, rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_gather_kernel(SampleParams p) {
  __shared__ uint64_t sh[kWaves];
  __shared__ float tops[kMostSlices];
  __shared__ double factor[kMostSlices];
  __shared__ int shift[kMostSlices];
  __shared__ int k_bin, p_bin;
  __shared__ uint64_t upto_n, bin_n, above_m;
  __shared__ uint32_t used;
  const int tid = threadIdx.x, s = blockIdx.x, r = blockIdx.y;
  const Settings set(p, r);
  const int64_t row = (int64_t)r * p.slices;
  if (tid < p.slices) tops[tid] = p.stats[row + tid].top;
  if (tid == 0) {
    k_bin = p_bin = kBins - 1;
    used = 0;
    upto_n = bin_n = above_m = 0;
  }
  __syncthreads();
  float top = -INFINITY;
  for (int i = 0; i < p.slices; ++i) top = fmaxf(top, tops[i]);
  if (!set.filtered() || top == -INFINITY) {
    if (s == 0 && tid == 0) p.plan[r] = RowPlan{top, kEverything, 0, 0, 0, 0};
    return;
  }
  uint64_t sum = 0, some = 0, total, n_finite;
  if (tid < p.slices) {
    factor[tid] = factor_of(tops[tid], top, set.to_log2);
    shift[tid] = shift_of(set, tops[tid], top);
    sum = scaled(p.stats[row + tid].total, factor[tid]);
    some = (uint32_t)p.stats[row + tid].n;
  }
  block_scan64(sum, sh, total);
  block_scan64(some, sh, n_finite);
  const int k = (uint64_t)set.k < n_finite ? set.k : 0;
  if (k == 0 && set.top_p == 1.f && set.min_p == 0.f) {
    if (s == 0 && tid == 0) p.plan[r] = RowPlan{top, kEverything, 0, 0, 0, 0};
    return;
  }
  // thread b: bin b of the row
  uint64_t m = 0, n = 0, all;
  if (tid < kBins - 1)
    for (int i = 0; i < p.slices; ++i) {
      const int b = tid - shift[i];
      if (b < 0) continue;
      n += p.count[(row + i) * kBins + b];
      m += scaled(p.mass[(row + i) * kBins + b], factor[i]);
    }
  const uint64_t n_upto = block_scan64(n, sh, all), m_upto = block_scan64(m, sh, all);
  const uint64_t limit = limit_of(set.top_p, total);
  if (k > 0) {
    if (n_upto >= (uint64_t)k && n_upto - n < (uint64_t)k) k_bin = tid;
  } else if (set.top_p < 1.f) {
    if (m_upto >= limit && m_upto - m < limit) p_bin = tid;
  }
  __syncthreads();
  int hi = k > 0 ? k_bin : p_bin;
  if (k == 0 && set.min_p > 0.f) {
    const float b = set.bin_of(top) - set.bin_of(key_logit(set.least_key(top)));
    const int m_bin = (int)fminf(b, (float)(kBins - 1));
    hi = set.top_p < 1.f ? min(hi, m_bin) : m_bin;
  }
  const int lo = k > 0 ? 0 : hi;
  if (tid == hi) {
    upto_n = n_upto;
    bin_n = n;
    above_m = m_upto - m;
  }
  __syncthreads();
  const uint64_t listed = k > 0 ? upto_n : bin_n;
  const bool slow = hi == kBins - 1 || listed > kList;
  if (s == 0 && tid == 0)
    p.plan[r] = RowPlan{top, slow ? kSlow : kFromList, (int)listed, k, limit, k > 0 ? 0 : above_m};
  if (slow) return;
  // this slice's tokens in the list's bins and above them, and those of the slices in front of it
  uint64_t front_mine = 0, above = 0;
  if (tid >= lo && tid <= hi)
    for (int i = 0; i <= s; ++i) {
      const int b = tid - shift[i];
      if (b < 0) continue;
      const uint64_t c = p.count[(row + i) * kBins + b];
      front_mine += i == s ? c << 32 : c;
    }
  if (tid < lo - shift[s]) above = p.mass[(row + s) * kBins + tid];
  uint64_t counts;
  block_scan64(front_mine, sh, counts);
  block_scan64(above, sh, all);
  if (tid == 0) p.stats[row + s].above = all;
  if ((counts >> 32) == 0) return;
  uint64_t* const list = p.list + (int64_t)r * kList;
  const uint32_t list_at = (uint32_t)counts;             // (the histogram's count of what this slice adds)
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  const int end = min((s + 1) * p.slice, p.V);
  const float first = set.bin_of(top);
  for (int v = s * p.slice + 4 * tid; v < end; v += 4 * kThreads) {
    const float4 f = logits4(x, v, end);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float l = get(f, e);
      if (l == -INFINITY) continue;
      const float b = first - set.bin_of(l);
      if (b >= (float)lo && b <= (float)hi) {
        const uint32_t to = list_at + atomicAdd(&used, 1u);
        if (to < kList) list[to] = ((uint64_t)~score_key(l) << 32) | (uint32_t)(v + e);
      }
    }
  }
}

// ---- draw ------------------------------------------------------------------------------------------

// Radix selection over the whole row: the largest key such that the tokens with keys above it have less than `limit` (of count, or
// weight) and those with it and above have at least that; `before`: what those above have.
template <typename T, bool WEIGHT>
__device__ uint32_t select_key(const T* x, int V, float top, double to_log2, const double* table, uint64_t limit,
                               unsigned long long* hist, uint64_t* sh, uint64_t& before) {
  uint32_t prefix = 0;
  before = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t hi_mask = shift == 24 ? 0u : (0xffffffffu << (shift + 8));
    for (int v = threadIdx.x; v < V; v += kThreads) {
      const float f = clean(load1(x + v));
      const uint32_t key = score_key(f);
      if ((key & hi_mask) == prefix)
        atomicAdd(&hist[(key >> shift) & 255], WEIGHT ? (unsigned long long)weight(f, (double)top, to_log2, table) : 1ull);
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

// The border of a row from all its logits.
template <typename T>
__device__ void slow_border(const T* x, int V, const Settings& set, int k, float top, const double* table, unsigned long long* hist,
                            uint64_t* sh, uint32_t& key, int& index) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  key = 0;
  uint64_t ties = (uint64_t)V, before;
  if (k > 0) {
    key = select_key<T, false>(x, V, top, set.to_log2, table, (uint64_t)k, hist, sh, before);
    ties = (uint64_t)k - before;
  }
  if (set.top_p < 1.f) {
    uint64_t mass = 0, same = 0, all;
    for (int v = tid; v < V; v += kThreads) {
      const float f = clean(load1(x + v));
      const uint32_t kf = score_key(f);
      if (kf > key) mass += weight(f, (double)top, set.to_log2, table);
      same += kf == key;
    }
    block_scan64(mass, sh, all);
    mass = all;
    block_scan64(same, sh, all);
    if (k > 0) mass += min(ties, all) * weight(key_logit(key), (double)top, set.to_log2, table);
    const uint64_t limit = limit_of(set.top_p, mass);
    const uint32_t at = select_key<T, true>(x, V, top, set.to_log2, table, limit, hist, sh, before);
    const uint64_t w = weight(key_logit(at), (double)top, set.to_log2, table);
    const uint64_t n = w == 0 ? (uint64_t)V : (limit - before + w - 1) / w;
    if (at > key) {
      key = at;
      ties = n;
    } else {
      ties = min(ties, n);
    }
  }
  const uint32_t least = set.least_key(top);
  if (least > key) {
    key = least;
    ties = (uint64_t)V;
  }
  // the index of the last tied token that stays: the wavefronts take consecutive shares
  const int share = (V + kWaves * 64 - 1) / (kWaves * 64) * 64, v0 = min(wave * share, V), v1 = min(v0 + share, V);
  uint64_t same = 0;
  for (int v = v0 + lane; v < v1; v += 64) same += score_key(clean(load1(x + v))) == key;
  same = wave_sum64(same);
  if (lane == 0) sh[wave] = same;
  if (tid == 0) hist[0] = (unsigned long long)V;
  __syncthreads();
  uint64_t seen = 0;
  for (int w = 0; w < wave; ++w) seen += sh[w];
  if (seen < ties && ties <= seen + same)
    for (int v = v0; v < v1; v += 64) {
      const uint64_t tied = __ballot(v + lane < v1 && score_key(clean(load1(x + min(v + lane, V - 1)))) == key);
      if ((tied >> lane & 1) && seen + __popcll(tied & ((1ull << lane) - 1)) + 1 == ties) hist[0] = (unsigned long long)(v + lane);
      seen += __popcll(tied);
    }
  __syncthreads();
  index = (int)hist[0];
  __syncthreads();
}

// grid: (rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleParams p) {
  __shared__ uint64_t list[kList];
  __shared__ double table[kTable];
  __shared__ uint64_t sh[kWaves];
  __shared__ float tops[kMostSlices];
  __shared__ double factor[kMostSlices];
  __shared__ unsigned long long kept[kMostSlices];       // weight that a slice keeps, relative to its maximum
  __shared__ int at_slice;
  __shared__ uint64_t in_slice, row_total;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x;
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  const RowPlan plan = p.plan[r];
  const float top = plan.top;
  if (top == -INFINITY) {
    if (tid == 0) {
      if (p.tokens) p.tokens[r] = -1;
      p.border[r] = Border{0xffffffffu, -1, 0.0};
    }
    return;
  }
  const Settings set(p, r);
  fill_table(table);
  if (tid < p.slices) {
    const SliceStats st = p.stats[(int64_t)r * p.slices + tid];
    tops[tid] = st.top;
    factor[tid] = factor_of(st.top, top, set.to_log2);
    kept[tid] = plan.how == kEverything ? st.total : plan.how == kFromList ? st.above : 0;
  }
  uint32_t key = 0;
  int index = p.V;
  if (plan.how == kFromList) {
    const int n = plan.listed;
    int n2 = 64;
    while (n2 < n) n2 *= 2;
    for (int i = tid; i < n2; i += kThreads) list[i] = i < n ? p.list[(int64_t)r * kList + i] : ~0ull;
    __syncthreads();
    for (int size = 2; size <= n2; size *= 2)
      for (int step = size / 2; step > 0; step /= 2) {
        for (int i = tid; i < n2 / 2; i += kThreads) {
          const int a = 2 * i - (i & (step - 1)), b = a + step;
          const uint64_t xa = list[a], xb = list[b];
          if ((xa > xb) == ((a & size) == 0)) {
            list[a] = xb;
            list[b] = xa;
          }
        }
        __syncthreads();
      }
    const auto weight_at = [&](int i) -> uint64_t {
      return i < n ? weight(key_logit(~(uint32_t)(list[i] >> 32)), (double)top, set.to_log2, table) : 0;
    };
    const int n_k = plan.k > 0 ? min(plan.k, n) : n;
    uint64_t limit = plan.limit, all;
    if (plan.k > 0 && set.top_p < 1.f) {
      uint64_t w = 0;
      for (int i = tid; i < n_k; i += kThreads) w += weight_at(i);
      block_scan64(w, sh, all);
      limit = limit_of(set.top_p, all);
    }
    const uint32_t least = set.least_key(top);
    uint64_t before = plan.above, stay = 0;
    for (int i0 = 0; i0 < n_k; i0 += kThreads) {
      const int i = i0 + tid;
      const uint64_t w = weight_at(i);
      const uint64_t upto = before + block_scan64(w, sh, all);
      stay += i < n_k && (set.top_p == 1.f || upto - w < limit) && ~(uint32_t)(list[min(i, n2 - 1)] >> 32) >= least;
      before += all;
    }
    block_scan64(stay, sh, all);
    const int kept_n = (int)all;
    if (kept_n > 0) {
      key = ~(uint32_t)(list[kept_n - 1] >> 32);
      index = (int)(uint32_t)list[kept_n - 1];
    } else {
      key = least;
    }
    for (int i = tid; i < kept_n; i += kThreads) {
      const int s = (int)(uint32_t)list[i] / p.slice;
      atomicAdd(&kept[s], (unsigned long long)weight(key_logit(~(uint32_t)(list[i] >> 32)), (double)tops[s], set.to_log2, table));
    }
  }
  __syncthreads();
  if (plan.how == kSlow) {
    slow_border<T>(x, p.V, set, plan.k, top, table, reinterpret_cast<unsigned long long*>(list), sh, key, index);
    for (int s = 0; s < p.slices; ++s) {
      if (tops[s] == -INFINITY) continue;
      uint64_t w = 0, all;
      for (int v = s * p.slice + tid; v < min((s + 1) * p.slice, p.V); v += kThreads) {
        const float f = clean(load1(x + v));
        const uint32_t kf = score_key(f);
        if (kf > key || (kf == key && v <= index)) w += weight(f, (double)tops[s], set.to_log2, table);
      }
      block_scan64(w, sh, all);
      if (tid == 0) kept[s] = all;
    }
    __syncthreads();
  }
  // the target, and the slice it falls in
  if (tid == 0) {
    uint64_t total = 0;
    for (int s = 0; s < p.slices; ++s) total += scaled(kept[s], factor[s]);
    row_total = total;
    const double t = p.tokens ? (double)p.u[r] * (double)total : 0.0;
    uint64_t target = t > 0.0 ? (uint64_t)t : 0;
    target = min(target, total - 1);
    int s = 0;
    for (; s < p.slices - 1; ++s) {
      const uint64_t m = scaled(kept[s], factor[s]);
      if (target < m) break;
      target -= m;
    }
    at_slice = s;
    in_slice = target;
    p.border[r] = Border{key, index, 1.0 / (double)total};
  }
  __syncthreads();
  if (!p.tokens) return;
  // the token: the wavefronts take consecutive shares of the slice
  const int s = at_slice, end = min((s + 1) * p.slice, p.V), share = p.slice / kWaves, v0 = s * p.slice + wave * share;
  const float slice_top = tops[s];
  const double f_s = factor[s];
  const uint64_t target = in_slice;
  const auto kept_weights = [&](int v, uint64_t (&w)[4]) {
    const float4 f = logits4(x, v, end);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float l = get(f, e);
      const uint32_t kf = score_key(l);
      w[e] = l > -INFINITY && (kf > key || (kf == key && v + e <= index)) ? weight(l, (double)slice_top, set.to_log2, table) : 0;
    }
  };
  uint64_t sum = 0;
  for (int v = v0 + 4 * lane; v < min(v0 + share, end); v += 256) {
    uint64_t w[4];
    kept_weights(v, w);
    sum += (w[0] + w[1]) + (w[2] + w[3]);
  }
  sum = wave_sum64(sum);
  if (lane == 0) sh[wave] = sum;
  __syncthreads();
  uint64_t run = 0;
  for (int w = 0; w < wave; ++w) run += sh[w];
  if (scaled(run, f_s) > target || !(scaled(run + sum, f_s) > target)) return;
  for (int v = v0 + 4 * lane; v - 4 * lane < min(v0 + share, end); v += 256) {
    uint64_t w[4];
    kept_weights(v, w);
    const uint64_t mine = (w[0] + w[1]) + (w[2] + w[3]), upto = run + wave_scan64(mine, lane);
    const uint64_t hit = __ballot(scaled(upto, f_s) > target);
    if (hit) {
      if (lane == __builtin_ctzll(hit)) {
        uint64_t c = upto - mine;
        int e = 0;
        for (; e < 3; ++e) {
          c += w[e];
          if (scaled(c, f_s) > target) break;
        }
        p.tokens[r] = v + e;
      }
      return;
    }
    run = __shfl((unsigned long long)upto, 63, 64);
  }
}

// ---- probabilities ---------------------------------------------------------------------------------

// grid: (slices, rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_probs_kernel(SampleParams p) {
  __shared__ double table[kTable];
  const int tid = threadIdx.x, s = blockIdx.x, r = blockIdx.y;
  const Settings set(p, r);
  const Border border = p.border[r];
  const float top = p.plan[r].top;
  fill_table(table);
  __syncthreads();
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  float* const out = p.probs + (int64_t)r * p.V;
  const int end = min((s + 1) * p.slice, p.V);
  for (int v = s * p.slice + 4 * tid; v < end; v += 4 * kThreads) {
    const float4 f = logits4(x, v, end);
    float4_u w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float l = get(f, e);
      const uint32_t kf = score_key(l);
      const bool keep = l > -INFINITY && (kf > border.key || (kf == border.key && v + e <= border.index));
      w[e] = keep ? (float)(weight_real(l, (double)top, set.to_log2, table) * border.inv_total) : 0.f;
    }
    if (v + 3 < end) {
      *reinterpret_cast<float4_u*>(out + v) = w;
    } else {
      for (int e = 0; v + e < end; ++e) out[v + e] = w[e];
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------

// Tokens of a slice: as many workgroups as there are compute units, if the rows have that many slices of 4096.
int slice_of(int rows, int V) {
  const int wanted = std::max(1, 256 / rows), each = (V + wanted - 1) / wanted;
  int s = 4096;
  while (s < each && s < 32768) s *= 2;
  return s;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

struct Layout {
  int slice, slices;
  size_t stats, mass, count, list, plan, border, bytes;
  Layout(int rows, int V) {
    slice = slice_of(rows, V);
    slices = (V + slice - 1) / slice;
    const size_t n = (size_t)rows * slices;
    size_t off = 0;
    stats = off;
    off += align256(n * sizeof(SliceStats));
    mass = off;
    off += align256(n * kBins * sizeof(uint64_t));
    count = off;
    off += align256(n * kBins * sizeof(uint32_t));
    list = off;
    off += align256((size_t)rows * kList * sizeof(uint64_t));
    plan = off;
    off += align256((size_t)rows * sizeof(RowPlan));
    border = off;
    off += align256((size_t)rows * sizeof(Border));
    bytes = off;
  }
};

template <typename T>
hipError_t launch_sample(const SampleParams& p, hipStream_t st) {
  const dim3 grid((unsigned)p.slices, (unsigned)p.rows), block(kThreads);
  switch (p.slice) {
    case 4096: hipLaunchKernelGGL((sample_stats_kernel<T, 4>), grid, block, 0, st, p); break;
    case 8192: hipLaunchKernelGGL((sample_stats_kernel<T, 8>), grid, block, 0, st, p); break;
    case 16384: hipLaunchKernelGGL((sample_stats_kernel<T, 16>), grid, block, 0, st, p); break;
    default: hipLaunchKernelGGL((sample_stats_kernel<T, 32>), grid, block, 0, st, p); break;
  }
  hipLaunchKernelGGL(sample_gather_kernel<T>, grid, block, 0, st, p);
  hipLaunchKernelGGL(sample_draw_kernel<T>, dim3((unsigned)p.rows), block, 0, st, p);
  if (p.probs) hipLaunchKernelGGL(sample_probs_kernel<T>, grid, block, 0, st, p);
  return hipGetLastError();
}

}  // namespace

}  // namespace svf

extern "C" {

size_t svf_sample_workspace_bytes(int32_t rows, int32_t V) {
  if (rows < 1 || rows > 65535 || V < 1 || V > 524288) return 0;
  return svf::Layout(rows, V).bytes;
}

int svf_sample(const void* logits, int32_t dtype, int64_t logits_stride, int32_t rows, int32_t V,
               const float* temperature_or_null, const int32_t* top_k_or_null, const float* top_p_or_null,
               const float* min_p_or_null, const float* u_or_null, int32_t* tokens_or_null, float* probs_or_null,
               void* ws, size_t ws_bytes, void* stream) {
  if (dtype != SVF_F32 && dtype != SVF_BF16) return SVF_ERR_DTYPE;
  if (!logits || (u_or_null == nullptr) != (tokens_or_null == nullptr) || (!tokens_or_null && !probs_or_null)) return SVF_ERR_NULL;
  if (rows < 1 || rows > 65535 || V < 1 || V > 524288 || (logits_stride != 0 && logits_stride < V)) return SVF_ERR_SHAPE;
  const auto misaligned = [](const void* q, uintptr_t to) { return reinterpret_cast<uintptr_t>(q) % to != 0; };
  if (misaligned(logits, dtype == SVF_F32 ? 4 : 2) || misaligned(temperature_or_null, 4) || misaligned(top_k_or_null, 4) ||
      misaligned(top_p_or_null, 4) || misaligned(min_p_or_null, 4) || misaligned(u_or_null, 4) || misaligned(tokens_or_null, 4) ||
      misaligned(probs_or_null, 4))
    return SVF_ERR_SHAPE;
  if (!ws || misaligned(ws, 256) || ws_bytes < svf_sample_workspace_bytes(rows, V)) return SVF_ERR_WORKSPACE;
  const svf::Layout at(rows, V);
  char* const w = static_cast<char*>(ws);
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
  p.slice = at.slice;
  p.slices = at.slices;
  p.stats = reinterpret_cast<svf::SliceStats*>(w + at.stats);
  p.mass = reinterpret_cast<uint64_t*>(w + at.mass);
  p.count = reinterpret_cast<uint32_t*>(w + at.count);
  p.list = reinterpret_cast<uint64_t*>(w + at.list);
  p.plan = reinterpret_cast<svf::RowPlan*>(w + at.plan);
  p.border = reinterpret_cast<svf::Border*>(w + at.border);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return (dtype == SVF_F32 ? svf::launch_sample<float>(p, st) : svf::launch_sample<__hip_bfloat16>(p, st)) == hipSuccess
             ? SVF_OK : SVF_ERR_HIP;
}

}  // extern "C"
