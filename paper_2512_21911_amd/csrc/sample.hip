// Sampling from logits (svf_sample): temperature, top-k, top-p, min-p, and the draw by inversion.
//
// All three filters keep a prefix of the tokens in descending order of their logits (ties by index), so what a row keeps
// is two numbers, a border: the last kept logit and the index of the last kept token with it.  Nothing is sorted but the few tokens around it.
// A row is cut into slices of up to 32 768 logits, which a workgroup holds in registers, and three steps find border and token:
//   stats    of a slice: the maximum and the sum of the weights or, if the row has a filter, a histogram of counts and weights over 1024 bins of
//            logits from the maximum down (those further down are counted and weighed together).
//   gather   the row's histograms are added up, and the bin is known that the border is in; the tokens in it go to the row's list (top-k: all from
//            the top on, so that the mass that top-p takes its share of is at hand).
//   draw     the list is sorted and walked to the border, what every slice keeps is added up, and the token is found: by the
//            list alone if everything kept is in it, else in the one slice that the target falls in.
// A row of one slice has all three in one launch (32 000 logits, top-k and top-p: 16 us; in three launches over eight slices 19), longer rows in
// three: a workgroup per slice, per slice (which reads its slice again if it has tokens for the list), per row.  A fourth, with a workgroup per
// slice again, writes the probabilities where they are asked for.
// A row whose border bin has more tokens than the list (many equal logits, a top-k of thousands) is settled in the third step by
// radix selection over the whole row, by its one workgroup: equal logits with top-p 0.9 0.23 ms (32 000) and 0.66 (129 280), nearly equal ones 0.13 and 0.32, a
// top-k of 5000 0.10 and 0.26, with top-p 0.17 and 0.45.  Temperatures above two weigh what is below the bins in fp64: 33 us instead of 25 with top-p.
//
// Weights.  Bins are a power of two of logits wide, at whole multiples of it, so a logit's bin and its place in the bin are exact in fp32.  A
// weight is its bin's, 2^(-bin c) in fp64, times 2^(place c), place c < 0.046: a short polynomial in fp32 whose rounding is 2^-24 of the
// excess over one.  That is good to 2^-27, which an fp32 exponential of the whole argument is not (2^-20 at 20 below the maximum), and a hundred
// thousand tokens' borders wait for the target in between; and a histogram adds whole numbers, count and weight in one 64-bit word, so that
// the order of the adding does not matter.
// Bound: for few rows by the steps' chains of barriers and reads (10 us for 4000 logits); for many by the vector instructions of the first step
// (256 rows of 129 280 in bf16: 31 us, 66 MB), the second's (29 us), and one workgroup a row in the third (20 us); the probabilities, 198 MB, take 40 us.
#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <type_traits>

#include "svf_device.h"
#include "svf_rules.h"

namespace svf {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kFraction = 43;                            // bits of a weight behind the point; 2^19 weights of 1.05 fit 63 bits
constexpr int kPlaceBits = 31;                           // of a weight relative to its bin's: at least one, below two
constexpr int kCountAt = 47;                             // a histogram's word: what 2^15 such weights have over one, and above that how many
constexpr int kBins = 1024;                              // from the maximum's down; logits further down are in none
constexpr int kList = 4096;                              // tokens around the border that are sorted
constexpr float kFar = 1.5e38f;                          // bins of logits further from zero are this one (twice as many have a number)
constexpr double kLog2e = 1.4426950408889634074;

struct SliceStats {
  float top;                 // largest logit; -inf: the slice has none above that
  int32_t n;                 // logits above -inf (rows with a filter)
  uint64_t total;            // weight of all of them, relative to the bin of top
  uint64_t above;            // weight that the slice keeps without those in the list, relative to the row's first bin
};
enum { kEverything, kFromList, kSlow };                  // how the border is found
struct RowPlan {
  float top;
  int32_t how, listed, k;    // k: top-k, 0 if it drops nothing
  uint64_t limit, above;     // without top-k: the weight that the kept tokens reach, and what is above the list's bin
};
struct Border {              // of what a row keeps: logits above `least`, and those with it up to `index`
  float least;
  int32_t index;
  double inv_total;          // 1 / their total weight
  // (NaN is kept by no comparison; +inf is the largest finite number)
  __device__ __forceinline__ bool keeps(float& l, int v) const {
    l = l > 3.402823466e38f ? 3.402823466e38f : l;
    return l > least || (l == least && v <= index);
  }
};

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
  uint64_t* bins;            // [rows][slices][kBins]: count << kCountAt | what the weights, relative to the bin's, have over one
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
  if (v < end) f.x = load1(x + v);
  if (v + 1 < end) f.y = load1(x + v + 1);
  if (v + 2 < end) f.z = load1(x + v + 2);
  if (v + 3 < end) f.w = load1(x + v + 3);
  return f;
}
// Tokens v0 + 4 (i THREADS + thread) .. + 3 of all i < N.  Whether all threads' are inside the row is the same for the workgroup, and then the
// loads are under no mask: under one they wait for each other (16.9 us instead of 16.1 for the first launch at 64 rows of 129 280).
template <int N, int THREADS, typename T>
__device__ __forceinline__ void read_logits(const T* x, int v0, int thread, int end, float4 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int v = v0 + 4 * i * THREADS;
    if (v + 4 * THREADS <= end) f[i] = load4(x + v + 4 * thread);
    else f[i] = logits4(x, v + 4 * thread, end);
  }
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float get(const float4& f, int i) { return i == 0 ? f.x : i == 1 ? f.y : i == 2 ? f.z : f.w; }

// the smallest fp32 number that is no less
__device__ __forceinline__ float at_least(double x) {
  const float f = (float)x;
  return (double)f < x ? nextafterf(f, INFINITY) : f;
}

// ---- a row's settings ------------------------------------------------------------------------------

struct Settings {
  float temperature, top_p, min_p, per_bin;              // per_bin: bins to a unit of the logits, a power of two
  double bin_log2;           // log2 of the weight from one bin to the next
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
    temperature = fmaxf(temperature, 0x1p-60f);
    if (k >= p.V || k < 0) k = 0;
    if (!(top_p < 1.f)) top_p = 1.f;
    if (!(min_p > 0.f)) min_p = 0.f;
    // a bin is 1/32 of a logit wide, and of the temperature's power of two if that is lower: the 1024 bins reach 32 logits, or 16
    // to 32 temperatures, below the maximum
    const int e = min(0, (int)((__float_as_uint(temperature) >> 23) & 255) - 127);
    per_bin = __uint_as_float((uint32_t)(127 + 5 - e) << 23);
    bin_log2 = kLog2e / (double)temperature / (double)per_bin;
  }
  __device__ __forceinline__ bool filtered() const { return k > 0 || top_p < 1.f || min_p > 0.f; }
  // the bin's number (from the logits' zero up; whole) and the place in it, 0 <= place < 1: both exact
  __device__ __forceinline__ float bin_of(float x, float& place) const {
    const float at = __builtin_amdgcn_fmed3f(x * per_bin, -kFar, kFar), b = floorf(at);   // (x is no NaN)
    place = at - b;
    return b;
  }
  __device__ __forceinline__ float bin_of(float x) const {
    float place;
    return bin_of(x, place);
  }
  __device__ __forceinline__ uint32_t least_key(float top) const {
    if (min_p == 0.f) return 0;
    const double least = (double)top + (double)temperature * log((double)min_p);
    return score_key(fminf(at_least(least), top));
  }
};

// ---- weights ---------------------------------------------------------------------------------------

// 2^(place bin_log2) - 1 times `scale`: x + x^2/2 + x^3/6 + x^4/24, x = place z, z = bin_log2 ln 2 <= 1/32, with the last term, on 0 <= place < 1, by
// the cubic that Chebyshev's polynomial of degree four leaves (without its constant: no excess at place 0), 2^-30 of the weight at most.
struct PlaceExcess {
  float c1, c2, c3;
  __device__ __forceinline__ explicit PlaceExcess(const Settings& set, float scale = 1.f) {
    const float z = (float)(set.bin_log2 * 0.69314718055994530942), x1 = z * scale, x2 = x1 * z * 0.5f, x3 = x2 * z * (1.f / 3.f), x4 = x3 * z * 0.25f;
    c1 = x1 + 0.25f * x4;
    c2 = x2 - 1.25f * x4;
    c3 = x3 + 2.f * x4;
  }
  __device__ __forceinline__ float operator()(float place) const { return place * (c1 + place * (c2 + place * c3)); }
};
// 2^(place bin_log2) in fixed point; of an excess scaled by kPlaceOne
constexpr float kPlaceOne = (float)(1u << kPlaceBits);
__device__ __forceinline__ uint32_t place_weight(float place, const PlaceExcess& excess) { return (1u << kPlaceBits) + (uint32_t)excess(place); }
// 2^t, t <= 0: ten terms of the series around the nearest whole number, 2^-36 relative
__device__ __forceinline__ double exp2_series(double t) {
  t = fmax(t, -1200.0);
  const double n = rint(t), x = (t - n) * 0.69314718055994530942;
  double y = 1.0 / 362880;
  y = __builtin_fma(y, x, 1.0 / 40320);
  y = __builtin_fma(y, x, 1.0 / 5040);
  y = __builtin_fma(y, x, 1.0 / 720);
  y = __builtin_fma(y, x, 1.0 / 120);
  y = __builtin_fma(y, x, 1.0 / 24);
  y = __builtin_fma(y, x, 1.0 / 6);
  y = __builtin_fma(y, x, 0.5);
  y = __builtin_fma(y, x, 1.0);
  y = __builtin_fma(y, x, 1.0);
  return ldexp(y, (int)n);
}
// weight of the lower end of the bin that lies b bins (a whole number, any size) below the first
__device__ __forceinline__ double bin_weight(float b, const Settings& set) { return exp2_series(-(double)b * set.bin_log2); }
// Below the 1024 bins a weight is e^-16 and less at temperatures up to two, and all of a row's together 0.06 of the row's at most (2^19 tokens): an
// fp32 exponential of the whole argument does, good to 2^-18.
__device__ __forceinline__ bool rest_is_small(const Settings& set) { return set.temperature <= 2.f; }
__device__ __forceinline__ float small_rest(float below, float bin_log2) { return __builtin_amdgcn_exp2f(bin_log2 * -below); }
constexpr double kPlaceToRow = (double)(1u << (kFraction - kPlaceBits));

// All weights of a row, relative to the bin of its maximum: table[b] = bin_weight(b) 2^(kFraction - kPlaceBits)
struct Weights {
  const double* table;
  float first;
  PlaceExcess excess;
  __device__ __forceinline__ Weights(const Settings& set, float top, const double* t)
      : table(t), first(set.bin_of(top)), excess(set, kPlaceOne) {}
  __device__ __forceinline__ uint64_t operator()(const Settings& set, float x) const {
    if (x == -INFINITY) return 0;
    float place;
    const float b = first - set.bin_of(x, place);
    constexpr double kShift = 4503599627370496.0;        // 2^52: the sum's low bits are the rounded whole number
    double w;
    if (b < (float)kBins) w = __builtin_fma(table[(int)b], (double)place_weight(place, excess), kShift);
    else if (rest_is_small(set)) w = __builtin_fma((double)small_rest(b - place, (float)set.bin_log2), (double)(1ull << kFraction), kShift);
    else w = __builtin_fma(bin_weight(b, set) * kPlaceToRow, (double)place_weight(place, excess), kShift);
    return __builtin_bit_cast(uint64_t, w) - __builtin_bit_cast(uint64_t, kShift);
  }
};
// the weight that the kept tokens reach, of `mass`
__device__ __forceinline__ uint64_t limit_of(float top_p, uint64_t mass) {
  const double share = ceil((double)top_p * (double)mass);
  return share < 1.0 ? 1 : (uint64_t)share;
}

// ---- sums over a wavefront and a workgroup ---------------------------------------------------------

// (moves inside a row of sixteen lanes and from row to row: no trips through LDS)
template <int CTRL, int ROWS, bool BOUND>
__device__ __forceinline__ uint64_t lane_move64(uint64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, BOUND);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, BOUND);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t x) {
  x += lane_move64<0x111, 0xf, true>(x);    // row_shr:1
  x += lane_move64<0x112, 0xf, true>(x);    // row_shr:2
  x += lane_move64<0x114, 0xf, true>(x);    // row_shr:4
  x += lane_move64<0x118, 0xf, true>(x);    // row_shr:8
  x += lane_move64<0x142, 0xa, false>(x);   // row_bcast:15 -> rows 1, 3
  x += lane_move64<0x143, 0xc, false>(x);   // row_bcast:31 -> rows 2, 3
  return x;
}
__device__ __forceinline__ uint64_t lane64(uint64_t x, int l) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, l), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), l);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t x) { return lane64(wave_scan64(x), 63); }
// Inclusive scans of N numbers over the workgroup; every thread also gets the totals.  sh: N * kWaves words, free when the call begins.
template <int N>
__device__ __forceinline__ void block_scan64(uint64_t (&x)[N], uint64_t (&total)[N], uint64_t* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = wave_scan64(x[i]);
    if (lane == 63) sh[i * kWaves + wave] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint64_t upto = wave_scan64(lane < kWaves ? sh[i * kWaves + lane] : 0);
    total[i] = lane64(upto, kWaves - 1);
    if (wave > 0) x[i] += lane64(upto, __builtin_amdgcn_readfirstlane(wave) - 1);
  }
  __syncthreads();
}
__device__ __forceinline__ uint64_t block_scan64(uint64_t x, uint64_t* sh, uint64_t& total) {
  uint64_t a[1] = {x}, t[1];
  block_scan64<1>(a, t, sh);
  total = t[0];
  return a[0];
}
__device__ __forceinline__ float wave_max(float x) {
#define SVF_MAX(CTRL, ROWS) \
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, ROWS, 0xf, false)))
  SVF_MAX(0x111, 0xf);
  SVF_MAX(0x112, 0xf);
  SVF_MAX(0x114, 0xf);
  SVF_MAX(0x118, 0xf);
  SVF_MAX(0x142, 0xa);
  SVF_MAX(0x143, 0xc);
#undef SVF_MAX
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float block_max(float x, float* sh) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  x = wave_max((threadIdx.x & 63) < kWaves ? sh[threadIdx.x & 63] : -INFINITY);
  __syncthreads();
  return x;
}

// ---- stats -----------------------------------------------------------------------------------------

constexpr uint64_t kExcessMask = (1ull << kCountAt) - 1;
__device__ __forceinline__ uint32_t count_of(uint64_t word) { return (uint32_t)(word >> kCountAt); }
__device__ __forceinline__ uint64_t weight_of(uint64_t word) { return (word & kExcessMask) + ((uint64_t)count_of(word) << kPlaceBits); }

struct StatsShared {
  uint64_t bins[kBins];                                  // the histogram, or the bins' weights
  float shf[kWaves];
  uint64_t sums[2 * kWaves];
};
struct SliceFound {
  float top;
  uint64_t total;
  uint32_t n;
  uint64_t word;             // thread b: bin b
};

// By a workgroup, from its logits in registers (my_bin: bin_weight(thread); f: token 4 (i kThreads + thread) + e of x, which has n_x; NaN is among them still).
template <typename T, int EPT>
__device__ __forceinline__ SliceFound slice_stats(const Settings& set, double my_bin, const T* x, int n_x, const float4 (&f)[EPT / 4],
                                                  StatsShared& sh) {
  const int tid = threadIdx.x;
  const bool filtered = set.filtered();
  unsigned long long* const bins = reinterpret_cast<unsigned long long*>(sh.bins);
  double* const table = reinterpret_cast<double*>(sh.bins);
  if (filtered) bins[tid] = 0;
  else table[tid] = my_bin;
  SliceFound at;
  at.top = -INFINITY;
#pragma unroll
  for (int i = 0; i < EPT / 4; ++i) at.top = fmaxf(at.top, fmaxf(fmaxf(f[i].x, f[i].y), fmaxf(f[i].z, f[i].w)));
  at.top = fminf(block_max(at.top, sh.shf), 3.402823466e38f);
  const float first = set.bin_of(at.top), bin_log2 = (float)set.bin_log2;
  // Nearly always the bins' numbers are small, and no logit needs a bound: those of -inf and NaN are in no bin.
  const bool near = fabsf(first) < 0x1p30f, small = rest_is_small(set);
  double total = 0.0;
  float rest = 0.f;
  uint32_t n = 0;
  if (near) {
    const PlaceExcess excess(set, filtered ? kPlaceOne : 1.f);
    const float first8 = 8.f * first;
    const auto each = [&](auto&& in_bin) {
#pragma unroll
      for (int i = 0; i < EPT / 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l = get(f[i], e), bin = l * set.per_bin, b = floorf(bin), b8 = __builtin_fmaf(-8.f, b, first8);
          if (b8 < 8.f * (float)kBins) {
            in_bin((uint32_t)b8, excess(bin - b));
          } else if (l > -INFINITY) {
            rest += small_rest(first - bin, bin_log2);
            ++n;
          }
        }
    };
    if (filtered) each([&](uint32_t b8, float y) { atomicAdd(reinterpret_cast<unsigned long long*>(reinterpret_cast<char*>(bins) + b8), 1ull << kCountAt | (uint32_t)y); });
    else each([&](uint32_t b8, float y) { total = __builtin_fma(*reinterpret_cast<double*>(reinterpret_cast<char*>(table) + b8), 1.0 + (double)y, total); });
    if (!small) rest = 0.f;
  }
  if (at.top > -INFINITY && !(near && small)) {            // the rest, or all, in 64 bits, from the logits once more
    const PlaceExcess excess(set);
    for (int v = tid; v < n_x; v += kThreads) {
      const float l = clean(load1(x + v));
      float place;
      const float b = first - set.bin_of(l, place);
      if (l == -INFINITY) continue;
      if (b >= (float)kBins) {
        total += bin_weight(b, set) * (1.0 + (double)excess(place));
        if (!near) ++n;
      } else if (!near) {
        if (filtered) atomicAdd(&bins[(int)b], 1ull << kCountAt | (uint32_t)(excess(place) * kPlaceOne));
        else total += table[(int)b] * (1.0 + (double)excess(place));
      }
    }
  }
  total += (double)rest;
  at.word = 0;
  if (filtered) {
    __syncthreads();
    at.word = bins[tid];
    total += (double)weight_of(at.word) * (1.0 / (double)kPlaceOne) * my_bin;
    n += count_of(at.word);
  }
  const uint64_t mine = wave_sum64((uint64_t)(total * (double)(1ull << kFraction))), count = wave_sum64(n);
  const int lane = tid & 63;
  if (lane == 63) {
    sh.sums[tid >> 6] = mine;
    sh.sums[kWaves + (tid >> 6)] = count;
  }
  __syncthreads();
  at.total = wave_sum64(lane < kWaves ? sh.sums[lane] : 0);
  at.n = (uint32_t)wave_sum64(lane < kWaves ? sh.sums[kWaves + lane] : 0);
  return at;
}

// grid: (slices, rows).  EPT: logits of a thread, four at a time
template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void sample_stats_kernel(SampleParams p) {
  __shared__ StatsShared sh;
  const int tid = threadIdx.x, s = blockIdx.x, r = blockIdx.y;
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  const int v0 = s * p.slice, end = min(v0 + p.slice, p.V);
  float4 f[EPT / 4];
  read_logits<EPT / 4, kThreads>(x, v0, tid, end, f);
  const Settings set(p, r);
  const SliceFound found = slice_stats<T, EPT>(set, bin_weight((float)tid, set), x + v0, end - v0, f, sh);
  const int64_t at = (int64_t)r * p.slices + s;
  if (set.filtered()) p.bins[at * kBins + tid] = found.word;
  if (tid == 0) {
    p.stats[at].top = found.top;
    p.stats[at].n = (int)found.n;
    p.stats[at].total = found.total;
  }
}

// ---- gather ----------------------------------------------------------------------------------------

constexpr int kMostSlices = 128;
constexpr int kReadAhead = 4;                            // loads of a thread on their way

// Bins from the row's first down to the slice's first; kBins: none of the slice's is among the row's.
__device__ __forceinline__ int shift_of(const Settings& set, float top, float row_top) {
  return top == -INFINITY ? kBins : (int)fminf(set.bin_of(row_top) - set.bin_of(top), (float)kBins);
}
// a slice's total relative to the row's first bin, in fixed point
__device__ __forceinline__ uint64_t total_of(const SliceStats& st, const Settings& set, float row_top) {
  if (st.top == -INFINITY) return 0;
  return (uint64_t)((double)st.total * bin_weight(set.bin_of(row_top) - set.bin_of(st.top), set));
}

struct GatherShared {
  uint64_t scan[2 * kWaves];
  int bin;
  uint64_t listed, above;
  uint32_t used;
  __device__ __forceinline__ void clear() {
    bin = kBins;
    used = 0;
    listed = above = 0;
  }
};
struct Bins { int lo, hi; };                             // those whose tokens are in the list

// By a workgroup, thread b having bin b of the row (n tokens of weight m).  whole, count: the row's weight and its number of logits above -inf.
// sh: cleared, a barrier ago.
__device__ __forceinline__ RowPlan plan_row(const Settings& set, float top, uint64_t n, uint64_t m, uint64_t whole, uint32_t count,
                                            GatherShared& sh, Bins& list) {
  const int tid = threadIdx.x;
  const int k = (uint32_t)set.k < count ? set.k : 0;
  if (k == 0 && set.top_p == 1.f && set.min_p == 0.f) return RowPlan{top, kEverything, 0, 0, 0, 0};
  const uint64_t limit = limit_of(set.top_p, whole), x = k > 0 ? n : m, wanted = k > 0 ? (uint64_t)k : limit;
  uint64_t all;
  const uint64_t upto = block_scan64(x, sh.scan, all);
  if ((k > 0 || set.top_p < 1.f) && upto >= wanted && upto - x < wanted) sh.bin = tid;
  __syncthreads();
  // the border's bin; kBins: below them all
  list.hi = sh.bin;
  if (k == 0 && set.min_p > 0.f) {
    const int m_bin = (int)fminf(set.bin_of(top) - set.bin_of(key_logit(set.least_key(top))), (float)kBins);
    list.hi = min(list.hi, m_bin);
  }
  list.lo = k > 0 ? 0 : list.hi;
  if (tid == list.hi) {
    sh.listed = k > 0 ? upto : n;
    sh.above = k > 0 ? 0 : upto - x;
  }
  __syncthreads();
  const bool slow = list.hi == kBins || sh.listed > kList;
  return RowPlan{top, slow ? kSlow : kFromList, (int)sh.listed, k, limit, sh.above};
}

// The list's bins as logits, least <= l <= most; both are exact, a bin's end times a power of two or the next number inwards.
struct ListRange {
  float least, most;
  __device__ __forceinline__ ListRange(const Settings& set, float top, Bins list) {
    const double first = (double)set.bin_of(top), lower = first - list.hi, past = first - list.lo + 1;
    least = lower <= -(double)kFar ? -3.402823466e38f : at_least(lower / (double)set.per_bin);
    // (no logit is above the first bin; its end has no number where bins are counted past 2^53, and a list further down begins far below that)
    most = list.lo == 0 ? INFINITY : nextafterf(at_least(past / (double)set.per_bin), -INFINITY);
  }
  __device__ __forceinline__ bool has(float l) const { return l >= least && l <= most; }           // (never NaN)
};
__device__ __forceinline__ uint64_t listed(float l, int v) { return (uint64_t)~score_key(clean(l)) << 32 | (uint32_t)v; }

// grid: (slices, rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_gather_kernel(SampleParams p) {
  __shared__ GatherShared sh;
  const int tid = threadIdx.x, lane = tid & 63, s = blockIdx.x, r = blockIdx.y;
  const int64_t row = (int64_t)r * p.slices;
  // every wavefront by itself: lane l has slices l and l + 64
  SliceStats st[2] = {{-INFINITY, 0, 0, 0}, {-INFINITY, 0, 0, 0}};
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (lane + 64 * i < p.slices) st[i] = p.stats[row + lane + 64 * i];
  const Settings set(p, r);
  if (tid == 0) sh.clear();
  const float top = wave_max(fmaxf(st[0].top, st[1].top));
  const uint64_t whole[2] = {total_of(st[0], set, top), total_of(st[1], set, top)};
  const auto keeps_all = [&] {
    if (tid == (s & 63)) p.stats[row + s].above = s < 64 ? whole[0] : whole[1];
  };
  if (!set.filtered() || top == -INFINITY) {
    if (s == 0 && tid == 0) p.plan[r] = RowPlan{top, kEverything, 0, 0, 0, 0};
    keeps_all();
    return;
  }
  const int shift[2] = {shift_of(set, st[0].top, top), shift_of(set, st[1].top, top)};
  // thread b: bin b of the row (what slices hold further down is in none of them)
  uint64_t mine = 0, m = 0, n = 0, n_front = 0;            // mine: this slice's; n_front: of those in front of it
  for (int i0 = 0; i0 < p.slices; i0 += 4) {
    uint64_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = min(i0 + i, p.slices - 1), b = tid - __builtin_amdgcn_readlane(at < 64 ? shift[0] : shift[1], at & 63);
      w[i] = p.bins[(row + at) * kBins + max(b, 0)];
      if (b < 0 || i0 + i >= p.slices) w[i] = 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i0 + i == s) {
        n_front = n;
        mine = w[i];
      }
      n += count_of(w[i]);
      m += w[i] & kExcessMask;
    }
  }
  const double to_row = bin_weight((float)tid, set) * kPlaceToRow;
  m = (uint64_t)((double)(m + (n << kPlaceBits)) * to_row);
  Bins bins;
  __syncthreads();
  const RowPlan plan = plan_row(set, top, n, m, wave_sum64(whole[0] + whole[1]), (uint32_t)wave_sum64((uint32_t)(st[0].n + st[1].n)), sh, bins);
  if (s == 0 && tid == 0) p.plan[r] = plan;
  if (plan.how == kEverything) keeps_all();
  if (plan.how != kFromList) return;
  // this slice's tokens in the list's bins, those of the slices in front of it, and what it has above the list's bins
  const bool among = tid >= bins.lo && tid <= bins.hi;
  uint64_t parts[2] = {among ? (uint64_t)count_of(mine) << 32 | n_front : 0, tid < bins.lo ? (uint64_t)((double)weight_of(mine) * to_row) : 0}, of[2];
  block_scan64<2>(parts, of, sh.scan);
  if (tid == 0) p.stats[row + s].above = of[1];
  if ((of[0] >> 32) == 0) return;
  uint64_t* const list = p.list + (int64_t)r * kList;
  const uint32_t list_at = (uint32_t)of[0];              // (the slice adds as many as the histogram says)
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  const int end = min((s + 1) * p.slice, p.V);
  const ListRange range(set, top, bins);
  for (int v0 = s * p.slice; v0 < end; v0 += 4 * kReadAhead * kThreads) {
    float4 f[kReadAhead];
    read_logits<kReadAhead, kThreads>(x, v0, tid, end, f);
#pragma unroll
    for (int i = 0; i < kReadAhead; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (range.has(get(f[i], e))) {
          const uint32_t to = list_at + atomicAdd(&sh.used, 1u);
          if (to < kList) list[to] = listed(get(f[i], e), v0 + 4 * (i * kThreads + tid) + e);
        }
  }
}

// ---- draw ------------------------------------------------------------------------------------------

// Radix selection over the whole row: the largest key such that the tokens with keys above it have less than `limit` (of count, or
// weight) and those with it and above have at least that; `before`: what those above have.
template <typename T, bool WEIGHT>
__device__ uint32_t select_key(const T* x, int V, const Settings& set, const Weights& weight, uint64_t limit, unsigned long long* hist,
                               uint64_t* sh, uint64_t& before) {
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
        atomicAdd(&hist[(key >> shift) & 255], WEIGHT ? (unsigned long long)weight(set, f) : 1ull);
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
__device__ void slow_border(const T* x, int V, const Settings& set, int k, float top, const Weights& weight, unsigned long long* hist,
                            uint64_t* sh, uint32_t& key, int& index) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  key = 0;
  uint64_t ties = (uint64_t)V, before;
  if (k > 0) {
    key = select_key<T, false>(x, V, set, weight, (uint64_t)k, hist, sh, before);
    ties = (uint64_t)k - before;
  }
  if (set.top_p < 1.f) {
    uint64_t mass = 0, same = 0, all;
    for (int v = tid; v < V; v += kThreads) {
      const float f = clean(load1(x + v));
      const uint32_t kf = score_key(f);
      if (kf > key) mass += weight(set, f);
      same += kf == key;
    }
    block_scan64(mass, sh, all);
    mass = all;
    block_scan64(same, sh, all);
    if (k > 0) mass += min(ties, all) * weight(set, key_logit(key));
    const uint64_t limit = limit_of(set.top_p, mass);
    const uint32_t at = select_key<T, true>(x, V, set, weight, limit, hist, sh, before);
    const uint64_t w = weight(set, key_logit(at));
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

// One step of a bitonic network among a wavefront's lanes, and all steps from STEP down.
template <int STEP>
__device__ __forceinline__ uint64_t other_lane64(uint64_t x) {
  if constexpr (STEP == 1) return lane_move64<0xb1, 0xf, true>(x);                                    // quad_perm 1 0 3 2
  if constexpr (STEP == 2) return lane_move64<0x4e, 0xf, true>(x);                                    // quad_perm 2 3 0 1
  if constexpr (STEP == 4) return lane_move64<0x141, 0xf, true>(lane_move64<0x1b, 0xf, true>(x));     // a quad's, then eight lanes' order turned round
  if constexpr (STEP == 8) return lane_move64<0x128, 0xf, true>(x);                                   // row_ror:8
  return (uint64_t)__shfl_xor((unsigned long long)x, STEP, 64);
}
template <int STEP>
__device__ __forceinline__ void sort_step(uint64_t& x, int lane, bool up) {
  const uint64_t y = other_lane64<STEP>(x);
  if ((y < x) == (((lane & STEP) == 0) == up)) x = y;
}
template <int STEP>
__device__ __forceinline__ void sort_half(uint64_t& x, int lane, bool up) {
  sort_step<STEP>(x, lane, up);
  if constexpr (STEP > 1) sort_half<STEP / 2>(x, lane, up);
}
// Ascending.  Up to 256: every element's place is the number of those below it, counted by four threads each.  More: a bitonic network, whose
// steps of less than 64 are done in registers.
constexpr int kRanked = 256;
__device__ __forceinline__ void sort_list(uint64_t* list, int n, uint64_t* spare, uint32_t* rank) {
  const int tid = threadIdx.x;
  if (n <= kRanked) {
    const int i = tid & (kRanked - 1), part = tid / kRanked;
    if (tid < kRanked) rank[tid] = 0;
    __syncthreads();
    const int each = (n + 3) / 4;
    if (i < n) {
      const uint64_t mine = list[i];
      uint32_t below = 0;
      for (int j = part * each; j < min((part + 1) * each, n); ++j) below += list[j] < mine;
      atomicAdd(&rank[i], below);
    }
    __syncthreads();
    if (tid < n) spare[rank[tid]] = list[tid];
    __syncthreads();
    if (tid < n) list[tid] = spare[tid];
    __syncthreads();
    return;
  }
  int n2 = 2 * kRanked;
  while (n2 < n) n2 *= 2;
  for (int i = n + tid; i < n2; i += kThreads) list[i] = ~0ull;
  __syncthreads();
  const int lane = tid & 63, wave = tid >> 6;
  for (int g = wave; g < n2 / 64; g += kWaves) {
    uint64_t x = list[64 * g + lane];
    sort_step<1>(x, lane, (lane & 2) == 0);
    sort_step<2>(x, lane, (lane & 4) == 0), sort_step<1>(x, lane, (lane & 4) == 0);
    sort_step<4>(x, lane, (lane & 8) == 0), sort_step<2>(x, lane, (lane & 8) == 0), sort_step<1>(x, lane, (lane & 8) == 0);
    sort_step<8>(x, lane, (lane & 16) == 0), sort_half<4>(x, lane, (lane & 16) == 0);
    sort_step<16>(x, lane, (lane & 32) == 0), sort_half<8>(x, lane, (lane & 32) == 0);
    sort_half<32>(x, lane, (g & 1) == 0);
    list[64 * g + lane] = x;
  }
  __syncthreads();
  for (int size = 128; size <= n2; size *= 2) {
    for (int step = size / 2; step >= 64; step /= 2) {
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
    for (int g = wave; g < n2 / 64; g += kWaves) {
      uint64_t x = list[64 * g + lane];
      sort_half<32>(x, lane, (64 * g & size) == 0);
      list[64 * g + lane] = x;
    }
    __syncthreads();
  }
}
__device__ __forceinline__ uint32_t listed_key(uint64_t x) { return ~(uint32_t)(x >> 32); }

struct DrawShared {
  uint64_t list[kList];
  uint64_t spare[kRanked];
  uint32_t rank[kRanked];
  double table[kBins];
  uint64_t scan[2 * kWaves];
  unsigned long long kept[kMostSlices];                  // weight that a slice keeps
  int at_slice;
  uint64_t in_slice, in_row;                             // the target in front of which so much of the slice, of the row, is
  uint32_t key;                                          // the border that the list gives
  int index, stay;
};

// The border and the token of a row, by a workgroup.  sh.list: the listed tokens in any order; sh.kept: what slices keep without those.
template <typename T>
__device__ __forceinline__ void draw_row(const SampleParams& p, int r, const T* x, const Settings& set, double my_bin, const RowPlan& plan,
                                         DrawShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  sh.table[tid] = my_bin * kPlaceToRow;
  const Weights weight(set, plan.top, sh.table);
  __syncthreads();
  uint32_t key = 0;
  int index = p.V;
  if (plan.how == kFromList) {
    const uint32_t least = set.least_key(plan.top);
    if (tid == 0) {
      sh.key = least;
      sh.index = p.V;
      sh.stay = 0;
    }
    sort_list(sh.list, plan.listed, sh.spare, sh.rank);
    const int n = plan.k > 0 ? min(plan.k, plan.listed) : plan.listed;
    const int each = (n + kThreads - 1) / kThreads, i0 = min(tid * each, n), i1 = min(i0 + each, n);
    uint64_t sum = 0, all;
    for (int i = i0; i < i1; ++i) sum += weight(set, key_logit(listed_key(sh.list[i])));
    uint64_t upto = plan.above + block_scan64(sum, sh.scan, all) - sum;
    const uint64_t limit = plan.k > 0 ? limit_of(set.top_p, all) : plan.limit;
    for (int i = i0; i < i1; ++i) {
      const uint32_t ki = listed_key(sh.list[i]);
      if ((set.top_p < 1.f && upto >= limit) || ki < least) break;
      const uint64_t w = weight(set, key_logit(ki));
      upto += w;
      const int v = (int)(uint32_t)sh.list[i];
      atomicAdd(&sh.kept[v / p.slice], (unsigned long long)w);
      if (i < kRanked) sh.spare[i] = w;
      if (i + 1 == n || (set.top_p < 1.f && upto >= limit) || listed_key(sh.list[i + 1]) < least) {
        sh.key = ki;
        sh.index = v;
        sh.stay = i + 1;
      }
    }
    __syncthreads();
    key = sh.key;
    index = sh.index;
  } else if (plan.how == kSlow) {
    slow_border<T>(x, p.V, set, plan.k, plan.top, weight, reinterpret_cast<unsigned long long*>(sh.list), sh.scan, key, index);
    for (int s = 0; s < p.slices; ++s) {
      uint64_t w = 0, all;
      for (int v = s * p.slice + tid; v < min((s + 1) * p.slice, p.V); v += kThreads) {
        const float f = clean(load1(x + v));
        const uint32_t kf = score_key(f);
        if (f > -INFINITY && (kf > key || (kf == key && v <= index))) w += weight(set, f);
      }
      block_scan64(w, sh.scan, all);
      if (tid == 0) sh.kept[s] = all;
    }
  }
  __syncthreads();
  Border border{key == 0 ? -INFINITY : key_logit(key), index, 0.0};
  if (border.least == -INFINITY) border.index = -1;
  // the target, and the slice it falls in
  if (wave == 0) {
    const uint64_t a = 2 * lane < p.slices ? sh.kept[2 * lane] : 0, b = 2 * lane + 1 < p.slices ? sh.kept[2 * lane + 1] : 0;
    const uint64_t upto = wave_scan64(a + b), total = lane64(upto, 63), front = upto - a - b;
    const double t = p.tokens ? (double)p.u[r] * (double)total : 0.0;
    uint64_t target = t > 0.0 ? (uint64_t)t : 0;
    target = min(target, total - 1);
    if (front <= target && target < upto) {
      const bool second = target >= front + a;
      sh.at_slice = 2 * lane + (second ? 1 : 0);
      sh.in_slice = target - front - (second ? a : 0);
      sh.in_row = target;
    }
    if (lane == 0) p.border[r] = Border{border.least, border.index, 1.0 / (double)total};
  }
  if (!p.tokens) return;
  __syncthreads();
  if (plan.how == kFromList && plan.k > 0 && sh.stay <= kRanked) {       // all kept tokens are in the list: by what is in front of each, by index
    uint64_t* const front = reinterpret_cast<uint64_t*>(sh.table);
    const int n = sh.stay, i = tid & (kRanked - 1), part = tid / kRanked, each = (n + 3) / 4;
    if (tid < kRanked) front[tid] = 0;
    __syncthreads();
    if (i < n) {
      const uint32_t mine = (uint32_t)sh.list[i];
      uint64_t sum = 0;
      for (int j = part * each; j < min((part + 1) * each, n); ++j) sum += (uint32_t)sh.list[j] < mine ? sh.spare[j] : 0;
      atomicAdd(reinterpret_cast<unsigned long long*>(&front[i]), (unsigned long long)sum);
    }
    __syncthreads();
    if (tid < n && front[tid] <= sh.in_row && sh.in_row < front[tid] + sh.spare[tid]) p.tokens[r] = (int)(uint32_t)sh.list[tid];
    return;
  }
  // the token: the wavefronts take consecutive shares of the slice, then all of them the share that it is in
  const int begin = sh.at_slice * p.slice, end = min(begin + p.slice, p.V), share = p.slice / kWaves;
  const auto kept_weight = [&](float l, int v) -> uint64_t { return border.keeps(l, v) ? weight(set, l) : 0; };
  uint64_t sum = 0;
  const int v1 = min(begin + (wave + 1) * share, end);
  for (int v0 = begin + wave * share; v0 < v1; v0 += 256 * kReadAhead) {
    float4 f[kReadAhead];
    read_logits<kReadAhead, 64>(x, v0, lane, v1, f);
#pragma unroll
    for (int i = 0; i < kReadAhead; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += kept_weight(get(f[i], e), v0 + 4 * (i * 64 + lane) + e);
  }
  sum = wave_sum64(sum);
  if (lane == 0) sh.scan[wave] = sum;
  __syncthreads();
  const uint64_t upto_wave = wave_scan64(lane < kWaves ? sh.scan[lane] : 0), in_all = lane64(upto_wave, kWaves - 1);
  if (in_all == 0) {                                     // (a slice whose weights are something together, and nothing each: its first kept token)
    if (tid == 0) sh.index = INT_MAX;
    __syncthreads();
    for (int v = begin + tid; v < end; v += kThreads) {
      float l = load1(x + v);
      if (border.keeps(l, v)) atomicMin(&sh.index, v);
    }
    __syncthreads();
    if (tid == 0) p.tokens[r] = sh.index < p.V ? sh.index : begin;
    return;
  }
  // (the bins' weights, rounded once each, may add up to a little more than the tokens': then it is the slice's last)
  const uint64_t target = min(sh.in_slice, in_all - 1);
  const int at = __builtin_ctzll(__ballot(upto_wave > target));
  const int each = (share + kThreads - 1) / kThreads, first = begin + at * share + tid * each, last = min(first + each, min(begin + (at + 1) * share, end));
  uint64_t mine = 0, all;
  for (int v = first; v < last; ++v) mine += kept_weight(load1(x + v), v);
  __syncthreads();
  uint64_t upto = (at > 0 ? lane64(upto_wave, at - 1) : 0) + block_scan64(mine, sh.scan, all);
  if (upto <= target || upto - mine > target) return;
  upto -= mine;
  for (int v = first; v < last; ++v) {
    upto += kept_weight(load1(x + v), v);
    if (upto > target) {
      p.tokens[r] = v;
      return;
    }
  }
}
__device__ __forceinline__ void nothing_to_draw(const SampleParams& p, int r) {
  if (threadIdx.x != 0) return;
  if (p.tokens) p.tokens[r] = -1;
  p.border[r] = Border{INFINITY, -1, 0.0};
}

// grid: (rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleParams p) {
  __shared__ DrawShared sh;
  const int tid = threadIdx.x, r = blockIdx.x;
  const RowPlan plan = p.plan[r];
  if (plan.top == -INFINITY) {
    nothing_to_draw(p, r);
    return;
  }
  if (tid < p.slices) sh.kept[tid] = plan.how == kSlow ? 0 : p.stats[(int64_t)r * p.slices + tid].above;
  if (plan.how == kFromList)
    for (int i = tid; i < plan.listed; i += kThreads) sh.list[i] = p.list[(int64_t)r * kList + i];
  const Settings set(p, r);
  draw_row<T>(p, r, static_cast<const T*>(p.logits) + (int64_t)r * p.stride, set, bin_weight((float)tid, set), plan, sh);
}

// ---- a row at a time -------------------------------------------------------------------------------

// All of it for rows that a workgroup's registers hold.  grid: (rows)
template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleParams p) {
  __shared__ StatsShared stats;
  __shared__ GatherShared gather;
  __shared__ DrawShared sh;
  const int tid = threadIdx.x, r = blockIdx.x;
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  float4 f[EPT / 4];
  read_logits<EPT / 4, kThreads>(x, 0, tid, p.V, f);
  const Settings set(p, r);
  const double my_bin = bin_weight((float)tid, set);
  if (tid == 0) gather.clear();
  const SliceFound found = slice_stats<T, EPT>(set, my_bin, x, p.V, f, stats);
  if (found.top == -INFINITY) {
    if (tid == 0 && p.probs) p.plan[r] = RowPlan{found.top, kEverything, 0, 0, 0, 0};
    nothing_to_draw(p, r);
    return;
  }
  RowPlan plan{found.top, kEverything, 0, 0, 0, 0};
  uint64_t above = found.total;
  if (set.filtered()) {
    const uint64_t m = (uint64_t)((double)weight_of(found.word) * (my_bin * kPlaceToRow));
    Bins bins;
    plan = plan_row(set, found.top, count_of(found.word), m, found.total, found.n, gather, bins);
    if (plan.how != kEverything) above = plan.how == kSlow ? 0 : plan.above;
    if (plan.how == kFromList) {
      const ListRange range(set, found.top, bins);
#pragma unroll
      for (int i = 0; i < EPT / 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (range.has(get(f[i], e))) {
            const uint32_t to = atomicAdd(&gather.used, 1u);
            if (to < kList) sh.list[to] = listed(get(f[i], e), 4 * (i * kThreads + tid) + e);
          }
    }
  }
  if (tid == 0) {
    sh.kept[0] = above;
    if (p.probs) p.plan[r] = plan;
  }
  draw_row<T>(p, r, x, set, my_bin, plan, sh);
}

// ---- probabilities ---------------------------------------------------------------------------------

// grid: (slices, rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_probs_kernel(SampleParams p) {
  __shared__ float table[kBins];                         // a bin's weight over the total
  const int tid = threadIdx.x, s = blockIdx.x, r = blockIdx.y;
  const Settings set(p, r);
  const Border border = p.border[r];
  const float top = p.plan[r].top, first = set.bin_of(top);
  const PlaceExcess excess(set);
  const double to_prob = border.inv_total * (double)(1ull << kFraction);
  table[tid] = (float)(bin_weight((float)tid, set) * to_prob);
  __syncthreads();
  const T* const x = static_cast<const T*>(p.logits) + (int64_t)r * p.stride;
  float* const out = p.probs + (int64_t)r * p.V;
  const int end = min((s + 1) * p.slice, p.V);
  for (int v0 = s * p.slice; v0 < end; v0 += 4 * kReadAhead * kThreads) {
    float4 f[kReadAhead];
    read_logits<kReadAhead, kThreads>(x, v0, tid, end, f);
#pragma unroll
    for (int i = 0; i < kReadAhead; ++i) {
      const int v = v0 + 4 * (i * kThreads + tid);
      float4_u w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float l = get(f[i], e);
        w[e] = 0.f;
        if (border.keeps(l, v + e)) {
          float place;
          const float b = first - set.bin_of(l, place), g = b < (float)kBins ? table[(int)b] : (float)(bin_weight(b, set) * to_prob);
          w[e] = __builtin_fmaf(g, excess(place), g);
        }
      }
      if (v + 3 < end) {
        *reinterpret_cast<float4_u*>(out + v) = w;
      } else {
        for (int e = 0; v + e < end; ++e) out[v + e] = w[e];
      }
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------

// Tokens of a slice: as many workgroups as there are compute units, if the rows have that many slices of 4096.
int slice_of(int rows, int V) {
  const int wanted = V <= 32768 ? 1 : std::max(1, 256 / rows), each = (V + wanted - 1) / wanted;
  int s = 4096;
  while (s < each && s < 32768) s *= 2;
  return s;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

struct Layout {
  int slice, slices;
  size_t stats, bins, list, plan, border, bytes;
  Layout(int rows, int V) {
    slice = slice_of(rows, V);
    slices = (V + slice - 1) / slice;
    const size_t n = slices > 1 ? (size_t)rows * slices : 0, lists = slices > 1 ? (size_t)rows : 0;       // (one: in its workgroup's LDS)
    size_t off = 0;
    stats = off;
    off += align256(n * sizeof(SliceStats));
    bins = off;
    off += align256(n * kBins * sizeof(uint64_t));
    list = off;
    off += align256(lists * kList * sizeof(uint64_t));
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
  const auto launch = [&](auto per_thread) {
    constexpr int EPT = decltype(per_thread)::value;
    if (p.slices == 1) hipLaunchKernelGGL((sample_row_kernel<T, EPT>), dim3((unsigned)p.rows), block, 0, st, p);
    else hipLaunchKernelGGL((sample_stats_kernel<T, EPT>), grid, block, 0, st, p);
  };
  switch (p.slice) {
    case 4096: launch(std::integral_constant<int, 4>()); break;
    case 8192: launch(std::integral_constant<int, 8>()); break;
    case 16384: launch(std::integral_constant<int, 16>()); break;
    default: launch(std::integral_constant<int, 32>()); break;
  }
  if (p.slices > 1) {
    hipLaunchKernelGGL(sample_gather_kernel<T>, grid, block, 0, st, p);
    hipLaunchKernelGGL(sample_draw_kernel<T>, dim3((unsigned)p.rows), block, 0, st, p);
  }
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
  p.bins = reinterpret_cast<uint64_t*>(w + at.bins);
  p.list = reinterpret_cast<uint64_t*>(w + at.list);
  p.plan = reinterpret_cast<svf::RowPlan*>(w + at.plan);
  p.border = reinterpret_cast<svf::Border*>(w + at.border);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return (dtype == SVF_F32 ? svf::launch_sample<float>(p, st) : svf::launch_sample<__hip_bfloat16>(p, st)) == hipSuccess
             ? SVF_OK : SVF_ERR_HIP;
}

}  // extern "C"
