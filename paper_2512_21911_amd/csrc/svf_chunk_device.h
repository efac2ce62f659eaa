// Shared by the kernels of include/svf_cache.h (not part of the C ABI).
#pragma once

#include "svf_cache.h"
#include "svf_device.h"

namespace svf {

// The page of a place, t < 2^30, without a division: 4 t m / 2^(32 + s) with m = ceil(2^(30 + s) / page_size), 2^s >= page_size.  What m
// is too large by, less than one, adds less than t / 2^(30 + s) <= 1 / page_size: never a whole page.  (m has at most 32 bits.)
struct PageOf {
  uint32_t m, s;
  __host__ explicit PageOf(int page_size) : m(0), s(0) {
    if (page_size <= 0) return;                          // contiguous: page 0 of the sequence's own
    while ((1ll << s) < page_size) ++s;
    m = (uint32_t)(((1ull << (30 + s)) + (uint64_t)page_size - 1) / (uint64_t)page_size);
  }
  __device__ __forceinline__ uint32_t of(uint32_t t) const { return __umulhi(4 * t, m) >> s; }
};

struct ChunkParams {
  KvLayout kv;
  PageOf page{0};
  uint32_t page16, tok16;    // strides of the cache in sixteen-byte chunks (bf16)
  const void* q;
  const void* K;
  const void* V;
  const int32_t* table;
  const int32_t* seq_lens;
  const int32_t* new_rows;
  const int32_t* new_lens;
  void* out;
  float* lse;                // may be null
  char* ws;
  int64_t q_stride, out_stride;      // elements
  int32_t B, Hq, Hkv, G, d, n_pages, max_seq_len, max_new, n_rows, window;
  int64_t share_bound;       // shares of work (chunk_share.h) that a call has at most
  float scale_log2;          // sm_scale * log2(e)
};

struct AppendParams {
  KvLayout kv;
  const void* k_new;
  const void* v_new;
  const void* q;             // may be null
  void* q_out;
  void* K;
  void* V;
  const int32_t* table;
  const int32_t* seq_lens;
  const int32_t* new_rows;
  const int32_t* new_lens;
  const int32_t* positions;  // may be null
  const double* inv_freq;
  int64_t q_stride, k_stride, v_stride;   // elements
  int32_t B, Hq, Hkv, d, n_pages, max_seq_len, max_new, n_rows, rotary_dim, interleaved;
  float rotary_scale;
};

// The tokens a sequence takes part with: clamped to what the shape has room for, so that no
// contents of the device arrays lead outside the tensors.
struct ChunkSeq { int len, row, n; };                    // cached tokens in front, first row, new tokens
__device__ __forceinline__ ChunkSeq chunk_seq(int len, int row, int n, int max_seq_len, int max_new, int n_rows) {
  ChunkSeq s{len, row, min(n, max_new)};
  if (len < 0 || row < 0 || row >= n_rows) s.n = 0;
  else s.n = max(0, min(s.n, min(n_rows - row, max_seq_len - len)));
  if (s.n == 0) s.len = s.row = 0;
  return s;
}

// Bytes at the front of a workspace that count arrivals: zero between calls, whatever kernel they took
constexpr size_t kChunkCounters = 1024;

hipError_t launch_append_kv(const AppendParams& p, int dtype, hipStream_t st);
size_t chunk_attn_workspace(int d);
hipError_t launch_chunk_attn(const ChunkParams& p, hipStream_t st);
// 32 rows of a (sequence, KV head) at a time: bf16 with no more of them, and fp32
bool chunk_attn_is_few(int G, int max_new);
size_t chunk_attn_few_workspace(int d);
hipError_t launch_chunk_attn_few(const ChunkParams& p, bool f32, hipStream_t st);

}  // namespace svf
