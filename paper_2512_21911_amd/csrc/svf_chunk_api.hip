// C ABI of the cache operators: argument checks, parameters, launches.
#include <cmath>

#include "svf_chunk_device.h"

namespace {

constexpr size_t kAlign = 256;
bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
int64_t or_dense(int64_t stride, int64_t dense) { return stride == 0 ? dense : stride; }

int check_chunk_shape(const svf_chunk_shape_t* s) {
  if (!s) return SVF_ERR_NULL;
  if (s->dtype != SVF_F32 && s->dtype != SVF_BF16) return SVF_ERR_DTYPE;
  if (s->B < 1 || s->B > 4096 || s->Hkv < 1 || s->Hq < 1 || s->Hq % s->Hkv != 0 || s->Hq / s->Hkv > 256 || s->Hq > 4096)
    return SVF_ERR_SHAPE;
  if (s->d != 64 && s->d != 128) return SVF_ERR_SHAPE;
  if (s->page_size < 0 || s->n_pages < 1 || s->max_seq_len < 1 || s->max_new < 1 || s->n_rows < 1 || s->window < 0)
    return SVF_ERR_SHAPE;
  // (places in a sequence, and places plus a tile, are 32-bit numbers)
  if (s->max_seq_len > (1 << 30) || s->max_new > (1 << 22) || s->n_rows > (1 << 28)) return SVF_ERR_SHAPE;
  const int vec = s->dtype == SVF_F32 ? 4 : 8;
  if (s->kv_stride_tok < s->d || s->kv_stride_head < s->d || s->kv_stride_page < s->d) return SVF_ERR_SHAPE;
  if (s->kv_stride_tok % vec || s->kv_stride_head % vec || s->kv_stride_page % vec) return SVF_ERR_SHAPE;
  // (strides in sixteen-byte chunks are 32-bit numbers too)
  if ((s->kv_stride_tok | s->kv_stride_head | s->kv_stride_page) >> 34) return SVF_ERR_SHAPE;
  const int64_t q_row = (int64_t)s->Hq * s->d, kv_row = (int64_t)s->Hkv * s->d;
  if (or_dense(s->q_stride, q_row) < q_row || or_dense(s->out_stride, q_row) < q_row ||
      or_dense(s->k_stride, kv_row) < kv_row || or_dense(s->v_stride, kv_row) < kv_row) return SVF_ERR_SHAPE;
  if (s->q_stride % vec || s->k_stride % vec || s->v_stride % vec || s->out_stride % vec) return SVF_ERR_SHAPE;
  if (std::isnan(s->sm_scale) || std::isinf(s->sm_scale) || std::isnan(s->rotary_scale) || std::isinf(s->rotary_scale))
    return SVF_ERR_SHAPE;
  if (s->rotary_dim < 0 || s->rotary_dim % 16 || s->rotary_dim > s->d) return SVF_ERR_SHAPE;
  if (s->rotary_interleaved != 0 && s->rotary_interleaved != 1) return SVF_ERR_SHAPE;
  if (s->page_size > 0) {
    if (s->max_pages_per_seq < 1 || (int64_t)s->max_pages_per_seq * s->page_size < (int64_t)s->max_seq_len)
      return SVF_ERR_PAGING;
  } else if (s->n_pages < s->B) {
    return SVF_ERR_PAGING;
  }
  return SVF_OK;
}

svf::KvLayout layout_of(const svf_chunk_shape_t& s) {
  svf::KvLayout kv;
  kv.stride_page = s.kv_stride_page;
  kv.stride_tok = s.kv_stride_tok;
  kv.stride_head = s.kv_stride_head;
  kv.page_size = s.page_size;
  kv.page_shift = -1;
  if (s.page_size > 0 && (s.page_size & (s.page_size - 1)) == 0) kv.page_shift = __builtin_ctz((unsigned)s.page_size);
  kv.max_pages = s.max_pages_per_seq;
  return kv;
}

// The choice between the kernels: the one for few rows takes 32 at a time and keeps memory busier, which binds where rows are few.  Four sequences of
// 32k, one token of four heads a KV head: 111 us against 169 by the other; nine tokens, whose 36 rows it reads the keys twice for: 203 against 150.
bool few_rows(const svf_chunk_shape_t& s) { return s.dtype == SVF_F32 || svf::chunk_attn_is_few(s.Hq / s.Hkv, s.max_new); }

size_t workspace_of(const svf_chunk_shape_t& s) {
  const size_t n = few_rows(s) ? svf::chunk_attn_few_workspace(s.d) : svf::chunk_attn_workspace(s.d);
  return (n + kAlign - 1) / kAlign * kAlign;
}

}  // namespace

extern "C" {

int svf_append_kv(const svf_chunk_shape_t* shape, const void* k_new, const void* v_new, const int32_t* block_table,
                  const int32_t* seq_lens, const int32_t* new_rows, const int32_t* new_lens, void* K, void* V,
                  const void* q_or_null, void* q_out_or_null, const double* inv_freq_or_null,
                  const int32_t* positions_or_null, void* stream) {
  const int rc = check_chunk_shape(shape);
  if (rc) return rc;
  if (!k_new || !v_new || !seq_lens || !new_rows || !new_lens || !K || !V || (shape->page_size > 0 && !block_table))
    return SVF_ERR_NULL;
  if ((q_or_null == nullptr) != (q_out_or_null == nullptr) || (shape->rotary_dim > 0 && !inv_freq_or_null)) return SVF_ERR_NULL;
  if (misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(K, 16) || misaligned(V, 16) || misaligned(q_or_null, 16) ||
      misaligned(q_out_or_null, 16) || misaligned(block_table, 4) || misaligned(seq_lens, 4) || misaligned(new_rows, 4) ||
      misaligned(new_lens, 4) || misaligned(positions_or_null, 4) || misaligned(inv_freq_or_null, 8))
    return SVF_ERR_SHAPE;
  svf::AppendParams p;
  p.kv = layout_of(*shape);
  p.k_new = k_new;
  p.v_new = v_new;
  p.q = q_or_null;
  p.q_out = q_out_or_null;
  p.K = K;
  p.V = V;
  p.table = block_table;
  p.seq_lens = seq_lens;
  p.new_rows = new_rows;
  p.new_lens = new_lens;
  p.positions = positions_or_null;
  p.inv_freq = inv_freq_or_null;
  p.q_stride = or_dense(shape->q_stride, (int64_t)shape->Hq * shape->d);
  p.k_stride = or_dense(shape->k_stride, (int64_t)shape->Hkv * shape->d);
  p.v_stride = or_dense(shape->v_stride, (int64_t)shape->Hkv * shape->d);
  p.B = shape->B;
  p.Hq = q_or_null ? shape->Hq : 0;
  p.Hkv = shape->Hkv;
  p.d = shape->d;
  p.n_pages = shape->n_pages;
  p.max_seq_len = shape->max_seq_len;
  p.max_new = shape->max_new;
  p.n_rows = shape->n_rows;
  p.rotary_dim = shape->rotary_dim;
  p.interleaved = shape->rotary_interleaved;
  p.rotary_scale = shape->rotary_scale > 0.f ? shape->rotary_scale : 1.f;
  return svf::launch_append_kv(p, shape->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? SVF_OK : SVF_ERR_HIP;
}

size_t svf_chunk_workspace_bytes(const svf_chunk_shape_t* shape) {
  return check_chunk_shape(shape) == SVF_OK ? workspace_of(*shape) : 0;
}

int svf_chunk_attn(const svf_chunk_shape_t* shape, const void* q, const void* K, const void* V,
                   const int32_t* block_table, const int32_t* seq_lens, const int32_t* new_rows,
                   const int32_t* new_lens, void* out, float* lse_or_null, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_chunk_shape(shape);
  if (rc) return rc;
  if (!q || !K || !V || !seq_lens || !new_rows || !new_lens || !out || (shape->page_size > 0 && !block_table))
    return SVF_ERR_NULL;
  if (misaligned(q, 16) || misaligned(K, 16) || misaligned(V, 16) || misaligned(out, 16) || misaligned(lse_or_null, 4) ||
      misaligned(block_table, 4) || misaligned(seq_lens, 4) || misaligned(new_rows, 4) || misaligned(new_lens, 4))
    return SVF_ERR_SHAPE;
  if (!ws || misaligned(ws, kAlign) || ws_bytes < workspace_of(*shape)) return SVF_ERR_WORKSPACE;
  svf::ChunkParams p;
  p.kv = layout_of(*shape);
  p.page = svf::PageOf(shape->page_size);
  p.page16 = (uint32_t)(shape->kv_stride_page / 8);
  p.tok16 = (uint32_t)(shape->kv_stride_tok / 8);
  p.q = q;
  p.K = K;
  p.V = V;
  p.table = block_table;
  p.seq_lens = seq_lens;
  p.new_rows = new_rows;
  p.new_lens = new_lens;
  p.out = out;
  p.lse = lse_or_null;
  p.ws = static_cast<char*>(ws);
  p.q_stride = or_dense(shape->q_stride, (int64_t)shape->Hq * shape->d);
  p.out_stride = or_dense(shape->out_stride, (int64_t)shape->Hq * shape->d);
  p.B = shape->B;
  p.Hq = shape->Hq;
  p.Hkv = shape->Hkv;
  p.G = shape->Hq / shape->Hkv;
  p.d = shape->d;
  p.n_pages = shape->n_pages;
  p.max_seq_len = shape->max_seq_len;
  p.max_new = shape->max_new;
  p.n_rows = shape->n_rows;
  // (one that reaches past every sequence is none: the kernels take places less a window as 32-bit numbers)
  p.window = shape->window >= shape->max_seq_len ? 0 : shape->window;
  // (items of 32 rows, units of 32 keys, no more than sixteen shares beside them; up to 2^24 of both each: no overflow below 2^62)
  const int64_t share_items = ((int64_t)shape->max_new * p.G + 31) / 32, share_units = (int64_t)shape->max_seq_len / 32 + 18;
  p.share_bound = share_items > (1 << 30) / share_units ? INT64_MAX : (int64_t)shape->B * shape->Hkv * share_items * share_units;
  const float scale = shape->sm_scale > 0.f ? shape->sm_scale : 1.0f / std::sqrt((float)shape->d);
  p.scale_log2 = scale * 1.44269504088896340736f;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return (few_rows(*shape) ? svf::launch_chunk_attn_few(p, shape->dtype == SVF_F32, st) : svf::launch_chunk_attn(p, st)) == hipSuccess
             ? SVF_OK : SVF_ERR_HIP;
}

}  // extern "C"
