/*
 * libsvf - filling the KV cache and dense attention of new tokens over it, on AMD MI355X (gfx950).
 *
 * What happens around the verification steps of svf.h: prompts are read in chunks, accepted drafts
 * join the cache, and some layers or phases attend to everything that is cached.  New tokens of all
 * sequences of a batch come packed, any number per sequence (none and one included); their keys
 * and values are written into the cache, rotated to their positions on the way (svf_append_kv), and
 * their queries attend to all cached tokens up to themselves (svf_chunk_attn).
 *
 * Conventions as in svf.h: the shape is a HOST pointer, every other pointer is a DEVICE pointer
 * owned by the caller; work is enqueued on `stream` and the call returns immediately; 0 on
 * success, a negative SVF_ERR_* code (svf.h) otherwise, checked before any launch; inputs must be
 * finite (a NaN or infinity in a query stays in that query's output, one in a cached token spoils
 * the new tokens of sequences that see it; cache places that no new token sees may hold anything), and
 * values below 2^125 / (tokens of the sequence + 64), since their weighted sums are fp32 until they are divided.
 * A call runs on the current device, as every HIP launch does: stream and pointers are that device's.
 *
 * Tensors (last index fastest; element type = shape.dtype unless said otherwise):
 *   k_new, v_new  [n_rows][Hkv][d]     rows shape.k_stride / v_stride elements apart
 *   q, q_out      [n_rows][Hq][d]      rows shape.q_stride elements apart (both)
 *   out           [n_rows][Hq][d]      rows shape.out_stride elements apart
 *   lse           fp32 [n_rows][Hq]    natural log of sum(exp(scaled logits))
 *   K, V          cache pool of shape.n_pages pages, addressed as in svf.h (kv_stride_*, block_table)
 *   block_table   int32 [B][max_pages_per_seq]  (ignored for a contiguous cache, page_size = 0: page = sequence)
 *   seq_lens      int32 [B]            tokens a sequence has in front of the new ones, 0 .. max_seq_len
 *   new_rows      int32 [B]            row of a sequence's first new token
 *   new_lens      int32 [B]            its new tokens, in consecutive rows
 * New token j of sequence b is row new_rows[b] + j and takes place seq_lens[b] + j of its cache.  Rows
 * that belong to no sequence are gaps: nothing is done with them, and their outputs stay as they were.
 * Rows of two sequences must not overlap, nor may the cache places that one call writes.  What the
 * shape has no room for is left out, whatever the device arrays hold: a sequence takes part with
 *   min(new_lens[b], max_new, n_rows - new_rows[b], max_seq_len - seq_lens[b]) tokens (none if that, new_rows[b]
 *   or seq_lens[b] is negative),
 * a page outside 0 .. n_pages - 1 is not written to, and read as page 0 (any values, no access outside).
 */
#ifndef SVF_CACHE_H_
#define SVF_CACHE_H_

#include "svf.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct svf_chunk_shape {
  int32_t B;                 /* sequences in the batch, 1..4096                               */
  int32_t Hq, Hkv;           /* query heads, KV heads; Hq % Hkv == 0, Hq <= 4096, Hq / Hkv <= 256 */
  int32_t d;                 /* head dimension: 64 or 128                                     */
  int32_t dtype;             /* SVF_F32 or SVF_BF16                                           */
  int32_t page_size;         /* tokens per physical page; 0 = contiguous cache                */
  int32_t max_pages_per_seq; /* row length of block_table (unused when page_size == 0)        */
  int32_t n_pages;           /* pages of the pool (contiguous: sequences it has room for, >= B)   */
  int32_t max_seq_len;       /* tokens a sequence may have, the new ones included, 1..2^30    */
  int32_t max_new;           /* new tokens a sequence may have in one call, 1..2^22          */
  int32_t n_rows;            /* rows of q, k_new, v_new and the outputs, 1..2^28              */
  int32_t window;            /* a token sees the last `window` tokens, itself included; 0: all */
  int64_t kv_stride_page, kv_stride_tok, kv_stride_head; /* as in svf_shape_t, below 2^34 elements */
  int64_t q_stride, k_stride, v_stride, out_stride;      /* elements between rows; 0: dense   */
  float sm_scale;            /* softmax scale; <= 0 selects 1/sqrt(d)                         */
  int32_t rotary_dim;        /* leading channels that are rotated: 0 (none) or a multiple of 16, <= d */
  int32_t rotary_interleaved;/* 0: channel i pairs with i + rotary_dim / 2; 1: channels 2i, 2i + 1 */
  float rotary_scale;        /* factor of the rotated channels; <= 0 selects 1                */
} svf_chunk_shape_t;

/*
 * Appends the new tokens to the cache.  With rotary_dim > 0 the leading channels of every key, and of
 * every query if q is given, are rotated: pair i of a token at position p turns by the angle
 * p * inv_freq[i] (x, y -> x cos - y sin, y cos + x sin, times rotary_scale); inv_freq is fp64
 * [rotary_dim / 2], radians per position, and p = positions[row], or the token's place in the cache
 * if positions is NULL (a draft tree's nodes sit deeper or shallower than they are stored).  Angles are
 * taken modulo whole turns in fp64, so that far positions lose nothing; the rotation is fp32, rounded
 * once.  Values, and channels past rotary_dim, are copied.  q_out may be q itself (rotation in place);
 * k_new, v_new and q must not overlap the cache.  q and q_out are given both or not at all; with
 * rotary_dim = 0 inv_freq and positions are ignored and q is copied.
 * SVF_ERR_NULL, SVF_ERR_SHAPE (sizes, strides that are no multiple of 16 bytes, pointers that are not
 * 16-byte aligned), SVF_ERR_DTYPE, SVF_ERR_PAGING (max_pages_per_seq or n_pages too small).
 */
int svf_append_kv(const svf_chunk_shape_t* shape, const void* k_new, const void* v_new, const int32_t* block_table,
                  const int32_t* seq_lens, const int32_t* new_rows, const int32_t* new_lens, void* K, void* V,
                  const void* q_or_null, void* q_out_or_null, const double* inv_freq_or_null,
                  const int32_t* positions_or_null, void* stream);

/*
 * Bytes of device workspace svf_chunk_attn needs for `shape` (a multiple of 256; 0 if the shape is
 * invalid).  As svf_workspace_bytes' (svf.h): 256-byte aligned, cleared to zero once (svf_workspace_init) before
 * its first use, left reusable by every call; calls that share one must be ordered on one stream.
 * Unlike that one's it serves every shape that needs no more bytes.
 */
size_t svf_chunk_workspace_bytes(const svf_chunk_shape_t* shape);

/*
 * Attention of the new tokens, whose keys and values are in the cache already: query head h of new token j of
 * sequence b attends to places max(0, seq_lens[b] + j + 1 - window) .. seq_lens[b] + j of KV head
 * h / (Hq / Hkv) under one softmax with scale sm_scale.  lse_or_null is optional.  `out` must
 * not overlap q or the cache.
 * Arithmetic in bf16: products accumulate in fp32, softmax weights are rounded to bf16 before they
 * multiply V (where max_new * Hq / Hkv <= 32 to sixteen bits), their sum is taken in fp32 from the unrounded ones, everything
 * else stays fp32 until the output is rounded once.  fp32 shapes are fp32 throughout.  The same bits from call to call.
 * That limit also chooses the kernel: a step of single tokens is served 1.5 times as fast by a shape whose max_new says so.
 */
int svf_chunk_attn(const svf_chunk_shape_t* shape, const void* q, const void* K, const void* V,
                   const int32_t* block_table, const int32_t* seq_lens, const int32_t* new_rows,
                   const int32_t* new_lens, void* out, float* lse_or_null, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SVF_CACHE_H_ */
