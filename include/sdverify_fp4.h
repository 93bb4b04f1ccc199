/*
 * sdverify_fp4.h -- verification on a KV cache in 4 bits (MI355X, gfx950).
 *
 * Attention is bound by the bytes of the caches that it streams.  These calls
 * hold keys and values in 4-bit floating point (e2m1: magnitudes 0, 0.5, 1, 1.5,
 * 2, 3, 4, 6 and a sign), a quarter of bfloat16's bytes:
 *   sd_qk_norm_rope          norms of queries and keys for each head and the
 *                            position rotation: the attention's q, and the rows
 *                            that an append takes (to a cache of any type)
 *   sd_kv4_append            new key and value rows into a paged 4-bit cache
 *   sd_kv4_read              cached keys and values back as rows
 *   sd_verify_attention_kv4  verification attention over such caches: a draft
 *                            chain, a candidate tree, or one token per request
 * A key's scale is a power of two for each 32 columns, since a few columns of
 * keys are far larger than the others; a value's is one bfloat16 for the row.
 * No scale spans keys: an append touches its own keys alone, and a rejected draft
 * leaves no trace once its keys are cut off or written again.
 *
 * The conventions of sdverify_fp8.h hold: device pointers unless marked (host),
 * argument checks on the host before anything is enqueued, no allocation, no
 * synchronisation, no pointer kept, deterministic results, scratch from the
 * caller's workspace (sd_kv4_workspace_bytes), which one call at a time may use:
 * calls that may overlap, and graphs that may replay at once, need one each.
 * Work is enqueued on `stream`, which belongs to the current device, as do all
 * buffers.  sd_dims_t: gamma may be 0, flags must be 0, and a call reads only the
 * fields that it lists.
 */
#ifndef SDVERIFY_FP4_H
#define SDVERIFY_FP4_H

#include "sdverify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Keys of a block of the cache. */
#define SD_KV4_BLOCK 64
/* Columns of a key that share one scale. */
#define SD_KV4_GROUP 32

/*
 * A paged 4-bit KV cache.  Request b's key n is row n % page_size of page
 * block_table[b][n / page_size] (as in sd_kv_pages_t; page ids from
 * sd_kv_pool_block_table).  A byte holds two codes, the first column in its low
 * half; a block of 64 keys is 32 * head_dim bytes:
 *   k        [num_pages][n_kv_heads][page_size/64][4 t][4 g][16 r][D/8]
 *            key 16 t + r of the block, columns g * D/4 + 2 b and + 1 in byte b
 *   v        [num_pages][n_kv_heads][page_size/64][D/16][64 n][8]
 *            key n of the block, columns 16 i + 2 b and + 1 in byte b
 *   k_scale  [num_pages][n_kv_heads][page_size/64][D/32][16 r][4 t] exponent bytes:
 *            a code of key 16 t + r stands for code * 2^(byte - 127); 255 makes
 *            its 32 columns NaN
 *   v_scale  [num_pages][n_kv_heads][page_size/64][64 n] bfloat16: a code of key n
 *            stands for code * scale
 * k, v, k_scale and v_scale 16-byte aligned, block_table 4-byte aligned.
 */
typedef struct {
  void* k;
  void* v;
  uint8_t* k_scale;
  uint16_t* v_scale;
  const int32_t* block_table; /* device [B][max_pages]; an id outside [0, num_pages) is clamped into it */
  int32_t max_pages;          /* entries per request in block_table */
  int32_t page_size;          /* keys per page: a power of two in [64, 4096] */
  int32_t num_pages;          /* pages in each pool */
} sd_kv4_cache_t;

/* Workspace bytes of sd_verify_attention_kv4 with these dims and every kv_len <=
 * max_kv_len; 0 for an invalid shape. */
SD_API size_t sd_kv4_workspace_bytes(const sd_dims_t* dims, int32_t max_kv_len);

/*
 * Norms and position rotation of queries and keys, head by head:
 *   y = x * weight / sqrt(mean(x^2) + eps)   (y = x where the weight is NULL)
 *   of each pair (a, b) of y's first rotary_dim columns, i counting the pairs and
 *   t = positions[row] * inv_freq[i]:  (a cos t - b sin t, a sin t + b cos t)
 * and y's other columns as they are.
 *   rope     rows (0 .. 2^24 - 1; 0 enqueues nothing), n_q_heads and n_kv_heads (1 ..
 *            65535), head_dim (64 or 128), rotary_dim (a multiple of 16, 16 ..
 *            head_dim), dtype; interleaved: pairs are columns 2 i and 2 i + 1,
 *            else i and i + rotary_dim / 2
 *   q, k     rows of n_q_heads (n_kv_heads) * head_dim elements in dtype, row t
 *            at element t * stride: slices of a fused projection's output will
 *            do.  16-byte aligned, strides a multiple of 16 bytes, at least a row.
 *   positions  [rows] int32: of a tree's node its depth's, not its row's
 *   inv_freq [rotary_dim/2] float32
 *   q_weight, k_weight  [head_dim] in dtype, 16-byte aligned, either may be NULL
 *   q_out, k_out  like q and k.  Each may be its input, with its stride; other
 *            overlaps of inputs and outputs are not allowed.
 * Angles are float64, so that far positions keep theirs; sums, norms and rotations
 * float32, rounded to dtype once.  Squares that leave float32's range are summed in
 * float64.  A row of zeros with eps 0 is NaN (0 / 0).
 */
typedef struct {
  int32_t rows;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t rotary_dim;
  int32_t interleaved; /* 0 or 1 */
  int32_t dtype;       /* sd_dtype_t */
  float eps;           /* >= 0, finite */
} sd_rope_t;
SD_API int sd_qk_norm_rope(const sd_rope_t* rope, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                           const int32_t* positions, const float* inv_freq, const void* q_weight,
                           const void* k_weight, void* q_out, int64_t q_out_stride, void* k_out,
                           int64_t k_out_stride, sd_stream_t stream);

/*
 * Append rows to the caches.  Request b's keys kv_len[b] - new_len[b] ..
 * kv_len[b] - 1 become rows new_off[b] .. of k_new and v_new.
 *   dims     batch, n_kv_heads, head_dim (64 or 128), dtype (of the new rows)
 *   k_new, v_new  rows of n_kv_heads * head_dim elements in dtype, row t at
 *            element t * k_stride (v_stride); 16-byte aligned, strides a multiple
 *            of 16 bytes, at least a row
 *   new_off  (host) [B] first row of each request, >= 0
 *   new_len  (host) [B] rows to append, 0 .. kv_len[b]; a request with 0 is left as it is
 *   kv_len   (host) [B] cached length after the call, <= max_pages * page_size
 * With x the largest magnitude of a key's 32 columns, their scale is the smallest
 * 2^e >= 2^-100 with x <= 6 * 2^e; with x that of a value's row, its scale is the
 * smallest bfloat16 s >= 2^-100 with x <= 6 s.  Codes are nearest to the element
 * over its scale, ties to the even code.  The largest scales are those with which 6
 * is finite in float32, 2^125 and 170 * 2^118: elements past 6 * 2^125 = 1.5 * 2^127
 * (of values, past bfloat16's largest number) become that; nothing else saturates,
 * and what is finite stays finite.  Columns of a scale with an
 * infinity or NaN among them become NaN, all of them (scale byte 255, scale 0x7fc0,
 * codes 0).  Other keys' bytes are not touched.  The keys that a call writes
 * belong to one request each; calls on one cache run one after another.
 */
SD_API int sd_kv4_append(const sd_dims_t* dims, const sd_kv4_cache_t* cache, const void* k_new, int64_t k_stride,
                         const void* v_new, int64_t v_stride, const int64_t* new_off, const int32_t* new_len,
                         const int32_t* kv_len, sd_stream_t stream);

/*
 * Read keys and values back: request b's keys first[b] .. first[b] + count[b] - 1
 * become rows out_off[b] .. of k_out and v_out, rounded to dtype.
 *   dims     batch, n_kv_heads, head_dim (64 or 128), dtype (of the rows)
 *   first, count  (host) [B] >= 0, first[b] + count[b] <= max_pages * page_size
 *   out_off  (host) [B] >= 0; the rows of one request each
 *   k_out, v_out  rows as sd_kv4_append takes them; either may be NULL
 * Keys in float32, and in bfloat16 down to its smallest normal number, are exact;
 * appending float32 rows that were read gives the same codes' values again.  Only
 * rows' own elements are written.
 */
SD_API int sd_kv4_read(const sd_dims_t* dims, const sd_kv4_cache_t* cache, const int32_t* first, const int32_t* count,
                       const int64_t* out_off, void* k_out, int64_t k_stride, void* v_out, int64_t v_stride,
                       sd_stream_t stream);

/*
 * sd_verify_attention_paged (parent NULL) or sd_verify_attention_tree over a
 * 4-bit cache.
 *   dims     batch, gamma (0 .. 63), n_q_heads, n_kv_heads, head_dim (64 or
 *            128), dtype SD_DTYPE_BF16 (SD_ERR_UNSUPPORTED otherwise)
 *   q        [B][G][Hq][D] bf16, out likewise; 16-byte aligned
 *   kv_len   (host) [B], G <= kv_len[b] <= max_pages * page_size; the last G
 *            keys are this step's positions, appended before
 *   parent   NULL, or [B][gamma] int32 (device) as in sd_verify_attention_tree.
 *            After acceptance, append the accepted nodes' rows again, from
 *            key kv_len - gamma on, gathered from those that the caller kept: that
 *            is the cache's commit
 *   scale    softmax scale, > 0; scale * log2 e is finite in float32
 * G * (n_q_heads / n_kv_heads) <= 128.  Products are exact in float32 and summed
 * there; the weights exp(score - maximum) times the value's scale multiply V's codes
 * as the sum of two bfloat16 numbers (to 2^-16 of a term), or, where a wave holds more than
 * 16 query rows (more than 16 rows of a KV head over many keys), as one (2^-8).
 * Keys that a position does not see
 * contribute nothing, whatever they hold; a NaN that it sees makes its output NaN.
 * Products q k, scores, and 512 times the sum of |V| over a request's keys, have to lie
 * within float32's range: what passes it comes out as an infinity or NaN.
 */
SD_API int sd_verify_attention_kv4(const sd_dims_t* dims, const void* q, const sd_kv4_cache_t* cache,
                                   const int32_t* kv_len, const int32_t* parent, float scale, void* out,
                                   void* workspace, size_t workspace_bytes, sd_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SDVERIFY_FP4_H */
