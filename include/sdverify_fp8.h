/*
 * sdverify_fp8.h -- the verification step's data in 8 bits (MI355X, gfx950).
 *
 * A verification step is bound by the bytes that it streams: every request's
 * KV cache once and the vocabulary weights once.  These calls hold both in
 * 8-bit floating point (e4m3: four exponent bits, three fraction bits, largest
 * value 448, no infinities, NaN 0x7f), and so read half the bytes:
 *   sd_kv8_append            new key and value rows into a paged 8-bit cache
 *   sd_verify_attention_kv8  verification attention over such caches: a draft
 *                            chain, a candidate tree, or one token per request
 *   sd_residual_norm_fp8     the residual's addition, the root-mean-square norm
 *                            and its 8-bit output, the projection's input
 *   sd_verify_logits_fp8     the vocabulary projection of such rows with 8-bit
 *                            weights, and the rows' log-sum-exp, as
 *                            sd_accept_resample and its kin take them
 * Products and sums are float32: codes widen to bfloat16 exactly, their
 * products are exact, and scales enter in float32.  The attention's weights
 * exp(score - maximum) are rounded to bfloat16 where they multiply V, and the
 * sum that divides adds the rounded ones.
 *
 * The conventions of sdverify.h hold: device pointers unless marked (host),
 * argument checks on the host before anything is enqueued, no allocation, no
 * synchronisation, no pointer kept, deterministic results, scratch from the
 * caller's workspace (sd_fp8_workspace_bytes), which one call at a time may
 * use: calls that may overlap, and graphs that may replay at once, need one each.
 * Work is enqueued on `stream`, which belongs to the current device, as do all
 * buffers.
 * sd_dims_t is used with these differences: gamma may be 0 (one position per
 * request: plain decoding, whose token the caller draws from the logits, since
 * acceptance takes gamma >= 1), flags must be 0, and a call reads only the fields
 * that it lists.
 */
#ifndef SDVERIFY_FP8_H
#define SDVERIFY_FP8_H

#include "sdverify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Keys that share one cache scale, per KV head and for K and V apart. */
#define SD_KV8_BLOCK 64
/* Columns that share one scale of hidden rows, and columns and rows of weights. */
#define SD_FP8_BLOCK 128

/*
 * A paged 8-bit KV cache.  Request b's key n is row n % page_size of page
 * block_table[b][n / page_size] (as in sd_kv_pages_t; page ids from
 * sd_kv_pool_block_table).  A page holds, per KV head, page_size / 64 blocks of
 * 64 keys, head_dim * 64 bytes each, in the order in which the matrix
 * instructions take them, so that every load is 1 KB in a row:
 *   k        [num_pages][n_kv_heads][page_size/64][D/64][4 t][4 g][16 r][16 b]
 *            e4m3: key 16 t + r of the block, column 64 i + 16 g + b
 *   v        [num_pages][n_kv_heads][page_size/64][D/16][4 g][16 d][4 t][4 r]
 *            e4m3: key 16 t + 4 g + r of the block, column 16 i + d
 *   k_scale, v_scale  [num_pages][n_kv_heads][page_size/64] exponent bytes: a
 *            code stands for code * 2^(byte - 127).  sd_kv8_append writes bytes
 *            27 .. 247 (or a block's larger one); both calls take 1 .. 254.
 * k and v 16-byte aligned, block_table 4-byte aligned.
 */
typedef struct {
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  const int32_t* block_table; /* device [B][max_pages]; an id outside [0, num_pages) is clamped into it */
  int32_t max_pages;          /* entries per request in block_table */
  int32_t page_size;          /* keys per page: a power of two in [64, 4096] */
  int32_t num_pages;          /* pages in each pool */
} sd_kv8_cache_t;

/* Workspace bytes for any call below with these dims and every kv_len <=
 * max_kv_len; 0 for an invalid shape. */
SD_API size_t sd_fp8_workspace_bytes(const sd_dims_t* dims, int32_t max_kv_len);

/*
 * Append rows to the caches.  Request b's keys kv_len[b] - new_len[b] ..
 * kv_len[b] - 1 become rows new_off[b] .. of k_new and v_new.
 *   dims     batch, n_kv_heads, head_dim (64 or 128), dtype (of the new rows)
 *   k_new, v_new  rows of n_kv_heads * head_dim elements in dtype, row t at
 *            element t * k_stride (v_stride): a slice of a wider projection's
 *            output will do.  16-byte aligned, strides a multiple of 16 bytes,
 *            at least a row.
 *   new_off  (host) [B] first row of each request, >= 0
 *   new_len  (host) [B] rows to append, 0 .. kv_len[b]; a request with 0 is left as it is
 *   kv_len   (host) [B] cached length after the call, <= max_pages * page_size
 * Of each block of 64 keys and head, with x the largest finite magnitude of its
 * new rows: the scale is the smallest 2^e >= 2^-100 with x <= 448 * 2^e, but no
 * smaller than the block's present scale if the block holds earlier keys
 * (cut back to kv_len - new_len); those are rewritten for the new scale, which
 * is exact but for values that fall below the type's normal range.  Codes are
 * rounded to nearest, ties to even; infinities and NaN become NaN.  Bytes of keys
 * from kv_len on keep their values; other pages are not touched.  The pages that
 * a call writes belong to one request each; calls on one cache run one after another.
 * A block's scale never shrinks while it holds earlier keys.  A rejected draft that raised it
 * has requantised the earlier keys of its block, and they stay so after the cut back:
 * values below 2^-6 of the new scale keep fewer fraction bits than in a cache that
 * never saw the draft.  Acceptance is lossless with respect to the logits of the cache as it is.
 */
SD_API int sd_kv8_append(const sd_dims_t* dims, const sd_kv8_cache_t* cache, const void* k_new, int64_t k_stride,
                         const void* v_new, int64_t v_stride, const int64_t* new_off, const int32_t* new_len,
                         const int32_t* kv_len, sd_stream_t stream);

/*
 * sd_verify_attention_paged (parent NULL) or sd_verify_attention_tree over an
 * 8-bit cache.
 *   dims     batch, gamma (0 .. 63), n_q_heads, n_kv_heads, head_dim (64 or
 *            128), dtype SD_DTYPE_BF16 (SD_ERR_UNSUPPORTED otherwise)
 *   q        [B][G][Hq][D] bf16, out likewise; 16-byte aligned
 *   kv_len   (host) [B], G <= kv_len[b] <= max_pages * page_size; the last G
 *            keys are this step's positions, appended before
 *   parent   NULL, or [B][gamma] int32 (device) as in sd_verify_attention_tree.
 *            After acceptance, append the accepted nodes' rows again, from
 *            key kv_len - gamma on: that is the cache's commit.  Their rows, which the
 *            caller kept, have to be gathered first: an append takes consecutive rows.
 *   scale    softmax scale, finite and > 0
 * G * (n_q_heads / n_kv_heads) <= 128.  Keys that a position does not see
 * contribute nothing, whatever they hold; a NaN that it sees makes its output NaN.
 * Scores, and the sum of |V| over a request's keys, have to lie within float32's
 * range: what passes it comes out as an infinity or NaN.
 */
SD_API int sd_verify_attention_kv8(const sd_dims_t* dims, const void* q, const sd_kv8_cache_t* cache,
                                   const int32_t* kv_len, const int32_t* parent, float scale, void* out,
                                   void* workspace, size_t workspace_bytes, sd_stream_t stream);

/*
 * Residual, norm and 8-bit output of `rows` rows of `width` columns:
 *   h = x + residual, new_residual = h in dtype, y = h * weight / sqrt(mean(h^2) + eps),
 *   and per row and 128 columns: s = max(max|y| / 448, 2^-126), code = y / s in e4m3.
 * y is formed from the unrounded h; the mean in float64, the rest in float32.  1/rms
 * divides out of y / s: a code is the nearest to h * weight / (max|h * weight| / 448),
 * three float32 roundings.
 *   x, residual, new_residual  [rows][width] in dtype; residual NULL: h = x;
 *            new_residual NULL: not stored.  new_residual may be x or residual.
 *   weight   [width] in dtype
 *   out      [rows][width] e4m3, 16-byte aligned like all of the above
 *   out_scale  [ceil(width/128)][rows] float32: sd_verify_logits_fp8's hidden_scale
 * width: a multiple of 32, at most 32768 (SD_ERR_UNSUPPORTED otherwise); rows 1 .. 2^24.
 * A NaN or an infinity in h makes the row's codes NaN or, where h is finite
 * beside an infinity, 0; the scale stays a number.  So do zeros with eps 0 (0 / 0).
 */
typedef struct {
  int32_t rows;
  int32_t width;
  int32_t dtype; /* sd_dtype_t */
  float eps;     /* >= 0, finite */
} sd_norm_t;
SD_API int sd_residual_norm_fp8(const sd_norm_t* norm, const void* x, const void* residual, const void* weight,
                                void* new_residual, void* out, float* out_scale, sd_stream_t stream);

/*
 * sd_verify_logits with 8-bit rows and weights:
 *   logits[m][v] = sum_c hidden_scale[c][m] * w_scale[v/128][c] * sum_{k in block c} hidden[m][k] * w[v][k]
 * over the blocks c of 128 columns.
 *   dims     batch and gamma (M = B * G rows), hidden (a multiple of 32, at most 2^23), vocab
 *   hidden   [M][hidden] e4m3; hidden_scale [ceil(hidden/128)][M] float32
 *   w        [V][hidden] e4m3; w_scale [ceil(V/128)][ceil(hidden/128)] float32
 *   logits   [M][V] float32; row_lse [M] float32
 * hidden, w, logits, workspace 16-byte aligned.  The sum of a block is float32
 * over exact products; scales multiply it in float32.
 */
SD_API int sd_verify_logits_fp8(const sd_dims_t* dims, const void* hidden, const float* hidden_scale, const void* w,
                                const float* w_scale, float* logits, float* row_lse, void* workspace,
                                size_t workspace_bytes, sd_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SDVERIFY_FP8_H */
