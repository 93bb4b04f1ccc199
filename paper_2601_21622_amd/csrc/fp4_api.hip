// C-ABI of the 4-bit calls (sdverify_fp4.h): argument checks, workspace and
// launches.  Every check runs on the host before anything is enqueued.
#include <string.h>

#include <algorithm>
#include <cmath>

#include "sdverify_fp4.h"
#include "checks.h"
#include "fp4.h"

namespace {

using namespace sdv;

static_assert(SD_KV4_BLOCK == kKeyBlock4 && SD_KV4_GROUP == kGroup4, "the header's blocks are the kernels'");

int check_cache(const sd_kv4_cache_t* c) {
  if (c == nullptr || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->block_table) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16) ||
      !aligned(c->block_table, 4))
    return SD_ERR_INVALID_ARGUMENT;
  if (c->page_size < 64 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return SD_ERR_INVALID_ARGUMENT;
  if (c->max_pages < 1 || c->num_pages < 1) return SD_ERR_INVALID_ARGUMENT;
  return SD_OK;
}

bool length_ok(const sd_kv4_cache_t* c, int64_t n) {
  return n <= kMaxKvLen && n <= int64_t(c->max_pages) * c->page_size;
}

Kv4Pool pool_of(const sd_kv4_cache_t* c) {
  Kv4Pool p;
  p.k = static_cast<uint8_t*>(c->k);
  p.v = static_cast<uint8_t*>(c->v);
  p.k_scale = c->k_scale;
  p.v_scale = c->v_scale;
  p.table = c->block_table;
  p.max_pages = c->max_pages;
  p.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
  p.num_pages = c->num_pages;
  return p;
}

// Rows of `heads` heads at p, `stride` elements apart.
bool rows_ok(const sd_dims_t* d, const void* p, int64_t stride) {
  const int64_t unit = d->dtype == SD_DTYPE_F32 ? 4 : 8, row = int64_t(d->n_kv_heads) * d->head_dim;
  return aligned(p, 16) && stride >= row && stride % unit == 0;
}

// Launches over keys first[b] .. first[b] + count[b] - 1 of every request, as many keys to a
// launch as its table and its grid hold.
template <typename Launch>
int over_rows(const sd_dims_t* d, const int32_t* first, const int32_t* count, const int64_t* off, Launch launch) {
  const int64_t most = kMaxGrid * 4 / d->n_kv_heads;  // tiles of a launch: a wave for each and head, four to a workgroup
  Kv4Rows r;
  memset(&r, 0, sizeof(r));
  for (int b = 0; b < d->batch; ++b) {
    int64_t at = first[b], end = int64_t(first[b]) + count[b], row = off[b];
    while (at < end) {
      if (r.nreq == kMaxReqPerLaunch || r.prefix[r.nreq] == most) {
        if (launch(r) != hipSuccess) return SD_ERR_HIP;
        r.nreq = 0;
      }
      const int64_t tiles = std::min((end + kTile - 1) / kTile - at / kTile, most - r.prefix[r.nreq]);
      const int64_t stop = std::min(end, (at / kTile + tiles) * kTile);
      r.req[r.nreq] = b;
      r.first[r.nreq] = static_cast<int32_t>(at);
      r.count[r.nreq] = static_cast<int32_t>(stop - at);
      r.off[r.nreq] = row;
      r.prefix[r.nreq + 1] = static_cast<int32_t>(r.prefix[r.nreq] + tiles);
      ++r.nreq;
      row += stop - at;
      at = stop;
    }
  }
  return r.nreq == 0 || launch(r) == hipSuccess ? SD_OK : SD_ERR_HIP;
}

}  // namespace

extern "C" {

size_t sd_kv4_workspace_bytes(const sd_dims_t* d, int32_t max_kv_len) {
  if (check_attention(d) != SD_OK || max_kv_len <= d->gamma || max_kv_len > kMaxKvLen) return 0;
  const int rows = (d->gamma + 1) * (d->n_q_heads / d->n_kv_heads);
  const int64_t chunks = kv4_max_chunks(d->n_kv_heads, d->head_dim, d->batch, max_kv_len);
  return align_up(attn_partial_bytes(chunks, d->n_kv_heads, rows, d->head_dim));
}

int sd_qk_norm_rope(const sd_rope_t* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                    const int32_t* positions, const float* inv_freq, const void* q_weight, const void* k_weight,
                    void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, sd_stream_t stream) {
  if (r == nullptr || r->rows < 0 || r->n_q_heads < 1 || r->n_kv_heads < 1 || r->head_dim < 1 || r->rotary_dim < 1 ||
      r->rotary_dim > r->head_dim || (r->interleaved != 0 && r->interleaved != 1) || !(r->eps >= 0.f) ||
      !std::isfinite(r->eps))
    return SD_ERR_INVALID_ARGUMENT;
  if (r->dtype != SD_DTYPE_F32 && r->dtype != SD_DTYPE_BF16) return SD_ERR_INVALID_ARGUMENT;
  if ((r->head_dim != 64 && r->head_dim != 128) || r->rotary_dim % 16 != 0 || r->n_q_heads > 65535 ||
      r->n_kv_heads > 65535 || r->rows > kMaxGrid)
    return SD_ERR_UNSUPPORTED;
  const int64_t unit = r->dtype == SD_DTYPE_F32 ? 4 : 8;
  const int64_t q_row = int64_t(r->n_q_heads) * r->head_dim, k_row = int64_t(r->n_kv_heads) * r->head_dim;
  if (q_stride < q_row || q_out_stride < q_row || k_stride < k_row || k_out_stride < k_row || q_stride % unit != 0 ||
      q_out_stride % unit != 0 || k_stride % unit != 0 || k_out_stride % unit != 0)
    return SD_ERR_INVALID_ARGUMENT;
  if (r->rows == 0) return SD_OK;
  if (!q || !k || !positions || !inv_freq || !q_out || !k_out) return SD_ERR_INVALID_ARGUMENT;
  const void* p16[] = {q, k, q_weight, k_weight, q_out, k_out};
  for (const void* p : p16)
    if (p != nullptr && !aligned(p, 16)) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(positions, 4) || !aligned(inv_freq, 4)) return SD_ERR_INVALID_ARGUMENT;
  RopeArgs a;
  a.rows = r->rows;
  a.Hq = r->n_q_heads;
  a.Hkv = r->n_kv_heads;
  a.rotary = r->rotary_dim;
  a.eps = r->eps;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  return launch_qk_rope(a, r->head_dim, r->dtype == SD_DTYPE_F32, r->interleaved != 0, q, k, positions, inv_freq,
                        q_weight, k_weight, q_out, k_out, static_cast<hipStream_t>(stream)) == hipSuccess
             ? SD_OK
             : SD_ERR_HIP;
}

int sd_kv4_append(const sd_dims_t* d, const sd_kv4_cache_t* cache, const void* k_new, int64_t k_stride,
                  const void* v_new, int64_t v_stride, const int64_t* new_off, const int32_t* new_len,
                  const int32_t* kv_len, sd_stream_t stream) {
  int st = check_heads(d);
  if (st != SD_OK) return st;
  st = check_cache(cache);
  if (st != SD_OK) return st;
  if (!k_new || !v_new || !new_off || !new_len || !kv_len) return SD_ERR_INVALID_ARGUMENT;
  if (!rows_ok(d, k_new, k_stride) || !rows_ok(d, v_new, v_stride)) return SD_ERR_INVALID_ARGUMENT;
  for (int b = 0; b < d->batch; ++b)
    if (new_off[b] < 0 || new_len[b] < 0 || new_len[b] > kv_len[b] || !length_ok(cache, kv_len[b]))
      return SD_ERR_INVALID_ARGUMENT;
  const Kv4Pool pool = pool_of(cache);
  int32_t first[kMaxReqPerLaunch];
  sd_dims_t part = *d;
  for (int r0 = 0; r0 < d->batch; r0 += kMaxReqPerLaunch) {
    part.batch = std::min(kMaxReqPerLaunch, d->batch - r0);
    for (int i = 0; i < part.batch; ++i) first[i] = kv_len[r0 + i] - new_len[r0 + i];
    st = over_rows(&part, first, new_len + r0, new_off + r0, [&](Kv4Rows& r) {
      for (int i = 0; i < r.nreq; ++i) r.req[i] += r0;
      return launch_kv4_append(r, pool, d->n_kv_heads, d->head_dim, d->dtype == SD_DTYPE_F32, k_new, k_stride, v_new,
                               v_stride, static_cast<hipStream_t>(stream));
    });
    if (st != SD_OK) return st;
  }
  return SD_OK;
}

int sd_kv4_read(const sd_dims_t* d, const sd_kv4_cache_t* cache, const int32_t* first, const int32_t* count,
                const int64_t* out_off, void* k_out, int64_t k_stride, void* v_out, int64_t v_stride,
                sd_stream_t stream) {
  int st = check_heads(d);
  if (st != SD_OK) return st;
  st = check_cache(cache);
  if (st != SD_OK) return st;
  if (!first || !count || !out_off || (!k_out && !v_out)) return SD_ERR_INVALID_ARGUMENT;
  if ((k_out && !rows_ok(d, k_out, k_stride)) || (v_out && !rows_ok(d, v_out, v_stride))) return SD_ERR_INVALID_ARGUMENT;
  for (int b = 0; b < d->batch; ++b)
    if (out_off[b] < 0 || first[b] < 0 || count[b] < 0 || !length_ok(cache, int64_t(first[b]) + count[b]))
      return SD_ERR_INVALID_ARGUMENT;
  const Kv4Pool pool = pool_of(cache);
  return over_rows(d, first, count, out_off, [&](Kv4Rows& r) {
    return launch_kv4_read(r, pool, d->n_kv_heads, d->head_dim, d->dtype == SD_DTYPE_F32, k_out, k_stride, v_out,
                           v_stride, static_cast<hipStream_t>(stream));
  });
}

int sd_verify_attention_kv4(const sd_dims_t* d, const void* q, const sd_kv4_cache_t* cache, const int32_t* kv_len,
                            const int32_t* parent, float scale, void* out, void* workspace, size_t workspace_bytes,
                            sd_stream_t stream) {
  int st = check_attention(d);
  if (st != SD_OK) return st;
  st = check_cache(cache);
  if (st != SD_OK) return st;
  if (!q || !kv_len || !out || !workspace) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || (parent != nullptr && !aligned(parent, 4)))
    return SD_ERR_INVALID_ARGUMENT;
  if (!scale_ok(scale)) return SD_ERR_INVALID_ARGUMENT;
  const int G = d->gamma + 1;
  for (int b = 0; b < d->batch; ++b)
    if (kv_len[b] < G || !length_ok(cache, kv_len[b])) return SD_ERR_INVALID_ARGUMENT;
  const AttnShape s = kv4_shape(G, d->n_q_heads, d->n_kv_heads, d->head_dim, scale, kv_len, d->batch);
  const int64_t chunks = s.chunk_keys > 0 ? count_chunks(kv_len, d->batch, s.chunk_keys) : 0;
  if (chunks * s.Hkv * s.row_groups > kMaxGrid) return SD_ERR_UNSUPPORTED;
  if (workspace_bytes < attention_ws(s, chunks)) return SD_ERR_WORKSPACE;
  const AttnPartials parts = attn_carve(workspace, chunks, s.Hkv, s.rows, s.D);
  const Kv4Pool pool = pool_of(cache);
  hipStream_t stm = static_cast<hipStream_t>(stream);
  int32_t base = 0;
  for (int r0 = 0; r0 < d->batch; r0 += kMaxReqPerLaunch) {
    AttnBatch bt;
    memset(&bt, 0, sizeof(bt));
    bt.nreq = std::min(kMaxReqPerLaunch, d->batch - r0);
    bt.req0 = r0;
    bt.chunk_base = base;
    bt.parent = d->gamma > 0 ? parent : nullptr;
    for (int i = 0; i < bt.nreq; ++i) {
      bt.kv_len[i] = kv_len[r0 + i];
      bt.chunk_prefix[i + 1] = s.chunk_keys > 0 ? bt.chunk_prefix[i] + (kv_len[r0 + i] + s.chunk_keys - 1) / s.chunk_keys : 0;
    }
    if (launch_kv4_attention(s, bt, pool, bt.chunk_prefix[bt.nreq], q, parts, out, stm) != hipSuccess)
      return SD_ERR_HIP;
    base += bt.chunk_prefix[bt.nreq];
  }
  return SD_OK;
}

}  // extern "C"
