// C-ABI of the 8-bit calls (sdverify_fp8.h): argument checks, workspace and
// launches.  Every check runs on the host before anything is enqueued.
#include <string.h>

#include <algorithm>
#include <cmath>

#include "sdverify_fp8.h"
#include "fp8.h"

namespace {

using namespace sdv;

static_assert(SD_KV8_BLOCK == kKeyBlock && SD_FP8_BLOCK == kColBlock, "the header's blocks are the kernels'");

constexpr int kMaxRows = 128;  // G * (Hq / Hkv)
constexpr int kMaxGamma = 63;
constexpr int kMaxVocab = 2097152;
constexpr int64_t kMaxKvLen = int64_t(1) << 30;
constexpr int kMaxWidth = 32768;   // of a normed row
constexpr int kMaxHidden = 1 << 23;  // a tile of 256 rows within 32-bit offsets
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;  // workgroups along x

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

int check_heads(const sd_dims_t* d) {
  if (d == nullptr || d->batch < 1 || d->n_kv_heads < 1 || d->head_dim < 1 || d->flags != 0) return SD_ERR_INVALID_ARGUMENT;
  if (d->dtype != SD_DTYPE_F32 && d->dtype != SD_DTYPE_BF16) return SD_ERR_INVALID_ARGUMENT;
  if (d->head_dim != 64 && d->head_dim != 128) return SD_ERR_UNSUPPORTED;
  if (d->n_kv_heads > 65535 || d->batch > (1 << 24)) return SD_ERR_UNSUPPORTED;
  return SD_OK;
}

int check_attention(const sd_dims_t* d) {
  const int st = check_heads(d);
  if (st != SD_OK) return st;
  if (d->gamma < 0 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads != 0) return SD_ERR_INVALID_ARGUMENT;
  if (d->dtype != SD_DTYPE_BF16 || d->gamma > kMaxGamma) return SD_ERR_UNSUPPORTED;
  if (int64_t(d->gamma + 1) * (d->n_q_heads / d->n_kv_heads) > kMaxRows) return SD_ERR_UNSUPPORTED;
  return SD_OK;
}

int check_projection(const sd_dims_t* d) {
  if (d == nullptr || d->batch < 1 || d->gamma < 0 || d->hidden < 1 || d->vocab < 1 || d->flags != 0)
    return SD_ERR_INVALID_ARGUMENT;
  if (d->hidden % 32 != 0 || d->hidden > kMaxHidden || d->vocab > kMaxVocab) return SD_ERR_UNSUPPORTED;
  if (int64_t(d->batch) * (int64_t(d->gamma) + 1) > (int64_t(1) << 24)) return SD_ERR_UNSUPPORTED;
  return SD_OK;
}

int check_cache(const sd_kv8_cache_t* c) {
  if (c == nullptr || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->block_table) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->block_table, 4)) return SD_ERR_INVALID_ARGUMENT;
  if (c->page_size < 64 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0) return SD_ERR_INVALID_ARGUMENT;
  if (c->max_pages < 1 || c->num_pages < 1) return SD_ERR_INVALID_ARGUMENT;
  return SD_OK;
}

bool length_ok(const sd_kv8_cache_t* c, int32_t n) {
  return n <= kMaxKvLen && int64_t(n) <= int64_t(c->max_pages) * c->page_size;
}

Kv8Pool pool_of(const sd_kv8_cache_t* c) {
  Kv8Pool p;
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

size_t attention_ws(const AttnShape& s, int64_t chunks) {
  return align_up(attn_partial_bytes(chunks, s.Hkv, s.rows, s.D));
}

int64_t count_chunks(const int32_t* kv_len, int n, int keys) {
  int64_t c = 0;
  for (int i = 0; i < n; ++i) c += (kv_len[i] + keys - 1) / keys;
  return c;
}

}  // namespace

extern "C" {

size_t sd_fp8_workspace_bytes(const sd_dims_t* d, int32_t max_kv_len) {
  size_t n = 0;
  if (check_attention(d) == SD_OK && max_kv_len > d->gamma && max_kv_len <= kMaxKvLen) {
    const int rows = (d->gamma + 1) * (d->n_q_heads / d->n_kv_heads);
    const int64_t chunks = kv8_max_chunks(d->n_kv_heads, d->head_dim, d->batch, max_kv_len);
    n = align_up(attn_partial_bytes(chunks, d->n_kv_heads, rows, d->head_dim));
  }
  if (check_projection(d) == SD_OK)
    n = std::max(n, align_up(fp8_logits_bytes(d->batch * (d->gamma + 1), d->vocab)));
  return n;
}

int sd_kv8_append(const sd_dims_t* d, const sd_kv8_cache_t* cache, const void* k_new, int64_t k_stride,
                  const void* v_new, int64_t v_stride, const int64_t* new_off, const int32_t* new_len,
                  const int32_t* kv_len, sd_stream_t stream) {
  int st = check_heads(d);
  if (st != SD_OK) return st;
  st = check_cache(cache);
  if (st != SD_OK) return st;
  if (!k_new || !v_new || !new_off || !new_len || !kv_len) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(k_new, 16) || !aligned(v_new, 16)) return SD_ERR_INVALID_ARGUMENT;
  const int64_t unit = d->dtype == SD_DTYPE_F32 ? 4 : 8, row = int64_t(d->n_kv_heads) * d->head_dim;
  if (k_stride < row || v_stride < row || k_stride % unit != 0 || v_stride % unit != 0) return SD_ERR_INVALID_ARGUMENT;
  for (int b = 0; b < d->batch; ++b)
    if (new_off[b] < 0 || new_len[b] < 0 || new_len[b] > kv_len[b] || !length_ok(cache, kv_len[b]))
      return SD_ERR_INVALID_ARGUMENT;
  const Kv8Pool pool = pool_of(cache);
  // Requests with rows to append, as many per launch as its table and its grid hold.
  Kv8Append a;
  memset(&a, 0, sizeof(a));
  for (int b = 0; b < d->batch; ++b) {
    if (new_len[b] > 0) {
      const int64_t blocks = (int64_t(kv_len[b]) + kKeyBlock - 1) / kKeyBlock - (kv_len[b] - new_len[b]) / kKeyBlock;
      if (blocks * d->n_kv_heads * 2 > kMaxGrid) return SD_ERR_UNSUPPORTED;
    }
  }
  for (int b = 0; b < d->batch; ++b) {
    if (new_len[b] > 0) {
      const int blocks = (kv_len[b] + kKeyBlock - 1) / kKeyBlock - (kv_len[b] - new_len[b]) / kKeyBlock;
      if (a.nreq == kMaxReqPerLaunch || (a.blk_prefix[a.nreq] + int64_t(blocks)) * d->n_kv_heads * 2 > kMaxGrid) {
        if (launch_kv8_append(a, pool, d->n_kv_heads, d->head_dim, d->dtype == SD_DTYPE_F32, k_new, k_stride, v_new,
                              v_stride, static_cast<hipStream_t>(stream)) != hipSuccess)
          return SD_ERR_HIP;
        a.nreq = 0;
      }
      a.req[a.nreq] = b;
      a.kv_len[a.nreq] = kv_len[b];
      a.new_len[a.nreq] = new_len[b];
      a.new_off[a.nreq] = new_off[b];
      a.blk_prefix[a.nreq + 1] = a.blk_prefix[a.nreq] + blocks;
      ++a.nreq;
    }
  }
  if (a.nreq > 0 &&
      launch_kv8_append(a, pool, d->n_kv_heads, d->head_dim, d->dtype == SD_DTYPE_F32, k_new, k_stride, v_new,
                        v_stride, static_cast<hipStream_t>(stream)) != hipSuccess)
    return SD_ERR_HIP;
  return SD_OK;
}

int sd_verify_attention_kv8(const sd_dims_t* d, const void* q, const sd_kv8_cache_t* cache, const int32_t* kv_len,
                            const int32_t* parent, float scale, void* out, void* workspace, size_t workspace_bytes,
                            sd_stream_t stream) {
  int st = check_attention(d);
  if (st != SD_OK) return st;
  st = check_cache(cache);
  if (st != SD_OK) return st;
  if (!q || !kv_len || !out || !workspace) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || (parent != nullptr && !aligned(parent, 4)))
    return SD_ERR_INVALID_ARGUMENT;
  if (!(scale > 0.f) || !std::isfinite(scale)) return SD_ERR_INVALID_ARGUMENT;
  const int G = d->gamma + 1;
  for (int b = 0; b < d->batch; ++b)
    if (kv_len[b] < G || !length_ok(cache, kv_len[b])) return SD_ERR_INVALID_ARGUMENT;
  const AttnShape s = kv8_shape(G, d->n_q_heads, d->n_kv_heads, d->head_dim, scale, kv_len, d->batch);
  const int64_t chunks = count_chunks(kv_len, d->batch, s.chunk_keys);
  if (chunks * s.Hkv * s.row_groups > kMaxGrid) return SD_ERR_UNSUPPORTED;
  if (workspace_bytes < attention_ws(s, chunks)) return SD_ERR_WORKSPACE;
  const AttnPartials parts = attn_carve(workspace, chunks, s.Hkv, s.rows, s.D);
  const Kv8Pool pool = pool_of(cache);
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
      bt.chunk_prefix[i + 1] = bt.chunk_prefix[i] + (kv_len[r0 + i] + s.chunk_keys - 1) / s.chunk_keys;
    }
    if (launch_kv8_attention(s, bt, pool, bt.chunk_prefix[bt.nreq], q, parts, out, stm) != hipSuccess)
      return SD_ERR_HIP;
    base += bt.chunk_prefix[bt.nreq];
  }
  return SD_OK;
}

int sd_residual_norm_fp8(const sd_norm_t* n, const void* x, const void* residual, const void* weight,
                         void* new_residual, void* out, float* out_scale, sd_stream_t stream) {
  if (n == nullptr || n->rows < 1 || n->width < 1 || !(n->eps >= 0.f) || !std::isfinite(n->eps))
    return SD_ERR_INVALID_ARGUMENT;
  if (n->dtype != SD_DTYPE_F32 && n->dtype != SD_DTYPE_BF16) return SD_ERR_INVALID_ARGUMENT;
  if (n->width % 32 != 0 || n->width > kMaxWidth || n->rows > (1 << 24)) return SD_ERR_UNSUPPORTED;
  if (!x || !weight || !out || !out_scale) return SD_ERR_INVALID_ARGUMENT;
  const void* p16[] = {x, residual, weight, new_residual, out};
  for (const void* p : p16)
    if (p != nullptr && !aligned(p, 16)) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(out_scale, 4)) return SD_ERR_INVALID_ARGUMENT;
  return launch_residual_norm(n->dtype == SD_DTYPE_F32, n->rows, n->width, n->eps, x, residual, weight, new_residual,
                              static_cast<uint8_t*>(out), out_scale, static_cast<hipStream_t>(stream)) == hipSuccess
             ? SD_OK
             : SD_ERR_HIP;
}

int sd_verify_logits_fp8(const sd_dims_t* d, const void* hidden, const float* hidden_scale, const void* w,
                         const float* w_scale, float* logits, float* row_lse, void* workspace, size_t workspace_bytes,
                         sd_stream_t stream) {
  const int st = check_projection(d);
  if (st != SD_OK) return st;
  if (!hidden || !hidden_scale || !w || !w_scale || !logits || !row_lse || !workspace) return SD_ERR_INVALID_ARGUMENT;
  if (!aligned(hidden, 16) || !aligned(w, 16) || !aligned(logits, 16) || !aligned(workspace, 16) ||
      !aligned(hidden_scale, 4) || !aligned(w_scale, 4) || !aligned(row_lse, 4))
    return SD_ERR_INVALID_ARGUMENT;
  const Fp8Plan p = fp8_plan(d->batch * (d->gamma + 1), d->hidden, d->vocab);
  if (int64_t(p.ntiles + 7) * p.mtiles > kMaxGrid) return SD_ERR_UNSUPPORTED;
  if (workspace_bytes < fp8_logits_bytes(p.M, p.V)) return SD_ERR_WORKSPACE;
  return launch_logits_fp8(p, hidden, hidden_scale, w, w_scale, logits, row_lse, workspace,
                           static_cast<hipStream_t>(stream)) == hipSuccess
             ? SD_OK
             : SD_ERR_HIP;
}

}  // extern "C"
