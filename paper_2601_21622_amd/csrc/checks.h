// Argument checks that the calls over quantised caches share (host only).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <cmath>

#include "common.h"
#include "launch.h"
#include "sdverify.h"

namespace sdv {

constexpr int kMaxRows = 128;  // G * (Hq / Hkv)
constexpr int kMaxGamma = 63;
constexpr int64_t kMaxKvLen = int64_t(1) << 30;
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;  // workgroups along x

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

inline int check_heads(const sd_dims_t* d) {
  if (d == nullptr || d->batch < 1 || d->n_kv_heads < 1 || d->head_dim < 1 || d->flags != 0) return SD_ERR_INVALID_ARGUMENT;
  if (d->dtype != SD_DTYPE_F32 && d->dtype != SD_DTYPE_BF16) return SD_ERR_INVALID_ARGUMENT;
  if (d->head_dim != 64 && d->head_dim != 128) return SD_ERR_UNSUPPORTED;
  if (d->n_kv_heads > 65535 || d->batch > (1 << 24)) return SD_ERR_UNSUPPORTED;
  return SD_OK;
}

inline int check_attention(const sd_dims_t* d) {
  const int st = check_heads(d);
  if (st != SD_OK) return st;
  if (d->gamma < 0 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads != 0) return SD_ERR_INVALID_ARGUMENT;
  if (d->dtype != SD_DTYPE_BF16 || d->gamma > kMaxGamma) return SD_ERR_UNSUPPORTED;
  if (int64_t(d->gamma + 1) * (d->n_q_heads / d->n_kv_heads) > kMaxRows) return SD_ERR_UNSUPPORTED;
  return SD_OK;
}

// The kernels work with scale * log2 e.
inline bool scale_ok(float scale) { return scale > 0.f && std::isfinite(scale * kLog2e); }

inline size_t attention_ws(const AttnShape& s, int64_t chunks) {
  return align_up(attn_partial_bytes(chunks, s.Hkv, s.rows, s.D));
}

inline int64_t count_chunks(const int32_t* kv_len, int n, int keys) {
  int64_t c = 0;
  for (int i = 0; i < n; ++i) c += (kv_len[i] + keys - 1) / keys;
  return c;
}

}  // namespace sdv
