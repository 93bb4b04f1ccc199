// Host-side launchers of the 8-bit kernels (internal to the library), and the
// device helpers that they share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.h"
#include "launch.h"

namespace sdv {

constexpr int kKeyBlock = 64;   // keys per cache scale
constexpr int kColBlock = 128;  // columns per hidden or weight scale

struct Kv8Pool {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  const int32_t* table;
  int32_t max_pages, page_shift, num_pages;
};

// Requests of one append launch; blk_prefix counts the 64-key blocks each touches.
struct Kv8Append {
  int32_t nreq;
  int32_t req[kMaxReqPerLaunch];  // rows of the block table
  int32_t blk_prefix[kMaxReqPerLaunch + 1];
  int32_t kv_len[kMaxReqPerLaunch];
  int32_t new_len[kMaxReqPerLaunch];
  int64_t new_off[kMaxReqPerLaunch];
};
hipError_t launch_kv8_append(const Kv8Append& a, const Kv8Pool& pool, int Hkv, int D, bool f32, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t stream);

// Attention over an 8-bit cache.  kv8_shape fills an AttnShape for these
// lengths (chunks are whole 64-key blocks); kv8_max_chunks bounds the chunk
// count of any lengths up to max_kv_len.  AttnBatch is used without kv_off and
// pages.
AttnShape kv8_shape(int G, int Hq, int Hkv, int D, float scale, const int32_t* kv_len, int B);
int64_t kv8_max_chunks(int Hkv, int D, int B, int64_t max_kv_len);
hipError_t launch_kv8_attention(const AttnShape& s, const AttnBatch& batch, const Kv8Pool& pool, int nchunks,
                                const void* q, AttnPartials parts, void* out, hipStream_t stream);

hipError_t launch_residual_norm(bool f32, int rows, int width, float eps, const void* x, const void* residual,
                                const void* weight, void* new_residual, uint8_t* out, float* out_scale,
                                hipStream_t stream);

// The projection's tiles for M rows, K columns, V entries.
struct Fp8Plan {
  int M, K, V;
  int mb, nw;       // 32-row blocks, and blocks of 32 entries, per tile
  int mtiles, ntiles;
};
Fp8Plan fp8_plan(int M, int K, int V);
size_t fp8_logits_bytes(int M, int V);
hipError_t launch_logits_fp8(const Fp8Plan& p, const void* hidden, const float* hidden_scale, const void* w,
                             const float* w_scale, float* logits, float* row_lse, void* ws, hipStream_t stream);

// Four codes of a dword, as bfloat16 pairs, each times 2^e of the power of two
// `scale` (exact: e4m3 has three fraction bits, bfloat16 seven and float32's range).
__device__ __forceinline__ uint32_t widen_lo(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true));
}
// Eight codes (two dwords) as one MFMA operand.
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float scale) {
  const u32x4 r = {widen_lo(a, scale), widen_hi(a, scale), widen_lo(b, scale), widen_hi(b, scale)};
  return __builtin_bit_cast(bf16x8, r);
}

// Four float32 values rounded to e4m3 (nearest, ties to even; NaN past 464).
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

}  // namespace sdv
