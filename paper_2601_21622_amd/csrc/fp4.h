// Host-side launchers of the 4-bit kernels (internal to the library), and the
// device helpers that they share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.h"
#include "launch.h"

namespace sdv {

constexpr int kKeyBlock4 = 64;  // keys of a block
constexpr int kGroup4 = 32;     // columns of a key's scale
constexpr int kTile = 16;       // keys of a tile: a score tile of the attention, a wave's work elsewhere

struct Kv4Pool {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scale;
  uint16_t* v_scale;
  const int32_t* table;
  int32_t max_pages, page_shift, num_pages;
};

// Requests of one append or read launch: keys first .. first + count - 1 are rows off .. .
// A wave takes a tile of 16 keys, the first of them a multiple of 16; `prefix` counts the
// tiles that a request takes.
struct Kv4Rows {
  int32_t nreq;
  int32_t req[kMaxReqPerLaunch];  // rows of the block table
  int32_t prefix[kMaxReqPerLaunch + 1];
  int32_t first[kMaxReqPerLaunch];
  int32_t count[kMaxReqPerLaunch];
  int64_t off[kMaxReqPerLaunch];
};
hipError_t launch_kv4_append(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int D, bool f32, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t stream);
hipError_t launch_kv4_read(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int D, bool f32, void* k_out,
                           int64_t k_stride, void* v_out, int64_t v_stride, hipStream_t stream);

// Attention over a 4-bit cache.  kv4_shape fills an AttnShape for these lengths
// (chunks are whole 64-key blocks; none, chunk_keys 0, where a workgroup takes a whole
// request and writes the output itself); kv4_max_chunks bounds the chunk count of any
// lengths up to max_kv_len.  AttnBatch is used without kv_off and pages.
AttnShape kv4_shape(int G, int Hq, int Hkv, int D, float scale, const int32_t* kv_len, int B);
int64_t kv4_max_chunks(int Hkv, int D, int B, int64_t max_kv_len);
hipError_t launch_kv4_attention(const AttnShape& s, const AttnBatch& batch, const Kv4Pool& pool, int nchunks,
                                const void* q, AttnPartials parts, void* out, hipStream_t stream);

// Queries' and keys' norms and rotation.
struct RopeArgs {
  int32_t rows, Hq, Hkv, rotary;
  float eps;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
};
hipError_t launch_qk_rope(const RopeArgs& a, int D, bool f32, bool interleaved, const void* q, const void* k,
                          const int32_t* positions, const float* inv_freq, const void* q_weight, const void* k_weight,
                          void* q_out, void* k_out, hipStream_t stream);

// Byte `sel` of a dword of codes as a bfloat16 pair, each times 2^e of the power of two
// `scale` (exact: e2m1 has one fraction bit); infinity as the scale gives NaN.
template <int sel>
__device__ __forceinline__ uint32_t widen2_fp4(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, sel));
}
// The eight codes of a dword as one MFMA operand.
__device__ __forceinline__ bf16x8 widen8_fp4(uint32_t codes, float scale) {
  const u32x4 r = {widen2_fp4<0>(codes, scale), widen2_fp4<1>(codes, scale), widen2_fp4<2>(codes, scale),
                   widen2_fp4<3>(codes, scale)};
  return __builtin_bit_cast(bf16x8, r);
}

// Eight float32 values over the power of two `scale` as e2m1 codes (nearest, ties to even).
__device__ __forceinline__ uint32_t encode8_fp4(const float (&x)[8], float scale) {
  uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}

// Eight consecutive elements, 16-byte aligned, as float32.
template <typename T>
__device__ __forceinline__ void load_row8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load_row8<uint16_t>(const uint16_t* p, float (&v)[8]) {
  const u32x4 r = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void load_row8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
  const f32x4 b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
// Rounded to the element type and stored.
template <typename T>
__device__ __forceinline__ void store_row8(T* p, const float (&v)[8]);
template <>
__device__ __forceinline__ void store_row8<uint16_t>(uint16_t* p, const float (&v)[8]) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (__bf16)v[i];
  *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, r);
}
template <>
__device__ __forceinline__ void store_row8<float>(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

}  // namespace sdv
