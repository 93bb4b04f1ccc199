// Appending key and value rows to a paged 4-bit cache, and reading them back (gfx950).
//
// No scale spans keys, so a key is its own unit and nothing in the cache is read
// when one is written.  A thread holds eight columns of one key: the 32 columns of a
// key's scale are four threads, a value's row D / 8, and eight codes are one dword.
#include <algorithm>

#include "fp4.h"

namespace sdv {

namespace {

constexpr int kRowThreads = 256;
constexpr int kLowestExp4 = 27;  // byte of the smallest scale, 2^-100
constexpr uint32_t kInfBits = 0x7f800000u;

// One thread's eight columns of one key.
template <int D>
struct Place {
  bool is_v, mine;  // mine: the key is one of the request's
  int head, col;
  int key;          // of its block
  int64_t block;    // of the pool: [page][head][block]
  int64_t row;      // of the rows
};

template <int D>
__device__ __forceinline__ Place<D> place_of(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int unit) {
  constexpr int TPR = D / 8;
  constexpr int kKeys = kv4_keys_per_wave(D);
  const int lane = threadIdx.x & 63;
  const int waves = r.prefix[r.nreq];
  const int c = unit % waves, hv = unit / waves;
  // The largest request with prefix <= c: one load, a request per lane.
  const int prefix = lane < r.nreq ? r.prefix[lane] : INT32_MAX;
  const int lo = __popcll(__ballot(prefix <= c)) - 1;
  const int first = r.first[lo], end = first + r.count[lo];
  const int key0 = (first / kKeys + c - __builtin_amdgcn_readlane(prefix, lo)) * kKeys;
  Place<D> p;
  p.is_v = hv >= Hkv;
  p.head = p.is_v ? hv - Hkv : hv;
  p.col = lane % TPR * 8;
  const int key = key0 + lane / TPR;
  p.mine = key >= first && key < end;
  const int at = min(max(key, first), end - 1);  // a key of the request's is read in its place
  p.row = r.off[lo] + (at - first);
  const int shift = pool.page_shift - 6, blk = at / kKeyBlock4;
  int page = pool.table[(int64_t)r.req[lo] * pool.max_pages + (blk >> shift)];
  page = min(max(page, 0), pool.num_pages - 1);
  p.block = (((int64_t)page * Hkv + p.head) << shift) + (blk & ((1 << shift) - 1));
  p.key = at % kKeyBlock4;
  return p;
}

// Where the dword of the codes of columns col .. + 7 of a key lies in its block.
template <int D>
__device__ __forceinline__ int k_dword(int key, int col) {  // [4 t][4 g][16 r][D/8 bytes]
  return (((key / 16 * 4 + col / (D / 4)) * 16 + key % 16) * (D / 8) + col % (D / 4) / 2) / 4;
}
__device__ __forceinline__ int v_dword(int key, int col) {  // [D/16][64 n][8 bytes]
  return (col / 16 * 64 + key) * 2 + col % 16 / 8;
}
__device__ __forceinline__ int k_scale_byte(int key, int col) {  // [D/32][16 r][4 t]
  return (col / kGroup4 * 16 + key % 16) * 4 + key / 16;
}

// Largest over the four threads of a key's scale.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp_u32<kDppXor1>(v));
  return max(v, dpp_u32<kDppXor2>(v));
}
// And over the threads of a value's row.
template <int D>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(quad_max(v), dpp_u32<kDppRowHalfMirror>(quad_max(v)));
  return D == 128 ? max(v, dpp_u32<kDppRowMirror>(v)) : v;
}

// Smallest exponent byte, at least 27, with x <= 6 * 2^(byte - 127); x by its bits.
// 6 = 1.5 * 2^2.
__device__ __forceinline__ int key_scale(uint32_t x) {
  return max((int)(x >> 23) - 2 + ((x & 0x7fffffu) > 0x400000u ? 1 : 0), kLowestExp4);
}

// Smallest bfloat16 s, at least 2^-100, with x <= 6 s (6 s is exact).  The product with
// 1/6 is off by less than a bfloat16 step, so that the truncated one is at most two below.
__device__ __forceinline__ float value_scale(float x) {
  uint32_t b = __float_as_uint(x * (1.f / 6.f)) & 0xffff0000u;
#pragma unroll
  for (int i = 0; i < 2; ++i) b += 6.f * __uint_as_float(b) < x ? 0x10000u : 0u;
  return fmaxf(__uint_as_float(b), 0x1p-100f);
}

// x / s for the code's rounding: the quotient rounded, which is exact where the true one
// is a border between codes (borders have three bits, s eight).  A float32 x may lie so near a
// border that the rounded quotient is the border: then the remainder's sign moves it off.
template <typename T>
__device__ __forceinline__ float over_scale(float x, float s, float inv) {
  float r = x * inv;
  r = fmaf(fmaf(-r, s, x), inv, r);
  if (sizeof(T) == 4) {
    const uint32_t b = __float_as_uint(r);
    const float rest = fmaf(-r, s, x);
    if ((b & 0x1fffffu) == 0 && rest != 0.f) r = __uint_as_float((rest > 0.f) == (x > 0.f) ? b + 1 : b - 1);
  }
  return __builtin_copysignf(r, x);  // of zeros too
}

template <typename T, int D>
__global__ __launch_bounds__(kRowThreads)
void kv4_append_kernel(Kv4Rows rows, Kv4Pool pool, int Hkv, int nunits, const T* __restrict__ k_new,
                       int64_t k_stride, const T* __restrict__ v_new, int64_t v_stride) {
  const int unit = blockIdx.x * (kRowThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= nunits) return;
  const Place<D> p = place_of<D>(rows, pool, Hkv, unit);
  float x[8];
  load_row8((p.is_v ? v_new + p.row * v_stride : k_new + p.row * k_stride) + p.head * D + p.col, x);
  uint32_t most = 0;  // of the magnitudes' bits, whose order is theirs, infinities and NaN last
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  if (p.is_v) {
    most = row_max<D>(most);
    const bool number = most < kInfBits;
    const float s = value_scale(number ? __uint_as_float(most) : 0.f), inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = number ? over_scale<T>(x[i], s, inv) : 0.f;
    if (p.mine) {
      reinterpret_cast<uint32_t*>(pool.v)[p.block * (8 * D) + v_dword(p.key, p.col)] = encode8_fp4(x, 1.f);
      if (p.col == 0) pool.v_scale[p.block * 64 + p.key] = number ? (uint16_t)(__float_as_uint(s) >> 16) : 0x7fc0;
    }
  } else {
    most = quad_max(most);
    const bool number = most < kInfBits;
    const int e = key_scale(number ? most : 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = number ? x[i] : 0.f;
    if (p.mine) {
      reinterpret_cast<uint32_t*>(pool.k)[p.block * (8 * D) + k_dword<D>(p.key, p.col)] =
          encode8_fp4(x, __uint_as_float((uint32_t)e << 23));
      if (p.col % kGroup4 == 0) pool.k_scale[p.block * (2 * D) + k_scale_byte(p.key, p.col)] = number ? (uint8_t)e : 255;
    }
  }
}

// The two values of byte `sel`, times a power of two.
template <int sel>
__device__ __forceinline__ void decode2(uint32_t codes, float scale, float (&x)[8]) {
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, sel);
  x[2 * sel] = v[0];
  x[2 * sel + 1] = v[1];
}

template <typename T, int D>
__global__ __launch_bounds__(kRowThreads)
void kv4_read_kernel(Kv4Rows rows, Kv4Pool pool, int Hkv, int nunits, int unit0, T* __restrict__ k_out, int64_t k_stride,
                     T* __restrict__ v_out, int64_t v_stride) {
  const int unit = unit0 + blockIdx.x * (kRowThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= nunits) return;
  const Place<D> p = place_of<D>(rows, pool, Hkv, unit);
  const uint32_t codes = reinterpret_cast<const uint32_t*>(
      p.is_v ? pool.v : pool.k)[p.block * (8 * D) + (p.is_v ? v_dword(p.key, p.col) : k_dword<D>(p.key, p.col))];
  const float scale =
      p.is_v ? bf16_to_f32(pool.v_scale[p.block * 64 + p.key])
             : __uint_as_float((uint32_t)pool.k_scale[p.block * (2 * D) + k_scale_byte(p.key, p.col)] << 23);
  float x[8];
  const float pow2 = p.is_v ? 1.f : scale;
  decode2<0>(codes, pow2, x);
  decode2<1>(codes, pow2, x);
  decode2<2>(codes, pow2, x);
  decode2<3>(codes, pow2, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = p.is_v ? x[i] * scale : x[i];
  if (p.mine) store_row8((p.is_v ? v_out + p.row * v_stride : k_out + p.row * k_stride) + p.head * D + p.col, x);
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int D, bool f32, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t stream) {
  const int nunits = r.prefix[r.nreq] * Hkv * 2;
  const dim3 grid((nunits + kRowThreads / kWave - 1) / (kRowThreads / kWave)), block(kRowThreads);
#define SDV_APPEND(T, DIM)                                                                                       \
  hipLaunchKernelGGL((kv4_append_kernel<T, DIM>), grid, block, 0, stream, r, pool, Hkv, nunits,                  \
                     static_cast<const T*>(k_new), k_stride, static_cast<const T*>(v_new), v_stride)
  if (f32 && D == 128) {
    SDV_APPEND(float, 128);
  } else if (f32) {
    SDV_APPEND(float, 64);
  } else if (D == 128) {
    SDV_APPEND(uint16_t, 128);
  } else {
    SDV_APPEND(uint16_t, 64);
  }
#undef SDV_APPEND
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int D, bool f32, void* k_out,
                           int64_t k_stride, void* v_out, int64_t v_stride, hipStream_t stream) {
  const int half = r.prefix[r.nreq] * Hkv;  // units of K; those of V follow
  const int begin = k_out != nullptr ? 0 : half, end = v_out != nullptr ? 2 * half : half;
  const dim3 grid((end - begin + kRowThreads / kWave - 1) / (kRowThreads / kWave)), block(kRowThreads);
#define SDV_READ(T, DIM)                                                                                         \
  hipLaunchKernelGGL((kv4_read_kernel<T, DIM>), grid, block, 0, stream, r, pool, Hkv, end, begin,                \
                     static_cast<T*>(k_out), k_stride, static_cast<T*>(v_out), v_stride)
  if (f32 && D == 128) {
    SDV_READ(float, 128);
  } else if (f32) {
    SDV_READ(float, 64);
  } else if (D == 128) {
    SDV_READ(uint16_t, 128);
  } else {
    SDV_READ(uint16_t, 64);
  }
#undef SDV_READ
  return hipGetLastError();
}

}  // namespace sdv
