// Appending key and value rows to a paged 4-bit cache, and reading them back (gfx950).
//
// No scale spans keys, so a key is its own unit and nothing in the cache is read
// when one is written.  A wave takes 16 keys of a block (a tile) and one KV head, K and V
// both: D / 8 threads hold a row of eight columns each, so that rows are read and written
// whole; on the cache's side a tile of K is 16 D / 2 bytes in a row and a tile of V 128 bytes
// in each of the D / 16 column groups, and the two orders meet in LDS.
//
// Bound by memory where there are many keys: appending 8 prompts of 1 to 6,001 bf16 rows (8 heads, D = 128, 124 MB) takes
// 26 us, 4.8 TB/s, and reading 8 sessions of 1 to 9,001 keys 39.5 us, 4.7 TB/s; a large copy's rate is 4.7-4.9.  In float32
// they take 47.7 us, 4.7 TB/s, and 88.5 us, 3.8 TB/s.  With a dword
// a thread and a wave per four keys, and no LDS, they took 40 and 71.  Steps of a few keys are bound by latency: 5 keys
// of 64 requests, 32 heads, 5.5 us (table, rows and stores, one behind the other).
#include <type_traits>

#include "fp4.h"

namespace sdv {

namespace {

constexpr int kRowThreads = 256;
constexpr int kLowestExp4 = 27;  // byte of the smallest scale, 2^-100
// Largest scales with which 6 stands for a finite float32: 2^125 of keys, by its byte, and 170 * 2^118 of values (6 of it is
// bfloat16's largest number).  With the next ones finite rows would come back infinite; elements past 6 of them become 6.
constexpr int kHighestExp4 = 252;
constexpr float kHighestScale4 = 0x1.54p125f;
constexpr uint32_t kInfBits = 0x7f800000u;

// A wave's tile.
struct Tile {
  int head;
  int key0;       // of its block: 0, 16, 32 or 48
  int from, to;   // keys key0 + from .. key0 + to - 1 are the request's
  int64_t block;  // of the pool: [page][head][block]
  int64_t row0;   // row of key0
};

__device__ __forceinline__ Tile tile_of(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int unit) {
  const int lane = threadIdx.x & 63;
  Tile t;
  t.head = unit % Hkv;
  const int c = unit / Hkv;
  // The largest request with prefix <= c: one load, a request per lane.
  const int prefix = lane < r.nreq ? r.prefix[lane] : INT32_MAX;
  const int lo = __popcll(__ballot(prefix <= c)) - 1;
  const int first = r.first[lo], end = first + r.count[lo];
  const int key = (first / kTile + c - __builtin_amdgcn_readlane(prefix, lo)) * kTile;
  t.from = __builtin_amdgcn_readfirstlane(max(first - key, 0));
  t.to = __builtin_amdgcn_readfirstlane(min(end - key, kTile));
  t.row0 = r.off[lo] + (key - first);
  const int shift = pool.page_shift - 6, blk = key / kKeyBlock4;
  int page = pool.table[(int64_t)r.req[lo] * pool.max_pages + (blk >> shift)];
  page = min(max(page, 0), pool.num_pages - 1);
  t.block = (((int64_t)page * Hkv + t.head) << shift) + (blk & ((1 << shift) - 1));
  t.key0 = key % kKeyBlock4;
  return t;
}

// Where the dword of the codes of columns col .. + 7 of a tile's key lies among the tile's.
template <int D>
__device__ __forceinline__ int k_dword(int key, int col) {  // [4 g][16 r][D/8 bytes]
  return ((col / (D / 4) * 16 + key) * (D / 8) + col % (D / 4) / 2) / 4;
}
__device__ __forceinline__ int v_dword(int key, int col) {  // [D/16][16 n][8 bytes]
  return (col / 16 * kTile + key) * 2 + col % 16 / 8;
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

// Smallest exponent byte, 27 to 252, with x <= 6 * 2^(byte - 127); x by its bits.
// 6 = 1.5 * 2^2.
__device__ __forceinline__ int key_scale(uint32_t x) {
  return min(max((int)(x >> 23) - 2 + ((x & 0x7fffffu) > 0x400000u ? 1 : 0), kLowestExp4), kHighestExp4);
}

// Smallest bfloat16 s, 2^-100 to 170 * 2^118, with x <= 6 s (6 s is exact).  The product with
// 1/6 is off by less than a bfloat16 step, so that the truncated one is at most two below.
__device__ __forceinline__ float value_scale(float x) {
  uint32_t b = __float_as_uint(x * (1.f / 6.f)) & 0xffff0000u;
#pragma unroll
  for (int i = 0; i < 2; ++i) b += 6.f * __uint_as_float(b) < x ? 0x10000u : 0u;
  return fminf(fmaxf(__uint_as_float(b), 0x1p-100f), kHighestScale4);
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
  constexpr int TPR = D / 8, kKeys = kWave / TPR;  // threads of a row, keys at once
  constexpr int kRounds = kTile / kKeys;
  constexpr int kWords = kTile * D / 8;            // dwords of a tile of K, or of V
  __shared__ __align__(16) uint32_t image[kRowThreads / kWave][2 * kWords];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x * (kRowThreads / kWave) + wave;
  if (unit >= nunits) return;
  const Tile t = tile_of(rows, pool, Hkv, unit);
  const int lane = threadIdx.x & 63, col = lane % TPR * 8;
  uint32_t* const k_image = image[wave];
  uint32_t* const v_image = k_image + kWords;
  float k[kRounds][8], v[kRounds][8];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int key = min(max(i * kKeys + lane / TPR, t.from), t.to - 1);  // one of the request's is read in its place
    load_row8(k_new + (t.row0 + key) * k_stride + t.head * D + col, k[i]);
    load_row8(v_new + (t.row0 + key) * v_stride + t.head * D + col, v[i]);
  }
  uint8_t* const k_scale = pool.k_scale + t.block * (2 * D) + t.key0 / kTile;
  uint16_t* const v_scale = pool.v_scale + t.block * kKeyBlock4 + t.key0;
  // A tile of few keys skips the rounds without any; a whole one has no branches.
  auto encode = [&](auto whole) {
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      if (!decltype(whole)::value && (i * kKeys >= t.to || (i + 1) * kKeys <= t.from)) continue;
      const int key = i * kKeys + lane / TPR;
      const bool mine = key >= t.from && key < t.to;
      uint32_t most_k = 0, most_v = 0;  // of the magnitudes' bits, whose order is theirs, infinities and NaN last
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        most_k = max(most_k, __float_as_uint(k[i][e]) & 0x7fffffffu);
        most_v = max(most_v, __float_as_uint(v[i][e]) & 0x7fffffffu);
      }
      most_k = quad_max(most_k);
      most_v = row_max<D>(most_v);
      const bool k_number = most_k < kInfBits, v_number = most_v < kInfBits;
      const int byte = key_scale(k_number ? most_k : 0u);
      const float s = value_scale(v_number ? __uint_as_float(most_v) : 0.f), inv = 1.f / s;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = over_scale<T>(v[i][e], s, inv);
      k_image[k_dword<D>(key, col)] = k_number ? encode8_fp4(k[i], __uint_as_float((uint32_t)byte << 23)) : 0u;
      v_image[v_dword(key, col)] = v_number ? encode8_fp4(v[i], 1.f) : 0u;
      if (mine && col % kGroup4 == 0) k_scale[(col / kGroup4 * 16 + key) * 4] = k_number ? (uint8_t)byte : 255;  // [D/32][16 r][4 t]
      if (mine && col == 0) v_scale[key] = v_number ? (uint16_t)(__float_as_uint(s) >> 16) : 0x7fc0;
    }
  };
  if (t.to - t.from == kTile) encode(std::true_type());
  else encode(std::false_type());
  lds_wait();  // the wave's own image is whole
  uint8_t* const k_out = pool.k + t.block * (32 * D) + t.key0 * (D / 2);
  uint8_t* const v_out = pool.v + t.block * (32 * D) + t.key0 * 8;
  {
    // D / 8 bytes of each key and column group of K.
    const int key = lane % kTile;
    if (key >= t.from && key < t.to) {
      if (D == 128)
        reinterpret_cast<u32x4*>(k_out)[lane] = reinterpret_cast<const u32x4*>(k_image)[lane];
      else
        reinterpret_cast<u32x2*>(k_out)[lane] = reinterpret_cast<const u32x2*>(k_image)[lane];
    }
  }
  if (lane < D / 2) {  // two keys of 16 columns of V: 16 bytes
    const int i = lane / 8, key = lane % 8 * 2;
    const u32x4 w = reinterpret_cast<const u32x4*>(v_image)[lane];
    uint8_t* const dst = v_out + i * 512 + key * 8;
    const bool a = key >= t.from && key < t.to, b = key + 1 >= t.from && key + 1 < t.to;
    if (a && b)
      *reinterpret_cast<u32x4*>(dst) = w;
    else if (a)
      *reinterpret_cast<u32x2*>(dst) = u32x2{w[0], w[1]};
    else if (b)
      *reinterpret_cast<u32x2*>(dst + 8) = u32x2{w[2], w[3]};
  }
}

// The two values of byte `sel`, times a power of two.
template <int sel>
__device__ __forceinline__ void decode2(uint32_t codes, float scale, float (&x)[8]) {
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, sel);
  x[2 * sel] = v[0];
  x[2 * sel + 1] = v[1];
}
__device__ __forceinline__ void decode8(uint32_t codes, float scale, float (&x)[8]) {
  decode2<0>(codes, scale, x);
  decode2<1>(codes, scale, x);
  decode2<2>(codes, scale, x);
  decode2<3>(codes, scale, x);
}

// K and V: which of them are asked for.  8 sessions of 1 to 9,001 keys, 8 heads, D = 128, us: both 40, one of them
// 19 (24-25 where the other's codes are read too); chosen at run time, by branches among the loads, 45 and 22.
template <typename T, int D, bool K, bool V>
__global__ __launch_bounds__(kRowThreads)
void kv4_read_kernel(Kv4Rows rows, Kv4Pool pool, int Hkv, int nunits, T* __restrict__ k_out, int64_t k_stride,
                     T* __restrict__ v_out, int64_t v_stride) {
  constexpr int TPR = D / 8, kKeys = kWave / TPR;
  constexpr int kRounds = kTile / kKeys;
  constexpr int kWords = kTile * D / 8;
  __shared__ __align__(16) uint32_t image[kRowThreads / kWave][2 * kWords];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x * (kRowThreads / kWave) + wave;
  if (unit >= nunits) return;
  const Tile t = tile_of(rows, pool, Hkv, unit);
  const int lane = threadIdx.x & 63, col = lane % TPR * 8;
  uint32_t* const k_image = image[wave];
  uint32_t* const v_image = k_image + kWords;
  const uint8_t* const k_in = pool.k + t.block * (32 * D) + t.key0 * (D / 2);
  const uint8_t* const v_in = pool.v + t.block * (32 * D) + t.key0 * 8;
  const uint8_t* const k_scale = pool.k_scale + t.block * (2 * D) + t.key0 / kTile;
  const uint16_t* const v_scale = pool.v_scale + t.block * kKeyBlock4 + t.key0;
  [[maybe_unused]] float ks[kRounds], vs[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int key = i * kKeys + lane / TPR;
    if constexpr (K) ks[i] = __uint_as_float((uint32_t)k_scale[(col / kGroup4 * 16 + key) * 4] << 23);
    if constexpr (V) vs[i] = bf16_to_f32(v_scale[key]);
  }
  if constexpr (K) {
    if (D == 128)
      reinterpret_cast<u32x4*>(k_image)[lane] = reinterpret_cast<const u32x4*>(k_in)[lane];
    else
      reinterpret_cast<u32x2*>(k_image)[lane] = reinterpret_cast<const u32x2*>(k_in)[lane];
  }
  if (V && lane < D / 2)
    reinterpret_cast<u32x4*>(v_image)[lane] = *reinterpret_cast<const u32x4*>(v_in + lane / 8 * 512 + lane % 8 * 16);
  lds_wait();
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int key = i * kKeys + lane / TPR;
    const bool mine = key >= t.from && key < t.to;
    const int64_t row = t.row0 + key;
    if (i * kKeys >= t.to || (i + 1) * kKeys <= t.from) continue;
    float x[8];
    if constexpr (K) {
      decode8(k_image[k_dword<D>(key, col)], ks[i], x);
      if (mine) store_row8(k_out + row * k_stride + t.head * D + col, x);
    }
    if constexpr (V) {
      decode8(v_image[v_dword(key, col)], 1.f, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= vs[i];
      if (mine) store_row8(v_out + row * v_stride + t.head * D + col, x);
    }
  }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Rows& r, const Kv4Pool& pool, int Hkv, int D, bool f32, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t stream) {
  const int nunits = r.prefix[r.nreq] * Hkv;
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
  const int nunits = r.prefix[r.nreq] * Hkv;
  const dim3 grid((nunits + kRowThreads / kWave - 1) / (kRowThreads / kWave)), block(kRowThreads);
#define SDV_READ_OF(T, DIM, K, V)                                                                                \
  hipLaunchKernelGGL((kv4_read_kernel<T, DIM, K, V>), grid, block, 0, stream, r, pool, Hkv, nunits,              \
                     static_cast<T*>(k_out), k_stride, static_cast<T*>(v_out), v_stride)
#define SDV_READ(T, DIM)                  \
  if (k_out != nullptr && v_out != nullptr) { \
    SDV_READ_OF(T, DIM, true, true);      \
  } else if (k_out != nullptr) {          \
    SDV_READ_OF(T, DIM, true, false);     \
  } else {                                \
    SDV_READ_OF(T, DIM, false, true);     \
  }
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
#undef SDV_READ_OF
  return hipGetLastError();
}

}  // namespace sdv
