// Appending key and value rows to a paged 8-bit cache (gfx950).
//
// One workgroup per (64-key block that a request's new rows touch, KV head, K
// or V): the block's scale needs the largest magnitude of all its new rows, and
// a block is the unit that is rewritten when its scale grows.  Scales are
// powers of two: an e4m3 code keeps its three fraction bits under any of them,
// so a finer scale would buy no precision, and a block whose scale grows is
// rewritten exactly (values that leave the normal range apart).
//
// A thread holds four consecutive keys by eight columns, read once with 16-byte
// loads (the 16 threads of a quad of keys read whole rows).  Codes go to an
// LDS image of the block in its layout and from there to the pool 16 bytes at
// a time; blocks that also hold earlier or later bytes merge them there.  Bound
// by memory: bf16 rows read 2 bytes and write 1 per element.
#include "fp8.h"

namespace sdv {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kLowestExp = 27;  // byte of the smallest scale, 2^-100

// Smallest e with most <= 448 * 2^e as a scale byte, at least 2^-100 (most
// finite, >= 0).  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(float most) {
  const uint32_t b = __float_as_uint(most);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(e, kLowestExp);
}

__device__ __forceinline__ float pow2_f32(int e) {  // 2^e, -126 <= e <= 127
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

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

// Codes of a dword rewritten for a scale 1 / f times theirs.
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return encode4(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// Bytes 0 .. n - 1 of a dword, n clamped to 0 .. 4.
__device__ __forceinline__ uint32_t first_bytes(int n) {
  return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

template <typename T, int D>
__global__ __launch_bounds__(kAppendThreads)
void kv8_append_kernel(Kv8Append a, Kv8Pool pool, int Hkv, const T* __restrict__ k_new, int64_t k_stride,
                       const T* __restrict__ v_new, int64_t v_stride) {
  constexpr int TPR = D / 8;                       // threads per row
  constexpr int kQuads = kAppendThreads / TPR;     // quads of keys in flight at once
  constexpr int kRounds = 16 / kQuads < 1 ? 1 : 16 / kQuads;
  constexpr int kPieces = D * kKeyBlock / 16;      // 16-byte pieces of a block
  __shared__ __align__(16) uint32_t image[D * kKeyBlock / 4];
  __shared__ float wave_most[kAppendThreads / kWave];

  const int c = blockIdx.x, head = blockIdx.y, t = threadIdx.x;
  const bool is_v = blockIdx.z != 0;
  int lo = 0, hi = a.nreq - 1;  // the largest request with blk_prefix <= c
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.blk_prefix[mid] <= c) lo = mid; else hi = mid - 1;
  }
  const int end = a.kv_len[lo], begin = end - a.new_len[lo];
  const int blk = begin / kKeyBlock + (c - a.blk_prefix[lo]);
  const int key0 = blk * kKeyBlock;
  const int per_page_shift = pool.page_shift - 6;
  int page = pool.table[(int64_t)a.req[lo] * pool.max_pages + (blk >> per_page_shift)];
  page = min(max(page, 0), pool.num_pages - 1);
  const int64_t at = ((((int64_t)page * Hkv + head) << per_page_shift)) + (blk & ((1 << per_page_shift) - 1));
  uint8_t* scale = (is_v ? pool.v_scale : pool.k_scale) + at;
  u32x4* block = reinterpret_cast<u32x4*>((is_v ? pool.v : pool.k) + at * (D * kKeyBlock));

  const bool has_old = begin > key0;                       // earlier keys stay in this block
  const bool whole = !has_old && end >= key0 + kKeyBlock;  // every byte is new
  const int was = has_old ? *scale : 0;
  u32x4 there[kPieces / kAppendThreads];  // what a partly written block holds, read with the rows
  if (!whole) {
#pragma unroll
    for (int i = 0; i < kPieces / kAppendThreads; ++i) there[i] = block[t + i * kAppendThreads];
  }

  const T* src = is_v ? v_new : k_new;
  const int64_t stride = is_v ? v_stride : k_stride;
  const int col = (t % TPR) * 8;
  float x[kRounds][4][8];
  float most = 0.f;
#pragma unroll
  for (int n = 0; n < kRounds; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int key = key0 + 4 * (t / TPR + n * kQuads) + r;
      const bool is_new = t / TPR + n * kQuads < 16 && key >= begin && key < end;
      if (is_new) {
        load_row8(src + (a.new_off[lo] + (key - begin)) * stride + head * D + col, x[n][r]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[n][r][e] = 0.f;
      }
    }
#pragma unroll
  for (int n = 0; n < kRounds; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = fabsf(x[n][r][e]);
        most = m < INFINITY ? fmaxf(most, m) : most;  // infinities and NaN do not set the scale
      }
  most = wave_max(most);
  if ((t & 63) == 0) wave_most[t >> 6] = most;
  __syncthreads();
  most = fmaxf(fmaxf(wave_most[0], wave_most[1]), fmaxf(wave_most[2], wave_most[3]));
  const int now = max(scale_byte(most), was);
  const float mul = pow2_f32(127 - now);

#pragma unroll
  for (int n = 0; n < kRounds; ++n) {
    const int quad = t / TPR + n * kQuads;
    if (quad < 16) {
      const int kt = quad >> 2, kg = quad & 3;
      if (is_v) {
        // [D/16][4 g][16 d][4 t][4 r]: the four keys of a quad are one dword.
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = col + e;
          image[((d / 16 * 4 + kg) * 16 + d % 16) * 4 + kt] =
              encode4(x[n][0][e] * mul, x[n][1][e] * mul, x[n][2][e] * mul, x[n][3][e] * mul);
        }
      } else {
        // [D/64][4 t][4 g][16 r][16 b]
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int p = (((col / 64 * 4 + kt) * 4 + col % 64 / 16) * 16 + kg * 4 + r) * 4 + col % 16 / 4;
          *reinterpret_cast<u32x2*>(image + p) =
              u32x2{encode4(x[n][r][0] * mul, x[n][r][1] * mul, x[n][r][2] * mul, x[n][r][3] * mul),
                    encode4(x[n][r][4] * mul, x[n][r][5] * mul, x[n][r][6] * mul, x[n][r][7] * mul)};
        }
      }
    }
  }
  __syncthreads();
  const bool grew = has_old && now > was;
  const float shrink = pow2_f32(max(was - now, -126));
#pragma unroll
  for (int i = 0; i < kPieces / kAppendThreads; ++i) {
    const int p = t + i * kAppendThreads;
    u32x4 r = reinterpret_cast<const u32x4*>(image)[p];
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // Keys of dword j: one key's four columns of K, four keys of V.
        const int key = is_v ? key0 + 16 * j + 4 * (p / 16 % 4) : key0 + 16 * (p / 64 % 4) + p % 16;
        const uint32_t before = is_v ? first_bytes(begin - key) : begin > key ? 0xffffffffu : 0u;
        const uint32_t upto = is_v ? first_bytes(end - key) : end > key ? 0xffffffffu : 0u;
        const uint32_t old = grew ? rescale4(there[i][j], shrink) : there[i][j];
        r[j] = (old & before) | (r[j] & upto & ~before) | (there[i][j] & ~upto);
      }
    }
    block[p] = r;
  }
  if (t == 0) *scale = (uint8_t)now;
}

}  // namespace

hipError_t launch_kv8_append(const Kv8Append& a, const Kv8Pool& pool, int Hkv, int D, bool f32, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t stream) {
  const dim3 grid(a.blk_prefix[a.nreq], Hkv, 2);
#define SDV_APPEND(T, DIM)                                                                                       \
  hipLaunchKernelGGL((kv8_append_kernel<T, DIM>), grid, dim3(kAppendThreads), 0, stream, a, pool, Hkv,            \
                     static_cast<const T*>(k_new), k_stride, static_cast<const T*>(v_new), v_stride)
  if (f32 && D == 128) SDV_APPEND(float, 128);
  else if (f32) SDV_APPEND(float, 64);
  else if (D == 128) SDV_APPEND(uint16_t, 128);
  else SDV_APPEND(uint16_t, 64);
#undef SDV_APPEND
  return hipGetLastError();
}

}  // namespace sdv
