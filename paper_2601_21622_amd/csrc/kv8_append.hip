// Appending key and value rows to a paged 8-bit cache (gfx950).
//
// The unit of work is a (64-key block that a request's new rows touch, KV head, K or
// V): the block's scale needs the largest magnitude of all its new rows, and a block
// is what is rewritten when its scale grows.  Scales are powers of two: an e4m3 code
// keeps its three fraction bits under any of them, so a finer scale would buy no
// precision, and a block whose scale grows is rewritten exactly (values that leave the
// normal range apart).
//
// A thread holds four consecutive keys by eight columns, read once with 16-byte loads
// (the threads of a quad of keys read whole rows).
//  * Prompts: a workgroup takes a unit.  Codes go to an LDS image of the block in its
//    layout and from there to the pool 16 bytes at a time, only the pieces that hold
//    new keys (or, where the scale grew, earlier ones); pieces of V that hold others
//    too are read with the rows and merged.  Bound by memory, 2 bytes read and 1
//    written per bf16 element: 8 prompts of 1 to 6,001 rows and 8 heads take 34 us,
//    4.3 TB/s, a large copy's rate being 4.8.
//  * Steps of a few keys: a wave takes a unit, so that all units of a large batch are
//    resident at once, and stores its codes straight away.  Bound by the latency of
//    table, rows and store, one behind the other, and by the sectors that V's layout
//    spreads a few keys over (5 keys touch 4 KB of a block's 8): 10 us for 64 requests of 5
//    keys and 32 heads, which read 28 MB and write 23 where rows and codes are 8.
#include "fp8.h"

namespace sdv {

namespace {

constexpr int kAppendThreads = 256;
// New keys per request up to which a wave takes a unit: at head dimension 128 its
// 16 threads per row hold four quads of keys.  64 requests of 5 keys and 32 heads:
// 21.5 us with a workgroup per unit, 10.0 with a wave.
constexpr int kFewKeys = 13;
constexpr int kLowestExp = 27;  // byte of the smallest scale, 2^-100

// Smallest e with most <= 448 * 2^e as a scale byte, at least 2^-100 (most
// finite, >= 0).  448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_byte(float most) {
  const uint32_t b = __float_as_uint(most);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(e, kLowestExp);
}

__device__ __forceinline__ float pow2_f32(int e) {  // 2^e, -127 <= e <= 127
  return __uint_as_float(e > -127 ? (uint32_t)(e + 127) << 23 : 0x400000u);
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

// One (block, head, K or V) that takes new keys.
struct Unit {
  u32x4* block;
  uint8_t* scale;
  int b0, e0;    // keys b0 .. e0 - 1 of the block are new
  int64_t row0;  // row of the new tensors for key 0 of the block
  int head;
  bool is_v;
};

template <int D>
__device__ __forceinline__ Unit unit_of(const Kv8Append& a, const Kv8Pool& pool, int Hkv, int unit, int lane) {
  Unit u;
  u.is_v = (unit & 1) != 0;
  u.head = (unit >> 1) % Hkv;
  const int c = (unit >> 1) / Hkv;
  // The largest request with blk_prefix <= c: one load, a request per lane.
  const int prefix = lane < a.nreq ? a.blk_prefix[lane] : INT32_MAX;
  const int lo = __popcll(__ballot(prefix <= c)) - 1;
  const int end = a.kv_len[lo], begin = end - a.new_len[lo];
  const int blk = begin / kKeyBlock + (c - __builtin_amdgcn_readlane(prefix, lo));
  const int key0 = blk * kKeyBlock;
  const int per_page_shift = pool.page_shift - 6;
  int page = pool.table[(int64_t)a.req[lo] * pool.max_pages + (blk >> per_page_shift)];
  page = min(max(page, 0), pool.num_pages - 1);
  const int64_t at = ((((int64_t)page * Hkv + u.head) << per_page_shift)) + (blk & ((1 << per_page_shift) - 1));
  u.scale = (u.is_v ? pool.v_scale : pool.k_scale) + at;
  u.block = reinterpret_cast<u32x4*>((u.is_v ? pool.v : pool.k) + at * (D * kKeyBlock));
  u.b0 = max(begin - key0, 0);
  u.e0 = min(end - key0, kKeyBlock);
  u.row0 = a.new_off[lo] + (key0 - begin);
  return u;
}

// Rows 4 quad .. + 3 of the block, 8 columns from col; zeros where no key is new (a
// new row is read in its place, so that the four loads are on their way together).
// Returns the largest finite magnitude.
template <typename T>
__device__ __forceinline__ float load_quad(const Unit& u, const T* src, int64_t stride, int quad, int col,
                                           float (&x)[4][8]) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    load_row8(src + (u.row0 + min(max(4 * quad + r, u.b0), u.e0 - 1)) * stride + col, x[r]);
  float most = 0.f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const bool is_new = 4 * quad + r >= u.b0 && 4 * quad + r < u.e0;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[r][e] = is_new ? x[r][e] : 0.f;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = fabsf(x[r][e]);
      most = m < INFINITY ? fmaxf(most, m) : most;  // infinities and NaN do not set the scale
    }
  return most;
}

// Index of the dword that holds columns col .. + 3 of a key in a block of K, and of
// the one that holds keys 4 quad .. + 3 of column d in a block of V.
__device__ __forceinline__ int k_dword(int key, int col) {
  // [D/64][4 t][4 g][16 r][16 b]
  return (((col / 64 * 4 + key / 16) * 4 + col % 64 / 16) * 16 + key % 16) * 4 + col % 16 / 4;
}
__device__ __forceinline__ int v_dword(int quad, int d) {
  // [D/16][4 g][16 d][4 t][4 r]
  return ((d / 16 * 4 + quad % 4) * 16 + d % 16) * 4 + quad / 4;
}

__device__ __forceinline__ u32x2 encode8(const float (&x)[8], float mul) {
  return u32x2{encode4(x[0] * mul, x[1] * mul, x[2] * mul, x[3] * mul),
               encode4(x[4] * mul, x[5] * mul, x[6] * mul, x[7] * mul)};
}

// A wave per unit, for at most kFewKeys new keys of a request: the quads that they
// lie in are one round of loads, and each thread stores its own codes where they
// belong.  Nothing of the block is read but the dwords of V that hold other keys too,
// unless the scale grows.
template <typename T, int D>
__global__ __launch_bounds__(kAppendThreads)
void kv8_append_few_kernel(Kv8Append a, Kv8Pool pool, int Hkv, int nunits, const T* __restrict__ k_new,
                           int64_t k_stride, const T* __restrict__ v_new, int64_t v_stride) {
  constexpr int TPR = D / 8;  // threads per row
  static_assert(kWave / TPR * 4 >= kFewKeys + 3, "one round of loads");
  constexpr int kPieces = D * kKeyBlock / 16;  // 16-byte pieces of a block
  const int unit = blockIdx.x * (kAppendThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= nunits) return;
  const int lane = threadIdx.x & 63;
  const Unit u = unit_of<D>(a, pool, Hkv, unit, lane);
  const int col = lane % TPR * 8, quad = u.b0 / 4 + lane / TPR;
  const bool mine = 4 * quad < u.e0;
  const int was = u.b0 > 0 ? *u.scale : 0;
  uint32_t* const words = reinterpret_cast<uint32_t*>(u.block);
  // Bytes of the quad's dwords of V that are new, and earlier keys.
  const uint32_t old_bytes = first_bytes(u.b0 - 4 * quad);
  const uint32_t new_bytes = first_bytes(u.e0 - 4 * quad) & ~old_bytes;
  uint32_t there[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    there[e] = u.is_v && mine && new_bytes != 0xffffffffu ? words[v_dword(quad, col + e)] : 0u;
  float x[4][8];
  const float most = wave_max(
      load_quad(u, (u.is_v ? v_new : k_new) + u.head * D, u.is_v ? v_stride : k_stride, quad, col, x));
  const int now = max(scale_byte(most), was);
  const float mul = pow2_f32(127 - now);
  const bool grew = u.b0 > 0 && now > was;
  const float shrink = pow2_f32(max(was - now, -126));
  if (mine) {
    if (u.is_v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t codes = encode4(x[0][e] * mul, x[1][e] * mul, x[2][e] * mul, x[3][e] * mul);
        const uint32_t old = grew ? rescale4(there[e], shrink) : there[e];
        words[v_dword(quad, col + e)] =
            (codes & new_bytes) | (old & old_bytes) | (there[e] & ~(new_bytes | old_bytes));
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * quad + r >= u.b0 && 4 * quad + r < u.e0)
          *reinterpret_cast<u32x2*>(words + k_dword(4 * quad + r, col)) = encode8(x[r], mul);
    }
  }
  // The other earlier keys, each dword by one thread: those of V below the first quad.
  if (grew) {
    for (int p = lane; p < kPieces; p += kWave) {
      const u32x4 old = u.block[p];
      if (!u.is_v) {
        if (p / 64 % 4 * 16 + p % 16 < u.b0)
          u.block[p] = u32x4{rescale4(old[0], shrink), rescale4(old[1], shrink), rescale4(old[2], shrink),
                             rescale4(old[3], shrink)};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * j + p / 16 % 4 < u.b0 / 4) words[4 * p + j] = rescale4(old[j], shrink);
      }
    }
  }
  if (lane == 0) *u.scale = (uint8_t)now;
}

// A workgroup per unit: the new codes are laid out in LDS and the touched pieces of
// the block written whole.
template <typename T, int D>
__global__ __launch_bounds__(kAppendThreads)
void kv8_append_kernel(Kv8Append a, Kv8Pool pool, int Hkv, const T* __restrict__ k_new, int64_t k_stride,
                       const T* __restrict__ v_new, int64_t v_stride) {
  constexpr int TPR = D / 8;  // threads per row
  constexpr int kQuads = kAppendThreads / TPR;
  static_assert(kQuads * 4 >= kKeyBlock, "one round of loads");
  constexpr int kPieces = D * kKeyBlock / 16;  // 16-byte pieces of a block
  constexpr int kMine = kPieces / kAppendThreads;
  __shared__ __align__(16) uint32_t image[D * kKeyBlock / 4];
  __shared__ float wave_most[kAppendThreads / kWave];

  const int t = threadIdx.x, lane = t & 63;
  const Unit u = unit_of<D>(a, pool, Hkv, blockIdx.x, lane);
  const int b0 = u.b0, e0 = u.e0;
  const bool is_v = u.is_v;
  u32x4* const block = u.block;

  // Keys of the block that are new, and earlier ones that stay in it.
  const uint64_t old_keys = b0 > 0 ? ~0ull >> (64 - b0) : 0ull;
  const uint64_t new_keys = (~0ull >> (64 - e0)) & ~old_keys;
  const int was = b0 > 0 ? *u.scale : 0;
  // A piece of 16 bytes holds one key's columns of K, a column of 16 keys of V.
  // Those of V that hold other keys beside new ones are read with the rows.
  auto keys_of = [&](int p) {
    return is_v ? 0x000f000f000f000full << (4 * (p / 16 % 4)) : 1ull << (16 * (p / 64 % 4) + p % 16);
  };
  u32x4 there[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int p = t + i * kAppendThreads;
    const uint64_t keys = keys_of(p);
    there[i] = u32x4{0u, 0u, 0u, 0u};
    if ((keys & new_keys) != 0 && (keys & ~new_keys) != 0) there[i] = block[p];
  }

  const int col = t % TPR * 8, quad = t / TPR;  // keys 4 quad .. + 3 of the block
  float x[4][8];
  float most = wave_max(load_quad(u, (is_v ? v_new : k_new) + u.head * D, is_v ? v_stride : k_stride, quad, col, x));
  if (lane == 0) wave_most[t >> 6] = most;
  __syncthreads();
  most = fmaxf(fmaxf(wave_most[0], wave_most[1]), fmaxf(wave_most[2], wave_most[3]));
  const int now = max(scale_byte(most), was);
  const float mul = pow2_f32(127 - now);

  if (quad < kKeyBlock / 4) {
    if (is_v) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        image[v_dword(quad, col + e)] = encode4(x[0][e] * mul, x[1][e] * mul, x[2][e] * mul, x[3][e] * mul);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<u32x2*>(image + k_dword(4 * quad + r, col)) = encode8(x[r], mul);
    }
  }
  __syncthreads();
  // A grown scale rewrites the earlier keys too.
  const bool grew = b0 > 0 && now > was;
  const float shrink = pow2_f32(max(was - now, -126));
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int p = t + i * kAppendThreads;
    const uint64_t keys = keys_of(p);
    u32x4 r = reinterpret_cast<const u32x4*>(image)[p];
    if (grew && (keys & old_keys) != 0) {
      there[i] = block[p];
    } else if ((keys & new_keys) == 0) {
      continue;
    }
    if ((keys & ~new_keys) != 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = is_v ? 16 * j + 4 * (p / 16 % 4) : 16 * (p / 64 % 4) + p % 16;
        const uint32_t before = is_v ? first_bytes(b0 - key) : b0 > key ? 0xffffffffu : 0u;
        const uint32_t upto = is_v ? first_bytes(e0 - key) : e0 > key ? 0xffffffffu : 0u;
        const uint32_t old = grew ? rescale4(there[i][j], shrink) : there[i][j];
        r[j] = (old & before) | (r[j] & upto & ~before) | (there[i][j] & ~upto);
      }
    }
    block[p] = r;
  }
  if (t == 0) *u.scale = (uint8_t)now;
}

}  // namespace

hipError_t launch_kv8_append(const Kv8Append& a, const Kv8Pool& pool, int Hkv, int D, bool f32, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t stream) {
  const int nunits = a.blk_prefix[a.nreq] * Hkv * 2;
  int most = 0;
  for (int i = 0; i < a.nreq; ++i) most = most > a.new_len[i] ? most : a.new_len[i];
  const bool few = most <= kFewKeys;
  const int per = few ? kAppendThreads / kWave : 1;
  const dim3 grid((nunits + per - 1) / per), block(kAppendThreads);
#define SDV_APPEND(T, DIM)                                                                                       \
  if (few)                                                                                                       \
    hipLaunchKernelGGL((kv8_append_few_kernel<T, DIM>), grid, block, 0, stream, a, pool, Hkv, nunits,             \
                       static_cast<const T*>(k_new), k_stride, static_cast<const T*>(v_new), v_stride);          \
  else                                                                                                           \
    hipLaunchKernelGGL((kv8_append_kernel<T, DIM>), grid, block, 0, stream, a, pool, Hkv,                         \
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

}  // namespace sdv
