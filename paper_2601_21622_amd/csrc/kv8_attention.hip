// Verification attention over a paged 8-bit cache (split-KV) for gfx950.
//
//   O = softmax(scale * Q K^T + mask) V,  K = code * 2^e of its 64-key block and head, V likewise.
//
// The G * group queries that share a KV head are the rows of one KV head.  One
// wave, a workgroup of its own, per work item (chunk of whole 64-key blocks of one
// request, KV head, group of rows); each item writes a partial (maximum, sum, O)
// and the merge joins them in chunk order.
//
// Bound by the cache's stream up to two 16-row blocks: 16 requests of 24,576 keys, 8 KV
// heads, D = 128 (805 MB) take 128-133 us with one block, 6.1-6.3 TB/s, and 145 with
// two.  Each block more adds about 20 us (152 with three, 178 with four, 200 with five), of
// which the vector instructions of its 64 x 16 scores are the larger part and its matrix
// products 12: LDS and registers allow one wave per SIMD there, and its phases follow one
// another.
// Scores are kept in vector registers by the build's choice of instruction form: in
// accumulation registers every score is moved once more (four blocks 194 us, five 214).
//
// The cache is laid out in the order in which the matrix instructions take
// their operands (sdverify_fp8.h): a lane's 16 bytes of K are two 32-wide steps
// of one key, its 16 bytes of V four keys in each of the block's four 16-key
// score tiles.  So a fragment is 1 KB in a row everywhere, and nothing is
// transposed: the probabilities that a lane holds after S^T = K Q^T (tile t:
// keys 16 t + 4 g + r of group g = lane / 16) are the keys that its V bytes hold,
// which is all that O^T += V^T P^T needs.  Codes widen to bfloat16 with the
// block's scale in the same instruction, exactly.  (The 8-bit matrix instructions
// would skip that, but they keep too few bits: sums of 128 products come out
// 1.4e-5 off, and P would have to be 8 bits.)
//
// K and V come by LDS DMA into a ring of half blocks (one block's K, or its V) of
// the wave's own, as many halves ahead as the CU's LDS holds; a half's place is
// filled again, DMA by DMA, under the products after it is free.  In registers the
// 128 of a block and its successor would push O out to scratch.
//
// Softmax in the log2 domain.  O is never rescaled (a branch that does so made
// the compiler spill up to 535 registers): a row's first scores in the chunk set
// its reference maximum, and later ones may exceed it by 2^64, less where V is so
// large that the sum of so many weights times values could leave float32
// (grow_limit).  A row that outgrows that makes the wave take the maxima
// of all its blocks and start its item again, once: this time scores are summed
// from zero, as they were for the maxima, and the reference is subtracted from the
// sum.  That gives the same bits, so that no difference is above zero and the largest
// is zero.  (Sums that start at the reference round differently: by more than 2^64
// in the exponential where scores are past 2^28, in either direction.)
// Where every item is taken up again, 16 requests of 24,570 keys and 72 rows, D = 128,
// take 460 us instead of 195.
#include <algorithm>
#include <atomic>

#include "fp8.h"

namespace sdv {

namespace {

constexpr int kMaxBlocks = 5;   // 16-row blocks of a wave
constexpr int kMaxTiles = 64;   // blocks per chunk: one lane holds one block's page
constexpr float kNoKey = -3.402823466e38f;  // reference maximum of a row that has seen no key: no score lies below it
constexpr int kGrowLog2 = 64;   // growth of a row's maximum, log2, that takes the item up anew

// The growth that weights of a block may have whose V scale byte is this: 2^30 keys
// (the longest cache) of weight 2^limit and value 448 * 2^(byte - 127) sum to less than
// 2^128.  None from byte 216 on, where the values alone have to sum to less.
__device__ __forceinline__ float grow_limit(int v_byte) { return (float)min(max(216 - v_byte, 0), kGrowLog2); }

// A wave's ring: halves of 64 D bytes, D / 16 DMAs of 1 KB each.  Four (D = 128) or
// eight fill a CU's 160 KB.
template <int D>
struct Ring {
  static constexpr int kHalf = D * kKeyBlock;
  static constexpr int kOps = D / 16;
  static constexpr int kSlots = 5;
};

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

template <bool X>
struct Kind {
  static constexpr bool value = X;
};
template <int X>
struct Int {
  static constexpr int value = X;
};

// LDS DMA of 1 KB: lane l copies 16 bytes from base + off into LDS bytes lds +
// 16 l (lds wave-uniform).  From inline assembly, so that the compiler adds no
// waits of its own.  The base is copied by a scalar instruction first: that is the
// wait state between the write of M0 and the load, and the load's base is never a
// register that a vector instruction (a lane's read, a spill's) wrote just before,
// which would take five.
__device__ __forceinline__ void ring_dma(const void* base, uint32_t off, uint32_t lds) {
  uint64_t from;
  asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0 nt"
               : "=&s"(from)
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base)
               : "m0", "memory");
}

__device__ __forceinline__ float max_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Positions that position `lane` (< G) sees of the step's own (bit a: position
// a): in a chain itself and those before it, in a tree itself and its
// ancestors, by pointer jumping over the parents.
__device__ __forceinline__ uint64_t position_mask(const int32_t* __restrict__ parent, int G) {
  const int lane = threadIdx.x & 63;
  if (parent == nullptr) return lane >= 63 ? ~0ull : (2ull << lane) - 1ull;
  int p = 0;
  if (lane > 0 && lane < G) {
    const int pp = parent[lane - 1];
    p = (pp >= -1 && pp < lane - 1) ? pp + 1 : 0;
  }
  uint64_t m = 1ull | (1ull << lane);
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const uint32_t lo = __shfl((uint32_t)m, p), hi = __shfl((uint32_t)(m >> 32), p);
    m |= ((uint64_t)hi << 32) | lo;
    p = __shfl(p, p);
  }
  return m;
}

// Bytes of a dword of four keys, the first of them `key`, that lie before `end`.
__device__ __forceinline__ uint32_t bytes_before(int key, int end) {
  const int n = end - key;
  return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

// 1 in each byte of a dword that is a NaN code.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t codes) {
  return (((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
}

// Bit i: whether key `off` + i (counted from the first of the step's positions)
// is seen: all keys before them, then the positions of `sees`, none after.
__device__ __forceinline__ uint64_t keys_seen(uint64_t sees, int off) {
  const uint64_t up = off < 64 ? sees >> (off & 63) : 0ull;
  const int n = -off;
  const uint64_t down = n < 64 ? (sees << (n & 63)) | ((1ull << (n & 63)) - 1ull) : ~0ull;
  return off >= 0 ? up : down;
}

template <int RB, int D>
struct Wave8 {
  bf16x8 q[RB][D / 32];
  f32x4 o[RB][D / 16];
  float m[RB], l[RB];  // reference maximum of the unscaled scores (kNoKey: no key seen yet), sum
  uint64_t sees[RB];   // of the step's own positions
  uint32_t nan;        // a NaN code was left out of O
};

// The instructions since the last call as M products with at most V vector
// instructions among them, one product first, so that the vector ones issue
// while the matrix core works.
template <int M, int V>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < M; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, (V + M - 1) / M, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Scores of half `hf` of a 64-key block (its score tiles 2 hf and 2 hf + 1) less
// `base`: the accumulators start there, so that the difference that the
// exponential takes costs no instruction and keeps its bits however large the
// scores are.  MASKED: some key lies past `first`, the first of the step's
// positions; what a row does not see is -inf.
template <int RB, int D, bool MASKED, typename Refill>
__device__ __forceinline__ void half_scores(const Wave8<RB, D>& w, const u32x4 (&k)[2][D / 64], int hf, float ks,
                                            int off, const float (&base)[RB], f32x4 (&sc)[RB][2], Refill refill) {
  constexpr int kSteps = D / 32;  // 32-wide steps of a score tile
  auto widen_k = [&](int n) {
    const u32x4 x = k[n / kSteps][n % kSteps / 2];
    return widen8(x[2 * (n & 1)], x[2 * (n & 1) + 1], ks);
  };
  bf16x8 kf = widen_k(0);
#pragma unroll
  for (int n = 0; n < 2 * kSteps; ++n) {
    const int t = n / kSteps;
    const bf16x8 now = kf;
    if (n + 1 < 2 * kSteps) kf = widen_k(n + 1);  // under this step's products
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      sc[rb][t] = mfma16x16x32(now, w.q[rb][n % kSteps],
                               n % kSteps == 0 ? f32x4{base[rb], base[rb], base[rb], base[rb]} : sc[rb][t]);
    if (n % kSteps == kSteps - 1) refill(2 * hf + t);
    interleave<RB, 4>();
  }
  if (MASKED) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const uint64_t win = keys_seen(w.sees[rb], off) >> (32 * hf);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t see = (uint32_t)(win >> (16 * t + r)) & 1u;
          const uint32_t x = __float_as_uint(sc[rb][t][r]);
          sc[rb][t][r] = __uint_as_float(see ? x : 0xff800000u);
        }
    }
  }
}

// K fragments of half `hf` of the block at kp.
template <int D>
__device__ __forceinline__ void read_k(const unsigned char* kp, int hf, u32x4 (&k)[2][D / 64]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < D / 64; ++i) k[t][i] = *reinterpret_cast<const u32x4*>(kp + (i * 4 + 2 * hf + t) * 1024);
}

// Each row's largest score of the half.
template <int RB>
__device__ __forceinline__ void half_max(const f32x4 (&sc)[RB][2], float (&mx)[RB]) {
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float x = fmaxf(fmaxf(sc[rb][0][0], sc[rb][0][1]), fmaxf(sc[rb][0][2], sc[rb][0][3]));
    x = fmaxf(fmaxf(fmaxf(x, sc[rb][1][0]), sc[rb][1][1]), fmaxf(sc[rb][1][2], sc[rb][1][3]));
    mx[rb] = max_over_groups(x);
  }
}

// Folds one block, half after half, into O and the sums; false when some row's
// maximum has outgrown its reference by `limit` (O is then not whole).  `again` (MASKED only):
// references are the maxima of all blocks, scores are summed from zero, and the
// result is true.  refill_v and
// refill_k take quarter `n` of the DMAs into the places of the last block's V and
// of this one's K; wait_v waits for this block's V.
template <int RB, int D, bool MASKED, typename WaitV, typename RefillV, typename RefillK>
__device__ __forceinline__ bool fold_block(Wave8<RB, D>& w, const unsigned char* kp, const unsigned char* vp, float ks,
                                           float vs, float limit, float scale_log2, int key0, int first, int end, bool again,
                                           WaitV wait_v, RefillV refill_v, RefillK refill_k) {
  const int lg = (threadIdx.x & 63) >> 4;
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  // V fragments in flight from LDS: a fragment's RB products cover its successors' latency.
  constexpr int kAhead = RB == 1 ? 8 : RB == 2 ? 4 : 2;
  const bool known = MASKED && again;
  u32x4 k[2][D / 64];
  read_k<D>(kp, 0, k);
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    f32x4 sc[RB][2];
    float base[RB], mx[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) base[rb] = w.m[rb] > kNoKey && !known ? -w.m[rb] : 0.f;
    half_scores<RB, D, MASKED>(w, k, hf, ks, key0 + 4 * lg - first, base, sc, refill_v);
    if (hf == 0) {
      read_k<D>(kp, 1, k);
      wait_v();
    }
    u32x2 v_in[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead && i < D / 16; ++i) v_in[i] = *reinterpret_cast<const u32x2*>(vp + i * 1024 + 8 * hf);
    half_max<RB>(sc, mx);
    bool grow = false, fresh = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      grow |= w.m[rb] > kNoKey && mx[rb] * scale_log2 > limit;
      fresh |= !(w.m[rb] > kNoKey) && mx[rb] > kNoKey;
    }
    if (__builtin_expect(__ballot(grow) != 0, 0) && !known) return false;
    if (__builtin_expect(__ballot(fresh) != 0 || known, 0)) {  // rows' first keys: their maximum is the reference
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const bool set = !known && !(w.m[rb] > kNoKey) && mx[rb] > kNoKey;
        w.m[rb] = set ? mx[rb] : w.m[rb];
        const float less = set || (known && w.m[rb] > kNoKey) ? w.m[rb] : 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[rb][t][r] -= less;
      }
    }
    // P in bfloat16, as the products take it; the sum adds the rounded values,
    // so that the weights that O accumulates sum to one.
    bf16x8 pf[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float acc = w.l[rb];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const f32x2 x = {__builtin_amdgcn_exp2f(sc[rb][t][r] * scale_log2),
                           __builtin_amdgcn_exp2f(sc[rb][t][r + 1] * scale_log2)};
          const bf16x2 pb = __builtin_convertvector(x, bf16x2);
          pf[rb][t * 4 + r] = pb[0];
          pf[rb][t * 4 + r + 1] = pb[1];
          acc = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, acc, false);
        }
      w.l[rb] = acc;
    }
    // Fragment db of V, cleared where it must not be read as numbers.
    auto widen_v = [&](int db) {
      u32x2 v = v_in[db % kAhead];
      if (db + kAhead < D / 16) v_in[db % kAhead] = *reinterpret_cast<const u32x2*>(vp + (db + kAhead) * 1024 + 8 * hf);
      if (MASKED) {
        // What lies past the last key is no number, and NaN codes are left to
        // spread_nan: 0 * NaN would reach the rows that do not see them.
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          v[t] &= bytes_before(key0 + 32 * hf + 16 * t + 4 * lg, end);
          const uint32_t hit = nan_bytes(v[t]);
          w.nan |= hit;
          v[t] &= ~(hit * 0xffu);
        }
      }
      return widen8(v[0], v[1], vs);
    };
    bf16x8 vf = widen_v(0);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const bf16x8 now = vf;
      if (db + 1 < D / 16) vf = widen_v(db + 1);  // under this fragment's products
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) w.o[rb][db] = mfma16x16x32(now, pf[rb], w.o[rb][db]);
      if (hf == 1 && db % (D / 64) == D / 64 - 1) refill_k(db / (D / 64));
      if (MASKED)
        __builtin_amdgcn_sched_barrier(0);
      else
        interleave<RB, 4>();
    }
  }
  return true;
}

// Makes the outputs NaN that a NaN code of this block reaches: those of the rows
// that see its key, in its column.
template <int RB, int D>
__device__ __forceinline__ void spread_nan(Wave8<RB, D>& w, const unsigned char* vp, int key0, int first, int end) {
  const int lg = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const uint64_t win = keys_seen(w.sees[rb], key0 + 4 * lg - first);
    bf16x8 sf[2];  // 1 where the row sees the key
#pragma unroll
    for (int j = 0; j < 16; ++j) sf[j >> 3][j & 7] = (__bf16)(float)((uint32_t)(win >> (16 * (j >> 2) + (j & 3))) & 1u);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(vp + db * 1024);
      u32x4 ind;  // 1 (code 0x38) where V is NaN
#pragma unroll
      for (int t = 0; t < 4; ++t) ind[t] = nan_bytes(v[t] & bytes_before(key0 + 16 * t + 4 * lg, end)) * 0x38u;
      f32x4 n = {0.f, 0.f, 0.f, 0.f};
      n = mfma16x16x32(widen8(ind[0], ind[1], 1.f), sf[0], n);
      n = mfma16x16x32(widen8(ind[2], ind[3], 1.f), sf[1], n);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w.o[rb][db][e] = __uint_as_float(n[e] > 0.f ? 0x7fc00000u : __float_as_uint(w.o[rb][db][e]));
    }
  }
}

// At head dimension 64 LDS holds two waves per SIMD, and half the registers each are
// enough (five blocks spill 52): 16 requests of 24,576 keys, 8 heads: of 64 rows 105 us,
// 133 with one wave per SIMD; of 72 rows 118-126 and 149.
template <int RB, int D>
__global__ __launch_bounds__(kWave, D == 64 ? 2 : 1)
void kv8_attn_kernel(AttnShape s, AttnBatch bt, Kv8Pool pool, int nchunks, const uint16_t* __restrict__ q,
                     AttnPartials parts) {
  using R = Ring<D>;
  __shared__ __align__(1024) unsigned char ring[R::kSlots * R::kHalf];
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, lg = lane >> 4;
  // Row groups of one (chunk, KV head) are 8 workgroups apart, on one XCD: the
  // second read of a block hits its L2.
  const int per = 8 * s.row_groups;
  const int item = blockIdx.x / per * 8 + (blockIdx.x & 7);
  const int rg = blockIdx.x % per >> 3;
  if (item >= nchunks * s.Hkv) return;
  const int head = item % s.Hkv;
  const int c = item / s.Hkv;
  // The largest request with chunk_prefix <= c: one load, a request per lane.
  const int prefix = lane < bt.nreq ? bt.chunk_prefix[lane] : INT32_MAX;
  const int lo = __popcll(__ballot(prefix <= c)) - 1;
  const int req = bt.req0 + lo;
  const int end = bt.kv_len[lo], first = end - s.G;
  const int key_begin = (c - __builtin_amdgcn_readlane(prefix, lo)) * s.chunk_keys;
  const int key_end = min(key_begin + s.chunk_keys, end);
  const int ntiles = (key_end - key_begin + kKeyBlock - 1) / kKeyBlock;
  const int blk0 = key_begin / kKeyBlock;

  // Lane j: where block j of the chunk lies, and its scales.
  const int shift = pool.page_shift - 6;
  const int blk = blk0 + min(lane, ntiles - 1);
  int page = pool.table[(int64_t)req * pool.max_pages + (blk >> shift)];
  page = min(max(page, 0), pool.num_pages - 1);
  const int64_t at = (((int64_t)page * s.Hkv + head) << shift) + (blk & ((1 << shift) - 1));
  const uint32_t at_lo = (uint32_t)at, at_hi = (uint32_t)(at >> 32);
  const int ks_all = pool.k_scale[at], vs_all = pool.v_scale[at];

  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
  const uint32_t off = lane * 16;
  // DMAs i .. n - 1 of half `half` (block half / 2: K, then V) into place `slot`.
  auto fetch = [&](int half, int slot, int i, int n) {
    const int t = half >> 1;
    const int64_t blk_at = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_hi, t) << 32) |
                                     (uint32_t)__builtin_amdgcn_readlane((int)at_lo, t));
    const uint8_t* src = ((half & 1) ? pool.v : pool.k) + blk_at * R::kHalf;
    const uint32_t dst = ring_at + slot * R::kHalf;
#pragma unroll
    for (int j = i; j < n; ++j) ring_dma(src + j * 1024, off, dst + j * 1024);
  };
  const int halves = __builtin_amdgcn_readfirstlane(2 * ntiles);
  // Half n is in once only DMAs of later halves are on their way: of as many as were
  // asked for by then, MOST if there are that many.
  auto wait_half = [&](int n, auto most) {
    constexpr int kMost = decltype(most)::value;
    static_assert(kMost > 2 * R::kOps && kMost <= 3 * R::kOps && kMost < 64, "vmcnt holds 6 bits");
    const int after = halves - 1 - n;
    if (after >= 3) wait_vmcnt<kMost>();
    else if (after == 2) wait_vmcnt<2 * R::kOps>();
    else if (after == 1) wait_vmcnt<R::kOps>();
    else wait_vmcnt<0>();
    asm volatile("" ::: "memory");
  };
  auto fill = [&] {
#pragma unroll
    for (int n = 0; n < R::kSlots; ++n)
      if (n < halves) fetch(n, n, 0, R::kOps);
  };
  fill();

  Wave8<RB, D> w;
  const int whole = min(max((first + 1 - key_begin) / kKeyBlock, 0), ntiles);  // blocks that every row sees whole
  uint64_t masks = 1;  // a chunk of whole blocks ends with position 0 at the latest: all rows see it
  if (whole < ntiles) masks = position_mask(bt.parent != nullptr ? bt.parent + (int64_t)req * (s.G - 1) : nullptr, s.G);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = (rg * RB + rb) * 16 + lr;
    const int rc = min(row, s.rows - 1);
    const int j = rc / s.group, h = head * s.group + rc - j * s.group;
    const uint16_t* src = q + (((int64_t)req * s.G + j) * s.Hq + h) * D + 16 * lg;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w.q[rb][i] = load_bf16x8(src + 64 * (i >> 1) + 8 * (i & 1));
    const uint32_t a = __shfl((uint32_t)masks, j), b = __shfl((uint32_t)(masks >> 32), j);
    w.sees[rb] = ((uint64_t)b << 32) | a;
    w.m[rb] = kNoKey;
  }

  auto pow2 = [&](int bytes, int t) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane(bytes, t) << 23);
  };
  bool again = false;
  for (;;) {  // twice at most
    for (int t = 0; again && t < ntiles; ++t) {
      fetch(2 * t, 0, 0, R::kOps);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      float zero[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) zero[rb] = 0.f;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        u32x4 k[2][D / 64];
        f32x4 sc[RB][2];
        float mx[RB];
        read_k<D>(ring + off, hf, k);
        if (t < whole)
          half_scores<RB, D, false>(w, k, hf, pow2(ks_all, t), 0, zero, sc, [](int) {});
        else
          half_scores<RB, D, true>(w, k, hf, pow2(ks_all, t), key_begin + t * kKeyBlock + 4 * lg - first, zero, sc,
                                   [](int) {});
        half_max<RB>(sc, mx);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) w.m[rb] = fmaxf(w.m[rb], mx[rb]);
      }
      lds_wait();  // read before the next DMA overwrites it
    }
    if (again) fill();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      w.l[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) w.o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    w.nan = 0;
    // Two loops: in one, the compiler widens the codes before it branches to
    // either kind of block, and spills what that takes.
    int t = 0, ks = 0;  // ks: place of K of block t
    bool done = true;
    auto step = [&](int block, auto masked) {
      constexpr bool MASKED = decltype(masked)::value;
      const int t = __builtin_amdgcn_readfirstlane(block);  // scalar branches
      const int vs = ks + 1 == R::kSlots ? 0 : ks + 1;    // place of V of block t
      const int last = ks == 0 ? R::kSlots - 1 : ks - 1;  // of V of block t - 1, free now
      const int nv = 2 * t - 1 + R::kSlots, nk = nv + 1;  // the halves that take free places
      // Before K of block t is read, three halves after it have been asked for; before V,
      // two and half of the one that takes the last V's place.
      static_assert(R::kSlots == 5, "as many as the waits count");
      wait_half(2 * t, Int<3 * R::kOps>());
      done = fold_block<RB, D, MASKED>(
          w, ring + ks * R::kHalf + off, ring + vs * R::kHalf + off, pow2(ks_all, t), pow2(vs_all, t),
          grow_limit(__builtin_amdgcn_readlane(vs_all, t)), s.scale_log2, key_begin + t * kKeyBlock, first, end, again,
          [&] { wait_half(2 * t + 1, Int<5 * R::kOps / 2>()); },
          [&](int n) {
            if (t > 0 && nv < halves) fetch(nv, last, n * R::kOps / 4, (n + 1) * R::kOps / 4);
          },
          [&](int n) {
            if (nk < halves) fetch(nk, ks, n * R::kOps / 4, (n + 1) * R::kOps / 4);
          });
      ks = vs + 1 == R::kSlots ? 0 : vs + 1;
    };
    for (; t < whole && done && !again; ++t) step(t, Kind<false>());
    for (; t < ntiles && done; ++t) step(t, Kind<true>());
    if (done || again) break;
    again = true;
    wait_vmcnt<0>();
    lds_wait();
  }

  if (__builtin_expect(__ballot(w.nan != 0) != 0, 0)) {
    for (int n = again ? 0 : whole; n < ntiles; ++n) {
      lds_wait();
      fetch(2 * n + 1, 0, 0, R::kOps);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      spread_nan<RB, D>(w, ring + off, key_begin + n * kKeyBlock, first, end);
    }
  }

  const int64_t slot = (int64_t)(bt.chunk_base + c) * s.Hkv + head;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = (rg * RB + rb) * 16 + lr;
    const float l = sum_over_groups(w.l[rb]);
    if (row < s.rows) {
      if (lg == 0) {
        parts.m[slot * s.rows + row] = w.m[rb];
        parts.l[slot * s.rows + row] = l;
      }
      float* dst = parts.o + (slot * s.rows + row) * D + 4 * lg;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(dst + db * 16) = w.o[rb][db];
    }
  }
}

// Joins the partials of each (request, position, head) in chunk order: O =
// sum_c w_c o_c / sum_c w_c l_c, w_c = 2^(scale_log2 (m_c - max m)).  A thread
// holds four columns.
template <int D, int MOST>
__global__ __launch_bounds__(256)
void kv8_merge_kernel(AttnShape s, AttnBatch bt, AttnPartials parts, uint16_t* __restrict__ out) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= s.rows * (D / 4)) return;
  const int head = blockIdx.y, b = blockIdx.z;
  const int row = i / (D / 4), d = i % (D / 4) * 4;
  const int c0 = bt.chunk_base + bt.chunk_prefix[b], c1 = bt.chunk_base + bt.chunk_prefix[b + 1];
  float m = kNoKey, den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  // Chunks c .. c + N - 1, whose partials are on their way together.
  auto join = [&](int c, auto count) {
    constexpr int N = decltype(count)::value;
    float mc[N], lc[N];
    f32x4 oc[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int64_t at = ((int64_t)min(c + k, c1 - 1) * s.Hkv + head) * s.rows + row;
      mc[k] = parts.m[at];
      lc[k] = parts.l[at];
      oc[k] = *reinterpret_cast<const f32x4*>(parts.o + at * D + d);
    }
    float mn = m;
#pragma unroll
    for (int k = 0; k < N; ++k) mn = fmaxf(mn, mc[k]);
    const float alpha = __builtin_amdgcn_exp2f((m - mn) * s.scale_log2);
    den *= alpha;
    num *= alpha;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (c + k < c1) {
        const float a = __builtin_amdgcn_exp2f((mc[k] - mn) * s.scale_log2);
        den = fmaf(a, lc[k], den);
        num += a * oc[k];
      }
    m = mn;
  };
  // Many at once where there are many, no more than there are where there are few:
  // where no request has more than four, MOST is 4, and the kernel needs a third of the
  // registers.  One request of 8,000 keys in 64 chunks, 40 rows, D = 128, whole call:
  // 23.3 us with up to 16, 25.6 with 8, 29.3 with 4; 64 requests of 2,000 keys in two:
  // 77 us with MOST 4, 81 with 16.
  for (int c = c0; c < c1;) {
    const int n = c1 - c;
    if (MOST > 8 && n > 8) {
      join(c, Int<16>());
      c += 16;
    } else if (MOST > 4 && n > 4) {
      join(c, Int<8>());
      c += 8;
    } else if (n > 2) {
      join(c, Int<4>());
      c += 4;
    } else {
      join(c, Int<2>());
      c += 2;
    }
  }
  const int j = row / s.group, h = head * s.group + row - j * s.group;
  uint16_t* dst = out + (((int64_t)(bt.req0 + b) * s.G + j) * s.Hq + h) * D + d;
  const float r = 1.f / den;
  const bf16x2 lo = __builtin_convertvector((f32x2{num[0] * r, num[1] * r}), bf16x2);
  const bf16x2 hi = __builtin_convertvector((f32x2{num[2] * r, num[3] * r}), bf16x2);
  *reinterpret_cast<u32x2*>(dst) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

int64_t cu_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n <= 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// 16-row blocks of a wave.  One holds up to five (at head dimension 128 O takes 32
// registers of each, Q 16); more rows are split over row groups, a wave each.  Where the
// caches are a few blocks of keys per place, what counts is how long a wave takes for
// its own: two row blocks, or one where there are three (two would leave a wave half
// empty, which costs more than a third wave; of five and more they do not), and
// the groups read the same keys from L2.  `blocks`: 64-key blocks times heads, few up to
// 10 per CU at D = 128 and 32 at 64, where twice as many waves run at once.
// 8 heads, 4 and 24 requests of one length, us with one or two row blocks / with all:
//   D = 128, 48 rows:  2,000 blocks 25, 29 / 25, 28; 3,200 31, 40 / 33, 32; 6,000 47, 66 / 40, 41
//            72 rows:  2,000 30, 35 / 34, 33; 3,200 37, 47 / 39, 40; 6,000 56, 77 / 49, 51
//   D = 64,  48 rows:  2,000 18, 17 / 20, 18; 6,000 29, 30 / 33, 31; 8,100 35, 36 / 37, 34
//            72 rows:  2,000 21, 22 / 28, 26; 6,000 36, 36 / 45, 42; 8,100 44, 45 / 49, 46
// 4 requests of 1,500 keys, D = 128, one and two row blocks: 40 rows 15.2 and 16.2, 72 rows
// 21.2 and 19.6, 112 rows 27.7 and 23.0.
int row_groups(int rows, int D, int64_t blocks) {
  const int b = (rows + 15) / 16;
  const int most = blocks > (D == 64 ? 32 : 10) * cu_count() ? kMaxBlocks : b == 3 ? 1 : 2;
  return (b + most - 1) / most;
}
int blocks_of(int rows, int groups) { return ((rows + 15) / 16 + groups - 1) / groups; }

// Workgroups (one wave, one item each) that run at once: what LDS holds.
int64_t places(int D) { return cu_count() * (D == 64 ? 8 : 4); }

}  // namespace

AttnShape kv8_shape(int G, int Hq, int Hkv, int D, float scale, const int32_t* kv_len, int B) {
  AttnShape s;
  s.G = G;
  s.Hq = Hq;
  s.Hkv = Hkv;
  s.D = D;
  s.group = Hq / Hkv;
  s.rows = G * s.group;
  int64_t blocks = 0;
  for (int b = 0; b < B; ++b) blocks += (kv_len[b] + kKeyBlock - 1) / kKeyBlock;
  s.row_groups = row_groups(s.rows, D, blocks * Hkv);
  s.scale_log2 = scale * kLog2e;
  // For a half to four rounds of items over the CUs' places the shortest chunk that
  // fits them; of these the one that is done first, counted in keys of a wave with up to
  // three blocks (with more a wave's own instructions bound it).  Up to one round
  // takes a chunk and an item's start (rows, pages, first block); items in more rounds
  // are handed out as places come free, and the last ones end half a chunk apart.  Then
  // the partials are written and read, 8 keys' bytes a row.  More items than
  // four rounds only with the longest chunk: the workspace holds no more partials.
  // Before and after the half round and the partials' cost came in: 8,000 keys, 8
  // heads of 40 rows, D = 128, 37 and 25.6 us; 13 requests of 1,500 keys, 48 rows, D = 64,
  // 24.2 and 21.3; with 80 rows, D = 128, 41.7 where five blocks count as three, 37.6 as it is.
  const int64_t slots = places(D);
  const int64_t start = 192 + 2 * s.rows;
  const int work = blocks_of(s.rows, s.row_groups) > 3 ? 3 : 2;
  auto items = [&](int tiles) {
    const int keys = tiles * kKeyBlock;
    int64_t n = 0;
    for (int b = 0; b < B; ++b) n += (kv_len[b] + keys - 1) / keys;
    return n * Hkv * s.row_groups;
  };
  const int64_t total = items(1) * kKeyBlock;
  int64_t best = INT64_MAX;
  int most = kMaxTiles;
  s.chunk_keys = kMaxTiles * kKeyBlock;
  for (int r : {1, 2, 4, 6, 8}) {  // half rounds
    const int64_t fit = r * slots / 2;
    if (items(most) > fit) continue;
    int lo = 1, hi = most;  // the shortest chunk lies in [lo, hi]
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (items(mid) <= fit) hi = mid; else lo = mid + 1;
    }
    const int64_t keys = int64_t(lo) * kKeyBlock;
    const int64_t n = items(lo);
    const int64_t cost = (r <= 2 ? keys * work / 2 + start : (total * work / 2 + n * start) / slots + keys / 2) +
                         n * s.rows * 8 / slots;
    if (cost < best) {
      best = cost;
      s.chunk_keys = lo * kKeyBlock;
    }
    most = lo;
    if (lo == 1) break;
  }
  return s;
}

int64_t kv8_max_chunks(int Hkv, int D, int B, int64_t max_kv_len) {
  const int64_t most = std::min(4 * places(D) / Hkv, B * ((max_kv_len + kKeyBlock - 1) / kKeyBlock));
  const int64_t at_longest = B * ((max_kv_len + kMaxTiles * kKeyBlock - 1) / (kMaxTiles * kKeyBlock));
  return std::max(most, at_longest);
}

hipError_t launch_kv8_attention(const AttnShape& s, const AttnBatch& batch, const Kv8Pool& pool, int nchunks,
                                const void* q, AttnPartials parts, void* out, hipStream_t stream) {
  const dim3 grid((nchunks * s.Hkv + 7) / 8 * 8 * s.row_groups), block(kWave);
#define SDV_KV8(RB)                                                                                               \
  case RB:                                                                                                        \
    if (s.D == 128)                                                                                               \
      hipLaunchKernelGGL((kv8_attn_kernel<RB, 128>), grid, block, 0, stream, s, batch, pool, nchunks,              \
                         static_cast<const uint16_t*>(q), parts);                                                 \
    else                                                                                                          \
      hipLaunchKernelGGL((kv8_attn_kernel<RB, 64>), grid, block, 0, stream, s, batch, pool, nchunks,               \
                         static_cast<const uint16_t*>(q), parts);                                                 \
    break;
  switch (blocks_of(s.rows, s.row_groups)) {
    SDV_KV8(1) SDV_KV8(2) SDV_KV8(3) SDV_KV8(4) SDV_KV8(5)
    default: return hipErrorInvalidValue;
  }
#undef SDV_KV8
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 mgrid((s.rows * (s.D / 4) + 255) / 256, s.Hkv, batch.nreq);
  int most = 0;
  for (int b = 0; b < batch.nreq; ++b) most = std::max(most, batch.chunk_prefix[b + 1] - batch.chunk_prefix[b]);
#define SDV_MERGE(DIM, MOST)                                                                                      \
  hipLaunchKernelGGL((kv8_merge_kernel<DIM, MOST>), mgrid, dim3(256), 0, stream, s, batch, parts,                 \
                     static_cast<uint16_t*>(out))
  if (s.D == 128) {
    if (most > 4) SDV_MERGE(128, 16); else SDV_MERGE(128, 4);
  } else {
    if (most > 4) SDV_MERGE(64, 16); else SDV_MERGE(64, 4);
  }
#undef SDV_MERGE
  return hipGetLastError();
}

}  // namespace sdv
