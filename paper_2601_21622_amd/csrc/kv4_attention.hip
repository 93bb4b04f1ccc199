// Verification attention over a paged 4-bit cache (split-KV) for gfx950.
//
//   O = softmax(scale * Q K^T + mask) V,  K = code * 2^e of its key's 32 columns, V = code * s of its key.
//
// The G * group queries that share a KV head are the rows of one KV head, in blocks of 16.  Two ways:
//  * In chunks: one wave, a workgroup of its own, per work item (chunk of whole 64-key
//    blocks of one request, KV head, group of up to five row blocks); each item writes a partial
//    (reference maximum, sum, O) and the merge joins them in chunk order.
//  * Joined: a workgroup of eight waves takes a whole request, KV head and row block, and joins its
//    waves' O in LDS: where requests are short, one launch and no partials.
// Which way, and how long a chunk is, kv4_shape decides by what either takes.
//
// What bounds it: with one row block the caches' stream, 6.0-6.1 TB/s on long chunks (4 x 200,000 keys, 8 KV
// heads, D = 128, 857 MB: 140 us with the merge) and 5.2 where items are short (64 pooled requests of
// 128-8,192 keys, 32 heads, 547 MB: kernel 105-109 us).  With more row blocks a wave's own instructions: of
// 72 rows (five blocks) 16 x 16,384-32,768 keys take 154-168 us, where the products alone are 83-96 at a
// large library product's rate and the stream 70.  A wave issues an instruction about every five cycles, a
// product hides two vector instructions, an exponential takes eight cycles, a widening four and a half; 917
// instructions fold 64 keys into 80 rows.  Five row blocks in one wave beat three and two in two (165 and 190
// us the whole call): keys are widened once, and two waves drift apart until the second reads the caches
// again from memory (820 MB instead of 415).
//
// A K fragment is what a lane loads: 8 codes of one key, whose scale the widening
// instruction takes.  V lies key by key, so that an append writes rows, and is transposed on
// its way out of LDS: a lane gets one column of the 16 keys whose scores it holds
// (S^T = K Q^T; tile t: keys 16 t + 4 g + r of group g = lane / 16), which is all that
// O^T += V^T P^T needs.  V's scale multiplies the weight, in float32; for the product with V's codes the weight
// is bfloat16, for its range, which a product with a scale needs.  A wave of one row block holds it in two such
// numbers, the second what the first leaves, 2^-16 of each term: outputs are then off by their own rounding (1.6e-3
// of them against 64 bits, one token over 1,000 keys; 2.5e-3 with one number).  That takes 24 vector instructions and the
// products with V once more; us with two and one: 8.8 and 8.4 (that case), 116.5 and 115.3 (the pooled requests), 14.7 and
// 13.9 (13 trees of 37-3,001 keys, D = 64), 83.5 and 77 (4 x 200,000 keys, D = 64).  Waves of more row blocks, bound by
// their instructions, round it once (half a step: 2^-8 of each term; 2.2e-3 of the output where its rounding is
// 1.7e-3): two numbers take 230 us instead of 164 (16 x 16,384-32,768 keys, 72 rows) and 145 instead of 111 (16 x 24,576, D = 64).
// The 4-bit matrix instructions would take K without widening, but keep
// too few bits of their sums: 6.6e-5 of the sum of magnitudes of 128 products, measured.
//
// Softmax in the log2 domain, against a reference that is the row's maximum as of the
// last time it was set: a lane's weights of a block may sum to 2^8 before the reference is set again and O
// rescaled, which a wave notices by the sums that it keeps anyway.  That happens outside the loop over the blocks:
// inside, the compiler spills O, and a spill's reload waits for the DMAs before it.  Accumulators start
// at -reference.  Where a reference is large (2^16 in the log2 domain: sums that start there round differently from those that
// start at zero, by up to 2^-8 and, further up, by any factor), and in joined requests for the block that sets it, scores are
// summed from zero and the reference is subtracted from the sum: equal scores stay equal, and none exceeds its own maximum.
#include <algorithm>

#include "fp4.h"
#include "fp8.h"
#include "kv_wave.h"

namespace sdv {

namespace {

constexpr int kMaxTiles4 = 64;   // blocks per chunk: one lane holds one block's page
// Waves of a workgroup that takes a request.  Sixteen, on rings of one block (weights in one number): 9.8 us where
// eight take 8.9 (1,000 keys, one token, D = 128), 14.2 and 12.5 (4 x 1,500 keys, 72 rows).
constexpr int kJoinWaves = 8;
constexpr int kManyChunks = 16;  // chunks of a request that one thread joins
constexpr float kNoKey4 = -3.402823466e38f;  // reference of a row that has seen no key: no score lies below it
constexpr float kGrow = 256.f;      // sum of a lane's 16 weights of a block that sets a new reference
constexpr float kCareful = 65536.f;  // log2 magnitude of a reference from which sums start at zero

// A wave's ring: the K and V of two blocks, codes and then scales.
template <int D>
struct Ring4 {
  static constexpr int kCodes = 32 * D;
  static constexpr int kHalf = kCodes + 256;
  static constexpr int kOps = D / 32 + 1;  // DMAs of a half
};

// The DMAs of a half: D / 32 KB of codes, 16 bytes a lane each, then a dword a lane of
// scales, whose base and offset are their own.  As ring_dma, with one base for the codes: a
// DMA's offset is added on both sides.
template <int D>
__device__ __forceinline__ void half_dma(const void* codes, uint32_t off16, uint32_t lds, const void* scales, uint32_t off4,
                                         uint32_t lds_scales) {
  uint64_t from;
  if (D == 128)
    asm volatile(
        "s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0 nt\n\t"
        "global_load_lds_dwordx4 %2, %0 offset:0x400 nt\n\tglobal_load_lds_dwordx4 %2, %0 offset:0x800 nt\n\t"
        "global_load_lds_dwordx4 %2, %0 offset:0xc00 nt"
        : "=&s"(from)
        : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off16), "s"(codes)
        : "m0", "memory");
  else
    asm volatile(
        "s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0 nt\n\t"
        "global_load_lds_dwordx4 %2, %0 offset:0x400 nt"
        : "=&s"(from)
        : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off16), "s"(codes)
        : "m0", "memory");
  asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0 nt"
               : "=&s"(from)
               : "s"(__builtin_amdgcn_readfirstlane(lds_scales)), "v"(off4), "s"(scales)
               : "m0", "memory");
}

// The lane's number, counted where it is asked for: a copy held in a register would be
// the first to be spilled, and a spill's reload waits for the DMAs before it.
__device__ __forceinline__ uint32_t lane_here() {
  uint32_t l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
  return l;
}

typedef __attribute__((__vector_size__(2 * sizeof(int)))) int i32x2;

// One column of 16 keys, from the 8 bytes (16 columns of a key) that each of 16 lanes
// points at: lane i of them gets column i, the codes in the order of the lanes.
__device__ __forceinline__ i32x2 lds_read_tr4(const unsigned char* p) {
  return __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) i32x2*)p);
}

// bfloat16 numbers that a weight is held in for its products.
template <int RB>
constexpr int kParts = RB == 1 ? 2 : 1;

// Four weights as two bfloat16 numbers each, from entry i on: rounded, and what that leaves of them, rounded.
__device__ __forceinline__ void put_weights(bf16x8 (&pf)[2], int i, const float (&y)[4]) {
  uint32_t first = 0x0000bf80u, second = 0xbf800000u;  // -1 and 0, 0 and -1, held in registers
  asm("" : "+s"(first), "+s"(second));
#pragma unroll
  for (int r = 0; r < 4; r += 2) {
    const bf16x2 hi = __builtin_convertvector((f32x2{y[r], y[r + 1]}), bf16x2);
    const f32x2 rest = {__builtin_amdgcn_fdot2_f32_bf16(hi, __builtin_bit_cast(bf16x2, first), y[r], false),
                        __builtin_amdgcn_fdot2_f32_bf16(hi, __builtin_bit_cast(bf16x2, second), y[r + 1], false)};
    const bf16x2 lo = __builtin_convertvector(rest, bf16x2);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      pf[0][i + r + k] = hi[k];
      pf[1][i + r + k] = lo[k];
    }
  }
}

template <int RB, int D>
struct Wave4 {
  bf16x8 q[RB][D / 32];
  f32x4 o[RB][D / 16];
  float m[RB], l[RB];  // reference of the unscaled scores (kNoKey4: no key seen yet), sum
  uint64_t sees[RB];   // of the step's own positions
};

// The instructions since the last call as M products with at most V vector
// instructions among them, one product first, so that the vector ones issue
// while the matrix core works.
template <int M, int V>
__device__ __forceinline__ void interleave4() {
#pragma unroll
  for (int i = 0; i < M; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, (V + M - 1) / M, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Scores of half `hf` of a block (tiles 2 hf and 2 hf + 1), accumulated from `base`; what a row does not
// see is -inf.  ks: the key's scale bytes of the four tiles.
template <int RB, int D, bool MASKED>
__device__ __forceinline__ void half_scores4(const Wave4<RB, D>& w, const unsigned char* kp, int hf, uint32_t ks, int off,
                                             const float (&base)[RB], f32x4 (&sc)[RB][2]) {
  constexpr int kSteps = D / 32;  // 32-wide steps of a score tile
  const int lane = lane_here();
  uint32_t codes[2 * kSteps];
  float scale[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    scale[t] = __uint_as_float(((ks >> (16 * hf + 8 * t)) & 255u) << 23);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      codes[t * kSteps + i] = reinterpret_cast<const uint32_t*>(kp + (2 * hf + t) * (8 * D) + lane * (D / 8))[i];
  }
  bf16x8 kf = widen8_fp4(codes[0], scale[0]);
  // The two tiles in turn: a product's sum is not asked for by the next RB * 2 - 1.
#pragma unroll
  for (int n = 0; n < 2 * kSteps; ++n) {
    const int t = n % 2, i = n / 2;
    const bf16x8 now = kf;
    if (n + 1 < 2 * kSteps) kf = widen8_fp4(codes[(n + 1) % 2 * kSteps + (n + 1) / 2], scale[(n + 1) % 2]);  // under this step's products
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      sc[rb][t] = mfma16x16x32(now, w.q[rb][i], i == 0 ? f32x4{base[rb], base[rb], base[rb], base[rb]} : sc[rb][t]);
    interleave4<RB, 4>();
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

template <int D>
__device__ __forceinline__ uint32_t key_scales4(const unsigned char* kp) {
  const int lane = lane_here();
  return *reinterpret_cast<const uint32_t*>(kp + Ring4<D>::kCodes + ((lane >> 4) * (D / 4) / kGroup4 * 16 + (lane & 15)) * 4);
}

// Sets the references that this block's scores outgrow, and rescales O and the sums.
// Returns whether a reference is large.
template <int RB, int D>
__device__ __forceinline__ bool set_reference(Wave4<RB, D>& w, const unsigned char* kp, float scale_log2, int off) {
  float zero[RB], x[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    zero[rb] = 0.f;
    x[rb] = kNoKey4;
  }
  const uint32_t ks = key_scales4<D>(kp);
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    f32x4 sc[RB][2];
    half_scores4<RB, D, true>(w, kp, hf, ks, off, zero, sc);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        x[rb] = fmaxf(fmaxf(x[rb], fmaxf(sc[rb][t][0], sc[rb][t][1])), fmaxf(sc[rb][t][2], sc[rb][t][3]));
  }
  bool large = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float m = fmaxf(w.m[rb], max_over_groups(x[rb]));
    const float alpha = __builtin_amdgcn_exp2f((w.m[rb] - m) * scale_log2);
    w.m[rb] = m;
    w.l[rb] *= alpha;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) w.o[rb][db] *= alpha;
    large |= m > kNoKey4 && fabsf(m) * scale_log2 >= kCareful;
  }
  return __ballot(large) != 0;
}

// O += P V: V's columns come out of LDS transposed.
template <int RB, int D>
__device__ __forceinline__ void add_products4(Wave4<RB, D>& w, const unsigned char* vp, const bf16x8 (&pf)[RB][2][kParts<RB>]) {
  const int lane = lane_here(), lr = lane & 15, lg = lane >> 4;
  const unsigned char* vl = vp + (16 * (lr / 4) + 4 * lg + lr % 4) * 8;
  i32x2 v[D / 16];
#pragma unroll
  for (int db = 0; db < D / 16; ++db) v[db] = lds_read_tr4(vl + db * 512);
  bf16x8 vf = widen8_fp4((uint32_t)v[0][0], 1.f);
#pragma unroll
  for (int n = 0; n < D / 8; ++n) {
    const int db = n % (D / 16), hf = n / (D / 16);
    const bf16x8 now = vf;
    if (n + 1 < D / 8) vf = widen8_fp4((uint32_t)v[(n + 1) % (D / 16)][(n + 1) / (D / 16)], 1.f);  // under this fragment's products
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < kParts<RB>; ++i) w.o[rb][db] = mfma16x16x32(now, pf[rb][hf][i], w.o[rb][db]);
    interleave4<RB * kParts<RB>, 4>();
  }
}

// Folds one block into O and the sums; false, with nothing changed, when a row's scores outgrow its
// reference (not asked where the reference is this block's own, `own`).  MASKED serves large references
// too (`careful`: scores are summed from zero).  refill_k asks for the block that takes K's place.
template <int RB, int D, bool MASKED, typename RefillK>
__device__ __forceinline__ bool fold_block4(Wave4<RB, D>& w, const unsigned char* kp, const unsigned char* vp, float scale_log2,
                                            int off, bool own, bool careful, RefillK refill_k) {
  float base[RB], sum[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    base[rb] = w.m[rb] > kNoKey4 && !(MASKED && careful) ? -w.m[rb] : 0.f;
    sum[rb] = 0.f;
  }
  const uint32_t ks = key_scales4<D>(kp);
  bf16x8 pf[RB][2][kParts<RB>];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    f32x4 sc[RB][2];
    half_scores4<RB, D, MASKED>(w, kp, hf, ks, off, base, sc);
    const int lg = lane_here() >> 4;
    u32x2 vs[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) vs[t] = *reinterpret_cast<const u32x2*>(vp + Ring4<D>::kCodes + (32 * hf + 16 * t + 4 * lg) * 2);
    if (MASKED && careful) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float m = w.m[rb] > kNoKey4 ? w.m[rb] : 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[rb][t][r] -= m;
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      [[maybe_unused]] float ys[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t pair = vs[t][r / 2];
        const float scale = __uint_as_float(r & 1 ? pair & 0xffff0000u : pair << 16);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const float p = __builtin_amdgcn_exp2f(sc[rb][t][r] * scale_log2);
          sum[rb] += p;
          float y = p * scale;
          if (MASKED) {
            // What a row does not see, and what lies past the last key, has a scale of any kind.
            const uint32_t see = (uint32_t)(keys_seen(w.sees[rb], off) >> (32 * hf + 16 * t + r)) & 1u;
            y = __uint_as_float(see ? __float_as_uint(y) : 0u);
          }
          if constexpr (kParts<RB> == 1) pf[rb][hf][0][t * 4 + r] = (__bf16)y;
          else ys[r] = y;
        }
      }
      if constexpr (kParts<RB> == 2) put_weights(pf[0][hf], t * 4, ys);
    }
    // The rounded weights are all that is kept of the scores.
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < kParts<RB>; ++i) asm volatile("" : "+v"(pf[rb][hf][i]));
  }
  bool grow = false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    grow |= sum[rb] > kGrow;
    // A row's first keys, whatever their weights.
    if (MASKED) grow |= !(w.m[rb] > kNoKey4) && (keys_seen(w.sees[rb], off) & 0x000f000f000f000full) != 0;
  }
  if (__builtin_expect(__ballot(grow) != 0 && !own, 0)) return false;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) w.l[rb] += sum[rb];
  lds_wait();  // K has been read
  refill_k();
  add_products4<RB, D>(w, vp, pf);
  return true;
}

// The same for one row block, which sets the reference itself (`set`: this block's scores are in it from now on);
// its registers allow the rescaling here.
template <int D, bool MASKED, typename RefillK>
__device__ __forceinline__ bool fold_block_one(Wave4<1, D>& w, const unsigned char* kp, const unsigned char* vp, float scale_log2,
                                               int off, bool set, bool& careful, RefillK refill_k) {
  const bool zero = set || (MASKED && careful);
  const float base[1] = {w.m[0] > kNoKey4 && !zero ? -w.m[0] : 0.f};
  const uint32_t ks = key_scales4<D>(kp);
  f32x4 sc[2][1][2];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) half_scores4<1, D, MASKED>(w, kp, hf, ks, off, base, sc[hf]);
  const int lg = lane_here() >> 4;
  u32x2 vs[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) vs[t] = *reinterpret_cast<const u32x2*>(vp + Ring4<D>::kCodes + (16 * t + 4 * lg) * 2);
  if (set) {
    float x = kNoKey4;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const f32x4 v = sc[t / 2][0][t % 2];
      x = fmaxf(fmaxf(x, fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
    }
    const float m = fmaxf(w.m[0], max_over_groups(x));
    const float alpha = __builtin_amdgcn_exp2f((w.m[0] - m) * scale_log2);
    w.m[0] = m;
    w.l[0] *= alpha;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) w.o[0][db] *= alpha;
    careful = __ballot(m > kNoKey4 && fabsf(m) * scale_log2 >= kCareful) != 0;
  }
  if (zero) {
    const float m = w.m[0] > kNoKey4 ? w.m[0] : 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[t / 2][0][t % 2][r] -= m;
  }
  bf16x8 pf[1][2][2];
  float sum = 0.f;
  const uint64_t win = MASKED ? keys_seen(w.sees[0], off) : 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float ys[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float scale = __uint_as_float(r & 1 ? vs[t][r / 2] & 0xffff0000u : vs[t][r / 2] << 16);
      const float p = __builtin_amdgcn_exp2f(sc[t / 2][0][t % 2][r] * scale_log2);
      sum += p;
      float y = p * scale;
      if (MASKED) {
        // What a row does not see, and what lies past the last key, has a scale of any kind.
        const uint32_t see = (uint32_t)(win >> (16 * t + r)) & 1u;
        y = __uint_as_float(see ? __float_as_uint(y) : 0u);
      }
      ys[r] = y;
    }
    put_weights(pf[0][t / 2], t % 2 * 4, ys);
  }
  bool grow = sum > kGrow;
  if (MASKED) grow |= !(w.m[0] > kNoKey4) && (win & 0x000f000f000f000full) != 0;  // a row's first keys, whatever their weights
  if (__builtin_expect(__ballot(grow) != 0 && !set, 0)) return false;
  w.l[0] += sum;
  lds_wait();  // K has been read
  refill_k();
  add_products4<1, D>(w, vp, pf);
  return true;
}

// Folds blocks blk0 .. blk0 + ntiles - 1 (at most 64) of request `lo` of the launch and one KV head
// into the rows from `row0` on; a ring of N blocks.  FEW: one row block, and so few blocks that the pass over the first
// one's scores counts (joined requests 0.3-0.8 us of 8-14 less; in chunks of a long stream 1 % more).
template <int RB, int D, int N, bool FEW>
__device__ __forceinline__ void fold_keys(Wave4<RB, D>& w, const AttnShape& s, const AttnBatch& bt, const Kv4Pool& pool,
                                          const uint16_t* __restrict__ q, unsigned char* ring, int lo, int head, int row0,
                                          int blk0, int ntiles) {
  using R = Ring4<D>;
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, lg = lane >> 4;
  const int req = bt.req0 + lo;
  const int first = bt.kv_len[lo] - s.G;
  const int key_begin = blk0 * kKeyBlock4;

  // Lane j: where block j lies.
  const int shift = pool.page_shift - 6;
  const int blk = blk0 + min(lane, max(ntiles - 1, 0));
  int page = pool.table[(int64_t)req * pool.max_pages + (blk >> shift)];
  page = min(max(page, 0), pool.num_pages - 1);
  const int64_t at = (((int64_t)page * s.Hkv + head) << shift) + (blk & ((1 << shift) - 1));
  const uint32_t at_lo = (uint32_t)at, at_hi = (uint32_t)(at >> 32);

  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
  // Block t's K (or V) into its place.
  auto fetch = [&](int t, bool is_v) {
    const int64_t b = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)at_hi, t) << 32) |
                                (uint32_t)__builtin_amdgcn_readlane((int)at_lo, t));
    const uint8_t* src = (is_v ? pool.v : pool.k) + b * R::kCodes;
    const uint32_t dst = ring_at + (t % N * 2 + (is_v ? 1 : 0)) * R::kHalf;
    const uint32_t l = lane_here();
    half_dma<D>(src, l * 16, dst,
                is_v ? reinterpret_cast<const uint8_t*>(pool.v_scale) + b * 128 : pool.k_scale + b * (2 * D),
                l * 4 & (is_v ? 127 : 2 * D - 1), dst + R::kCodes);
  };
#pragma unroll
  for (int t = 0; t < N; ++t)
    if (t < ntiles) {
      fetch(t, false);
      fetch(t, true);
    }

  const int whole = __builtin_amdgcn_readfirstlane(min(max((first + 1 - key_begin) / kKeyBlock4, 0), ntiles));  // blocks that every row sees whole
  uint64_t masks = 1;  // a chunk of whole blocks ends with position 0 at the latest: all rows see it
  if (whole < ntiles) masks = position_mask(bt.parent != nullptr ? bt.parent + (int64_t)req * (s.G - 1) : nullptr, s.G);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int rc = min(row0 + rb * 16 + lr, s.rows - 1);
    const int j = rc / s.group, h = head * s.group + rc - j * s.group;
    // Lane group g: the columns whose codes it holds of a key.
    const uint16_t* src = q + (((int64_t)req * s.G + j) * s.Hq + h) * D + (D / 4) * lg;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      w.q[rb][i] = load_bf16x8(src + 8 * i);
      // With five row blocks in the accumulation half of the registers, where the products take it from: the compiler
      // would move it to the other half for every block of keys.
      if (RB == 5) asm volatile("" : "+a"(w.q[rb][i]));
    }
    const uint32_t a = __shfl((uint32_t)masks, j), b = __shfl((uint32_t)(masks >> 32), j);
    w.sees[rb] = ((uint64_t)b << 32) | a;
    w.m[rb] = kNoKey4;
    w.l[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) w.o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  bool careful = false;  // some reference is large
  int own = 0;           // the block that last set references
  auto place = [&](int t) { return ring + t % N * 2 * R::kHalf; };
  auto offset = [&](int t) { return key_begin + t * kKeyBlock4 + 4 * ((int)lane_here() >> 4) - first; };
  // Block t is in once only the next N - 1 blocks' DMAs are on their way.
  auto arrived = [&](int t) {
    static_assert((N - 1) * 2 * R::kOps < 64 && N <= 4, "vmcnt holds 6 bits");
    const int after = min(ntiles - 1 - t, N - 1);
    if (N > 3 && after == 3) wait_vmcnt<6 * R::kOps>();
    else if (N > 2 && after == 2) wait_vmcnt<4 * R::kOps>();
    else if (after >= 1) wait_vmcnt<2 * R::kOps>();
    else wait_vmcnt<0>();
    asm volatile("" ::: "memory");
  };
  auto step = [&](int t, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    arrived(t);
    const unsigned char* kp = place(t);
    const bool more = t + N < ntiles;
    auto refill_k = [&] {
      if (more) fetch(t + N, false);
    };
    bool done;
    if constexpr (FEW)
      done = fold_block_one<D, MASKED>(w, kp, kp + R::kHalf, s.scale_log2, offset(t), t == own, careful, refill_k);
    else
      done = fold_block4<RB, D, MASKED>(w, kp, kp + R::kHalf, s.scale_log2, offset(t), t == own, careful, refill_k);
    if (done) {
      lds_wait();
      if (more) fetch(t + N, true);
    }
    return done;
  };
  int t = 0;
  if constexpr (!FEW) {
    if (ntiles > 0) arrived(0);
  }
  while (t < ntiles) {
    own = t;
    if constexpr (!FEW) careful = set_reference<RB, D>(w, place(t), s.scale_log2, offset(t));
    bool done = true;
    for (; t < whole && done && !careful; t += done) done = step(__builtin_amdgcn_readfirstlane(t), Kind<false>());
    for (; t < ntiles && done; t += done) done = step(__builtin_amdgcn_readfirstlane(t), Kind<true>());
  }
}

// One work item: rows from `row0` on of a chunk and KV head.
template <int RB, int D, int N>
__device__ __forceinline__ void attend_item(const AttnShape& s, const AttnBatch& bt, const Kv4Pool& pool,
                                            const uint16_t* __restrict__ q, const AttnPartials& parts, unsigned char* ring,
                                            int c, int head, int row0) {
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, lg = lane >> 4;
  // The largest request with chunk_prefix <= c: one load, a request per lane.
  const int prefix = lane < bt.nreq ? bt.chunk_prefix[lane] : INT32_MAX;
  const int lo = __popcll(__ballot(prefix <= c)) - 1;
  const int key_begin = (c - __builtin_amdgcn_readlane(prefix, lo)) * s.chunk_keys;
  const int key_end = min(key_begin + s.chunk_keys, bt.kv_len[lo]);
  Wave4<RB, D> w;
  fold_keys<RB, D, N, false>(w, s, bt, pool, q, ring, lo, head, row0, key_begin / kKeyBlock4,
                      __builtin_amdgcn_readfirstlane((key_end - key_begin + kKeyBlock4 - 1) / kKeyBlock4));
  const int64_t slot = (int64_t)(bt.chunk_base + c) * s.Hkv + head;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = row0 + rb * 16 + lr;
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

// The first `full` row groups take RB 16-row blocks, the others one less (UNEVEN).
template <int RB, bool UNEVEN, int D>
__global__ __launch_bounds__(kWave, RB > 3 ? 1 : 2)
void kv4_attn_kernel(AttnShape s, AttnBatch bt, Kv4Pool pool, int nchunks, int full, const uint16_t* __restrict__ q,
                     AttnPartials parts) {
  constexpr int N = RB > 3 ? 4 : 2;
  __shared__ __align__(1024) unsigned char ring[2 * N * Ring4<D>::kHalf];
  // Row groups of one (chunk, KV head) are 8 workgroups apart, on one XCD: the
  // second read of a block hits its L2.
  const int per = 8 * s.row_groups;
  const int item = blockIdx.x / per * 8 + (blockIdx.x & 7);
  const int rg = blockIdx.x % per >> 3;
  if (item >= nchunks * s.Hkv) return;
  const int head = item % s.Hkv, c = item / s.Hkv;
  if (!UNEVEN || rg < full)
    attend_item<RB, D, N>(s, bt, pool, q, parts, ring, c, head, rg * RB * 16);
  else
    attend_item<(UNEVEN ? RB - 1 : RB), D, N>(s, bt, pool, q, parts, ring, c, head, (rg * (RB - 1) + full) * 16);
}

// Four columns of a row's output, num / den.
__device__ __forceinline__ void store_four(uint16_t* out, const AttnShape& s, int req, int head, int row, int d, f32x4 num,
                                           float den) {
  const int j = row / s.group, h = head * s.group + row - j * s.group;
  const float inv = 1.f / den;
  const bf16x2 x = __builtin_convertvector((f32x2{num[0] * inv, num[1] * inv}), bf16x2);
  const bf16x2 y = __builtin_convertvector((f32x2{num[2] * inv, num[3] * inv}), bf16x2);
  *reinterpret_cast<u32x2*>(out + (((int64_t)req * s.G + j) * s.Hq + h) * s.D + d) =
      u32x2{__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y)};
}

// The requests of a launch, longest first: workgroups that have to share a CU are then short ones (13 requests
// of 37-3,001 keys, 312 workgroups: 14.6 us, 17.1 in the order of the batch).
struct ByLength {
  uint8_t req[kMaxReqPerLaunch];
};

// A request's blocks shared among the W waves of a workgroup, which join their O in
// LDS: no partials and no second launch, where a request's keys are few.
template <int W, int D>
__global__ __launch_bounds__(W * kWave, W / 4)
void kv4_attn_join_kernel(AttnShape s, AttnBatch bt, Kv4Pool pool, ByLength order, const uint16_t* __restrict__ q,
                          uint16_t* __restrict__ out) {
  constexpr int N = 2, kRing = 2 * N * Ring4<D>::kHalf, kRow = D + 4;  // bytes of a wave's ring; floats of a row of O, which spread over the banks
  static_assert(16 * kRow * 4 <= kRing, "a wave's O takes its ring's place");
  __shared__ __align__(1024) unsigned char ring[W * kRing];
  __shared__ float ms[W][16], ls[W][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int per = 8 * s.row_groups;
  const int item = blockIdx.x / per * 8 + (blockIdx.x & 7);
  const int rg = blockIdx.x % per >> 3;
  if (item >= bt.nreq * s.Hkv) return;
  const int head = item % s.Hkv, lo = order.req[item / s.Hkv];
  const int blocks = (bt.kv_len[lo] + kKeyBlock4 - 1) / kKeyBlock4;
  const int from = blocks * wave / W, to = blocks * (wave + 1) / W;
  unsigned char* const mine = ring + wave * kRing;
  Wave4<1, D> w;
  fold_keys<1, D, N, true>(w, s, bt, pool, q, mine, lo, head, rg * 16, from, __builtin_amdgcn_readfirstlane(to - from));
  lds_wait();
  float* const o = reinterpret_cast<float*>(mine) + lr * kRow + 4 * lg;
#pragma unroll
  for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(o + db * 16) = w.o[0][db];
  const float l = sum_over_groups(w.l[0]);
  if (lg == 0) {
    ms[wave][lr] = w.m[0];
    ls[wave][lr] = l;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * (D / 4); i += W * kWave) {
    const int r = i / (D / 4), d = i % (D / 4) * 4, row = rg * 16 + r;
    if (row >= s.rows) break;
    float m = ms[0][r];
#pragma unroll
    for (int k = 1; k < W; ++k) m = fmaxf(m, ms[k][r]);
    float den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float a = __builtin_amdgcn_exp2f((ms[k][r] - m) * s.scale_log2);
      den = fmaf(a, ls[k][r], den);
      num += a * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(ring + k * kRing) + r * kRow + d);
    }
    store_four(out, s, bt.req0 + lo, head, row, d, num, den);
  }
}

// 16-row blocks of a wave, at most; more rows are split over row groups, a wave each.  `blocks`: 64-key
// blocks times heads.  Where the caches are few blocks per CU, what counts is how long a wave takes for its own; where they are
// many, that keys are read and widened once.  8 heads, requests of one length, cut into chunks, us with at most 1, 2 and 5
// row blocks:
//   D = 128, 72 rows: 4 x 1,500 keys (750 blocks) 15.8, 17.1, 25.6; 64 x 1,500 (12,300) 91, 70, 66; 16 x 24,576 314, 218, 154
//            40 rows: 24 x 1,400 (4,200) 27.1, 27.6, 35.0;  128 rows: 8 x 9,000 (9,000) 77.5, 62.3, 66.7
//   D = 64:  48 rows: 13 x 1,500 (2,500) 16.8, 19.0, 18.6;  128 rows: 8 x 9,000 60.8, 52.7, 46.5;  72 rows: 16 x 24,576 165, 129, 111
int max_blocks4(int64_t blocks) { return blocks <= 24 * cu_count() ? 1 : blocks <= 40 * cu_count() ? 2 : 5; }
int blocks_of4(int rows, int groups) { return ((rows + 15) / 16 + groups - 1) / groups; }

// Workgroups (one wave, one item each) that run at once: what LDS and registers hold.
int64_t places4(int D, int most) {
  const int per = most > 3 ? 4 : D == 128 ? 8 : most == 1 ? 16 : most == 2 ? 12 : 8;
  return cu_count() * per;
}

// What a wave of one to five row blocks takes for a block of keys by itself, and what each of the waves on a SIMD takes at
// least, in ns, at head dimension 128 and 64: 50 blocks a wave, one wave and two per SIMD.
constexpr int kAlone[2][5] = {{1350, 1630, 2100, 2600, 3100}, {910, 1280, 1370, 1800, 2100}};
constexpr int kShared[2][5] = {{1390, 1530, 1920, 2750, 3200}, {800, 1020, 1270, 1780, 2150}};

// Whether requests are shared among the waves of one workgroup each (for 16 rows of a KV head)
// instead of cut into chunks, which take `chunked` ns: by `groups` of those workgroups, the blocks of the longest
// request, eight at once, and of all.  One launch less, against rows that are read once for each 16 and the longest
// request's time.  In us, joined / in chunks, requests of one length, 8 KV heads; D = 128: 1 x 1,000 keys
// 8.8-9.3 / 10.4, 1 x 4,000 20.9 / 10.5, 4 x 4,000 of 72 rows 21.3 / 24.1, 8 x 4,000 of one token 21.5 / 15.2,
// 32 x 1,000 11.5 / 14.4; D = 64: 13 x 1,500 of 48 rows 13.0 / 16.8, 24 x 1,400 of 40 rows 17.5 / 21.3, 16 x 24,576 of
// 72 rows 175 / 111.  Not of many more workgroups than run at once: 64 x 1,000 keys of one token, D = 128, 21.1 / 19.9.
bool joins(int64_t groups, int64_t longest, int64_t total, int D, int64_t chunked) {
  if (longest > kJoinWaves * kMaxTiles4 || groups > (D == 128 ? cu_count() : cu_count() * 5 / 2)) return false;
  const int64_t all = total * kShared[D == 64][0] / (4 * cu_count());
  const int64_t mine = std::max(longest * (D == 128 ? 200 : 190) + all / 3, all);
  return mine < chunked + 1000;
}

// Joins many partials: the chunks of each (request, position, head) are dealt to the slices of a workgroup,
// whose sums join in slice order.  A thread holds four columns.  One request of 30,000 keys, one token, 8 KV heads,
// D = 128: 5.5 us of 17.8 with 32 query heads, in 118 chunks, and 8.3 of 20.3 with 8, in 235.
template <int D>
__global__ __launch_bounds__(256)
void kv4_merge_many_kernel(AttnShape s, AttnBatch bt, AttnPartials parts, uint16_t* __restrict__ out) {
  constexpr int TPR = D / 4, S = 256 / TPR;
  __shared__ float ms[S], ls[S];
  __shared__ __align__(16) f32x4 os[S][TPR];
  const int row = blockIdx.x, head = blockIdx.y, b = blockIdx.z;
  const int slice = threadIdx.x / TPR, d = threadIdx.x % TPR;
  const int c0 = bt.chunk_base + bt.chunk_prefix[b], c1 = bt.chunk_base + bt.chunk_prefix[b + 1];
  float m = kNoKey4, den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  for (int c = c0 + slice; c < c1; c += 4 * S) {
    float mc[4], lc[4];
    f32x4 oc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t at = ((int64_t)min(c + k * S, c1 - 1) * s.Hkv + head) * s.rows + row;
      mc[k] = parts.m[at];
      lc[k] = parts.l[at];
      oc[k] = *reinterpret_cast<const f32x4*>(parts.o + at * D + 4 * d);
    }
    float mn = m;
#pragma unroll
    for (int k = 0; k < 4; ++k) mn = fmaxf(mn, mc[k]);
    const float alpha = __builtin_amdgcn_exp2f((m - mn) * s.scale_log2);
    den *= alpha;
    num *= alpha;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c + k * S < c1) {
        const float a = __builtin_amdgcn_exp2f((mc[k] - mn) * s.scale_log2);
        den = fmaf(a, lc[k], den);
        num += a * oc[k];
      }
    m = mn;
  }
  if (d == 0) {
    ms[slice] = m;
    ls[slice] = den;
  }
  os[slice][d] = num;
  __syncthreads();
  if (slice != 0) return;
  float mn = ms[0];
#pragma unroll
  for (int k = 1; k < S; ++k) mn = fmaxf(mn, ms[k]);
  den = 0.f;
  num = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const float a = __builtin_amdgcn_exp2f((ms[k] - mn) * s.scale_log2);
    den = fmaf(a, ls[k], den);
    num += a * os[k][d];
  }
  store_four(out, s, bt.req0 + b, head, row, 4 * d, num, den);
}

}  // namespace

AttnShape kv4_shape(int G, int Hq, int Hkv, int D, float scale, const int32_t* kv_len, int B) {
  AttnShape s;
  s.G = G;
  s.Hq = Hq;
  s.Hkv = Hkv;
  s.D = D;
  s.group = Hq / Hkv;
  s.rows = G * s.group;
  int64_t blocks = 0;
  for (int i = 0; i < B; ++i) blocks += (kv_len[i] + kKeyBlock4 - 1) / kKeyBlock4;
  const int b = (s.rows + 15) / 16, upto = max_blocks4(blocks * Hkv);
  s.row_groups = (b + upto - 1) / upto;
  s.scale_log2 = scale * kLog2e;
  int longest = 0;
  for (int i = 0; i < B; ++i) longest = std::max(longest, kv_len[i]);
  longest = (longest + kKeyBlock4 - 1) / kKeyBlock4;
  // For a half to four rounds of items over the CUs' places the shortest chunk that
  // fits them; of these the one that is done first, in ns.  A wave takes kAlone a block by itself and no less than
  // kShared for each of those on its SIMD (where the caches' stream or the SIMD's own instructions bound it).  Items in
  // more rounds are handed out as places come free, and the last ones end half a chunk apart.  Each item
  // costs its start, and its partial is written and read at 5 TB/s.
  // More items than four rounds only with the longest chunk: the workspace holds no more partials.
  const int most_rb = blocks_of4(s.rows, s.row_groups);
  const int64_t slots = places4(D, most_rb), simds = cu_count() * 4;
  const int64_t alone = kAlone[D == 64][most_rb - 1], shared = kShared[D == 64][most_rb - 1];
  const int64_t start = 1500;
  auto items = [&](int tiles) {
    const int keys = tiles * kKeyBlock4;
    int64_t n = 0;
    for (int i = 0; i < B; ++i) n += (kv_len[i] + keys - 1) / keys;
    return n * Hkv * s.row_groups;
  };
  const int64_t total = blocks * Hkv * s.row_groups;
  int64_t best = INT64_MAX / 2;
  int most = kMaxTiles4;
  s.chunk_keys = kMaxTiles4 * kKeyBlock4;
  for (int r : {1, 2, 4, 6, 8}) {  // half rounds
    const int64_t fit = r * slots / 2;
    if (items(most) > fit) continue;
    int lo = 1, hi = most;  // the shortest chunk lies in [lo, hi]
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (items(mid) <= fit) hi = mid; else lo = mid + 1;
    }
    const int64_t n = items(lo);
    const int64_t fold = n <= slots ? std::max(lo * alone, lo * shared * n / simds)
                                    : total * shared / simds + lo * std::max(alone, shared * slots / simds) / 2;
    const int64_t cost = fold + (n + slots - 1) / slots * start + n * (s.rows / s.row_groups) * (D + 2) * 8 / 5000;
    if (cost < best) {
      best = cost;
      s.chunk_keys = lo * kKeyBlock4;
    }
    most = lo;
    if (lo == 1) break;
  }
  if (joins(int64_t(B) * Hkv * b, longest, blocks * Hkv * b, D, best)) {
    s.row_groups = b;
    s.chunk_keys = 0;
  }
  return s;
}

int64_t kv4_max_chunks(int Hkv, int D, int B, int64_t max_kv_len) {
  const int64_t most = std::min(4 * places4(D, 1) / Hkv, B * ((max_kv_len + kKeyBlock4 - 1) / kKeyBlock4));
  const int64_t at_longest = B * ((max_kv_len + kMaxTiles4 * kKeyBlock4 - 1) / (kMaxTiles4 * kKeyBlock4));
  return std::max(most, at_longest);
}

hipError_t launch_kv4_attention(const AttnShape& s, const AttnBatch& batch, const Kv4Pool& pool, int nchunks,
                                const void* q, AttnPartials parts, void* out, hipStream_t stream) {
  if (s.chunk_keys == 0) {
    const dim3 grid((batch.nreq * s.Hkv + 7) / 8 * 8 * s.row_groups);
    ByLength order;
    for (int i = 0; i < kMaxReqPerLaunch; ++i) order.req[i] = static_cast<uint8_t>(i);
    std::sort(order.req, order.req + batch.nreq, [&](int a, int b) {
      return batch.kv_len[a] != batch.kv_len[b] ? batch.kv_len[a] > batch.kv_len[b] : a < b;
    });
#define SDV_JOIN(DIM)                                                                                             \
  hipLaunchKernelGGL((kv4_attn_join_kernel<kJoinWaves, DIM>), grid, dim3(kJoinWaves * kWave), 0, stream, s, batch, \
                     pool, order, static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out))
    if (s.D == 128) SDV_JOIN(128); else SDV_JOIN(64);
#undef SDV_JOIN
    return hipGetLastError();
  }
  const dim3 grid((nchunks * s.Hkv + 7) / 8 * 8 * s.row_groups), block(kWave);
  const int blocks = (s.rows + 15) / 16, most = blocks_of4(s.rows, s.row_groups);
  const int full = blocks - (most - 1) * s.row_groups;  // row groups of `most` blocks
#define SDV_KV4(RB, UNEVEN)                                                                                       \
  do {                                                                                                            \
    if (s.D == 128)                                                                                               \
      hipLaunchKernelGGL((kv4_attn_kernel<RB, UNEVEN, 128>), grid, block, 0, stream, s, batch, pool, nchunks, full, \
                         static_cast<const uint16_t*>(q), parts);                                                 \
    else                                                                                                          \
      hipLaunchKernelGGL((kv4_attn_kernel<RB, UNEVEN, 64>), grid, block, 0, stream, s, batch, pool, nchunks, full, \
                         static_cast<const uint16_t*>(q), parts);                                                 \
  } while (0)
  if (most == 1) SDV_KV4(1, false);
  else if (most == 2 && full == s.row_groups) SDV_KV4(2, false);
  else if (most == 2) SDV_KV4(2, true);
  else if (most == 3) SDV_KV4(3, false);
  else if (most == 4 && full == s.row_groups) SDV_KV4(4, false);
  else if (most == 4) SDV_KV4(4, true);
  else SDV_KV4(5, false);
#undef SDV_KV4
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  int chunks = 0;  // of a request
  for (int b = 0; b < batch.nreq; ++b) chunks = std::max(chunks, batch.chunk_prefix[b + 1] - batch.chunk_prefix[b]);
  if (chunks <= kManyChunks) return launch_kv_merge(s, batch, parts, out, stream);
  const dim3 mgrid(s.rows, s.Hkv, batch.nreq);
  if (s.D == 128)
    hipLaunchKernelGGL(kv4_merge_many_kernel<128>, mgrid, dim3(256), 0, stream, s, batch, parts, static_cast<uint16_t*>(out));
  else
    hipLaunchKernelGGL(kv4_merge_many_kernel<64>, mgrid, dim3(256), 0, stream, s, batch, parts, static_cast<uint16_t*>(out));
  return hipGetLastError();
}

}  // namespace sdv
