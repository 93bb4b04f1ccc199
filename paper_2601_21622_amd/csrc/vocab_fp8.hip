// Vocabulary projection of 8-bit rows with 8-bit weights (gfx950).
//
//   logits[m][v] = sum_c sa[c][m] * sw[v/128][c] * sum_{k in block c} a[m][k] * w[v][k],
//
// and per row and tile of vocabulary entries the maximum and the sum of
// exponentials, folded into the rows' log-sum-exp by the bf16 projection's kernel.
//
// Bound by the stream of W up to about 64 rows (1.05 GB for 64 x 128,256 x 8,192 in 192
// us, 5.5 TB/s), by the matrix cores' power past that: 224 x 128,256 x 4,096 takes 245 us,
// 0.96 PFLOP/s, where a large bfloat16 product of the library reaches 1.14 to 1.2 on the same
// card, and the same launch over codes that are all zero, with nothing else changed, takes 184.
// A row's 128 columns of one scale are one 128-byte line, so W [V][K] and the
// rows [M][K] are streamed as they are, in whole lines by LDS DMA, a line of
// every row of the tile per stage.  Codes widen to bfloat16 exactly on their way
// from LDS into MFMA 32x32x16: the 8-bit matrix instructions would need no
// widening and run twice as fast, but they keep too few bits of their sums
// (measured: 1.4e-5 of a 128-product sum, where bfloat16's products are exact).
// A line's products are summed from zero and then added to the accumulators
// times both scales.
//
// A workgroup is eight waves of 32 entries each: a tile of 256, every row line read by
// all of them.  Where tiles of 128 are one round of the CUs at most, two parts of four
// waves sum over one half of the columns each, over the same 128 entries, and the second
// part's sums are added to the first's: twice as many CUs work, each line by line as
// before.  96 x 32,000 x 4,096: 43.5 us so, 54 with tiles of 256; 160 x 50,304 x 4,096,
// where tiles of 128 are two rounds: 117 and 79.
//
// Of a 32-row group (four 1 KB blocks of eight rows), unit u (16 bytes) of row r
// sits at slot 8 r + (u + r / 2) mod 8, so that the 32 rows that a fragment read
// takes of one unit fall on distinct banks.  The line's eight units are read in
// pairs: lanes 0-31 take unit 2 j, lanes 32-63 unit 2 j + 1, which are the 32
// columns of two MFMA steps; both operands permute the columns alike.
#include "fp8.h"
#include "vocab_tile.h"

namespace sdv {

namespace {

constexpr int kScaleBytes = 1024;  // a stage's row scales: 256 floats

constexpr int kWaves = 8;
constexpr int kCUs = 256;  // of the MI355X

constexpr int line_bytes(int mb, int nw) { return 4 * (mb + nw) * 1024 + kScaleBytes; }
constexpr int stages(int mb, int nw) {
  const int n = 160 * 1024 / (kWaves / nw * line_bytes(mb, nw));
  return n < 4 ? n : 4;  // more bring nothing
}

// LDS DMA of 16 (or 4) bytes per lane from base + off into LDS bytes lds + 16 l
// (4 l), both bases wave-uniform.  The scalar copy of the base is the wait state
// between the write of M0 and the load, and the load's base is never a register that a
// vector instruction wrote just before, which would take five.
template <bool NT>
__device__ __forceinline__ void base_dma(const void* base, uint32_t off, uint32_t lds) {
  uint64_t from;
  if (NT)
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0 nt"
                 : "=&s"(from) : "s"(lds), "v"(off), "s"(base) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0"
                 : "=&s"(from) : "s"(lds), "v"(off), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void base_dma_word(const void* base, uint32_t off, uint32_t lds) {
  uint64_t from;
  asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0"
               : "=&s"(from) : "s"(lds), "v"(off), "s"(base) : "m0", "memory");
}

template <int X>
struct Int {
  static constexpr int value = X;
};

template <int MB, int NW>
__global__ __launch_bounds__(kWaves * kWave, 1)
void vocab_fp8_kernel(int M, int K, int V, int ntiles, int mtiles, const uint8_t* __restrict__ hidden,
                      const float* __restrict__ hidden_scale, const uint8_t* __restrict__ w,
                      const float* __restrict__ w_scale, float* __restrict__ logits, float2* __restrict__ partials) {
  constexpr int kHBlocks = 4 * MB;
  constexpr int kParts = kWaves / NW;
  constexpr int kLine = line_bytes(MB, NW);
  constexpr int kStage = kParts * kLine;
  constexpr int kScaleAt = kLine - kScaleBytes;
  constexpr int S = stages(MB, NW);
  constexpr int kHOps = (kHBlocks + NW - 1) / NW;  // hidden blocks per wave (past the last: the last again)
  constexpr int kOps = 4 + kHOps + 1;              // DMAs per wave and line
  constexpr int kSteps = 4 * MB;
  constexpr int kRowOps = kHOps + 1;
  static_assert(S >= 2 && (S - 1) * kOps < 64, "two stages; vmcnt holds 6 bits");
  static_assert(kParts == 1 || (kParts == 2 && MB * 16 * 1024 <= S * kStage), "the second part's sums");
  __shared__ __align__(1024) unsigned char lds_all[S * kStage];

  // The M-tiles of one vocabulary tile share an XCD (ids 8 apart).
  const int grp = 8 * mtiles;
  const int tile = (blockIdx.x / grp) * 8 + (blockIdx.x & 7);
  if (tile >= ntiles) return;
  const int m0 = ((blockIdx.x % grp) >> 3) * MB * 32;
  const int part = kParts == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (NW * kWave));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - part * NW;
  unsigned char* const lds = lds_all + part * kLine;
  const int lane = threadIdx.x & 63;
  const int blk0 = tile * NW + wave;
  // Each part of the waves sums over lines of its own, first .. first + nlines - 1; only
  // the last part has columns past the last whole line.
  const int all_lines = K / kColBlock;
  const int first = part * (all_lines / kParts);
  const int nlines = (part == kParts - 1 ? all_lines : all_lines / kParts) - first;
  const int nscales = (K + kColBlock - 1) / kColBlock;

  // Lane l of block q of a group brings unit (l % 8) - r / 2 of row r = 8 q + l
  // / 8.  Rows past V and past M repeat the last row.  Offsets count from the
  // tile's first rows, and its 256 rows of K < 2^23 bytes fit 32 bits.
  auto unit = [&](int q) { return ((lane & 7) - 4 * (q & 1) - (lane >> 4)) & 7; };
  const uint8_t* wbase = w + (int64_t)tile * NW * 32 * K;
  const uint8_t* hbase = hidden + (int64_t)m0 * K;
  uint32_t woff[4], hoff[kHOps];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    woff[q] = (uint32_t)min(wave * 32 + 8 * q + (lane >> 3), V - 1 - tile * NW * 32) * (uint32_t)K + unit(q) * 16;
  int hblk[kHOps];
#pragma unroll
  for (int i = 0; i < kHOps; ++i) {
    hblk[i] = min(wave + i * NW, kHBlocks - 1);
    hoff[i] = (uint32_t)min(8 * hblk[i] + (lane >> 3), M - 1 - m0) * (uint32_t)K + unit(hblk[i]) * 16;
  }
  const uint32_t soff = (uint32_t)min((int)(threadIdx.x & 255), M - 1 - m0) * 4u;  // each 4 waves bring all
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  // DMA j of line c into stage s, of its first `units` units (the others repeat the
  // first): the rows' and their scales, then the wave's own entries'.
  auto issue_op = [&](int j, int s, int c, int units = 8) {
    const uint32_t dst = lds_base + (uint32_t)s * kStage;
    const int64_t o = (int64_t)c * kLineBytes;
    const int q = j - kRowOps;
    uint32_t back = 0;
    if (units < 8 && j != kHOps) {
      const int u = unit(q >= 0 ? q : hblk[j < kHOps ? j : 0]);
      back = u >= units ? (uint32_t)u * 16 : 0;
    }
    if (q >= 0)
      base_dma<true>(wbase + o, woff[q < 0 ? 0 : q] - back, dst + (kHBlocks + wave * 4 + q) * 1024);
    else if (j < kHOps)
      base_dma<false>(hbase + o, hoff[j] - back, dst + hblk[j] * 1024);
    else
      base_dma_word(hidden_scale + (int64_t)c * M + m0, soff, dst + kScaleAt + (wave & 3) * 256);
  };
  // Units 2 j and 2 j + 1 of the wave's W rows, of the rows of hidden group mb.
  const int r = lane & 31;
  auto at = [&](int s, int j) {
    return lds + s * kStage + (r >> 3) * 1024 + (r & 7) * 128 + ((2 * j + (lane >> 5) + (r >> 1)) & 7) * 16;
  };
  auto read = [&](const unsigned char* p, int group) { return *reinterpret_cast<const u32x4*>(p + 4 * group * 1024); };

  f32x16 acc[MB][1];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[mb][0][e] = 0.f;

  // A wave's entries lie in one block of 128: lane j holds its scale of line 64 n + j.
  const float* wsc = w_scale + (int64_t)min(blk0 * 32 / kColBlock, (V - 1) / kColBlock) * nscales;
  float sw_all = 0.f;

  // Tiles start on different lines and wrap: rows a multiple of 4 KB apart would
  // otherwise send every workgroup to the same memory channels at once.
  int l = first + (nlines > 0 ? (int)((unsigned)tile % (unsigned)nlines) : 0);
  auto after = [&](int c) { return c + 1 == first + nlines ? first : c + 1; };
  // Line c asks for the rows of line c + S - 1, whose stage all waves have left, and
  // for the wave's own entries of line c + S, whose place is free as soon as the wave
  // has read line c's.  In this order they are on their way before line 0 too.
  int next_h = l, next_w = l;
#pragma unroll
  for (int c = 0; c < S; ++c) {
    if (c < nlines) {
#pragma unroll
      for (int j = kRowOps; j < kOps; ++j) issue_op(j, c, next_w);
      next_w = after(next_w);
    }
    if (c < S - 1 && c < nlines) {
#pragma unroll
      for (int j = 0; j < kRowOps; ++j) issue_op(j, c, next_h);
      next_h = after(next_h);
    }
  }
  int s = 0, left = nlines;
  // One line: the products of its 128 columns, from zero, times both scales.
  // FILL: it asks for rows and entries (2), for rows (1) or for nothing (0), bit by bit
  // between the products: a wave that asks for a whole stage at once stands still
  // while the CU's lines in flight (65 on average with 6 rows of 4,096) make room.
  auto line = [&](auto fill) {
    constexpr int kFill = decltype(fill)::value;
    // The line is in once only what was asked for after its rows is in flight.
    if (kFill > 0)
      wait_vmcnt<(S - 2) * kOps + 4>();
    else if (left > 2 && S > 3)
      wait_vmcnt<2 * kOps>();
    else if (left > 1 && S > 2)
      wait_vmcnt<kOps>();
    else
      wait_vmcnt<0>();
    lds_barrier();  // every wave's part is, and the last line has been read by all
    const int sp = s == 0 ? S - 1 : s - 1;
    const float sw = lane_f32(sw_all, l & 63);
    const float* sa = reinterpret_cast<const float*>(lds + s * kStage + kScaleAt) + r;
    constexpr f32x16 kZero = {};
    const unsigned char* p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = at(s, j);
    bf16x8 wf[8];
    u32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = read(p[j], 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4 y = *reinterpret_cast<const u32x4*>(p[j] + (kHBlocks + wave * 4) * 1024);
      wf[2 * j] = widen8(y[0], y[1], 1.f);
      wf[2 * j + 1] = widen8(y[2], y[3], 1.f);
    }
    lds_wait();  // the entries' place is free
    // A group's sum is added, scaled, while the next group is multiplied.
    f32x16 sum[2];
    float f[2];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      f[mb & 1] = sa[mb * 32] * sw;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8 h0 = widen8(x[j][0], x[j][1], 1.f), h1 = widen8(x[j][2], x[j][3], 1.f);
        if (mb + 1 < MB) x[j] = read(p[j], mb + 1);
        sum[mb & 1] = mfma32x32x16(wf[2 * j], h0, j == 0 ? kZero : sum[mb & 1]);
        if (mb > 0) {
#pragma unroll
          for (int e = 4 * j; e < 4 * j + 4; ++e)
            acc[mb - 1][0][e] = fmaf(sum[(mb - 1) & 1][e], f[(mb - 1) & 1], acc[mb - 1][0][e]);
        }
        sum[mb & 1] = mfma32x32x16(wf[2 * j + 1], h1, sum[mb & 1]);
        if (kFill > 0) {
          const int i = 4 * mb + j;
#pragma unroll
          for (int o = i * kOps / kSteps; o < (i + 1) * kOps / kSteps; ++o)
            if (o < kRowOps)
              issue_op(o, sp, next_h);
            else if (kFill > 1)
              issue_op(o, s, next_w);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
      acc[MB - 1][0][e] = fmaf(sum[(MB - 1) & 1][e], f[(MB - 1) & 1], acc[MB - 1][0][e]);
    if (kFill > 0) next_h = after(next_h);
    if (kFill > 1) next_w = after(next_w);
    s = s + 1 == S ? 0 : s + 1;
    l = after(l);
    --left;
  };
  sw_all = wsc[min((l & ~63) + lane, nscales - 1)];
  auto scales = [&]() {
    if ((l & 63) == 0 || l == first) sw_all = wsc[min((l & ~63) + lane, nscales - 1)];
  };
  while (left > S) {
    scales();
    line(Int<2>());
  }
  if (left == S) {
    scales();
    line(Int<1>());
  }
  while (left > 0) {
    scales();
    line(Int<0>());
  }
  if (kParts > 1 && part == 0 && all_lines % kParts != 0) lds_barrier();  // the last part's odd line
  if (nscales > all_lines) {  // the columns past the last whole line: 32, 64 or 96
    const int units = (K - all_lines * kColBlock) / 16;
    lds_barrier();
    if (part == kParts - 1) {
#pragma unroll
      for (int o = 0; o < kOps; ++o) issue_op(o, 0, all_lines, units);
      wait_vmcnt<0>();
    }
    lds_barrier();
    if (part == kParts - 1) {
      const float sw = wsc[all_lines];
      for (int j = 0; j < units / 2; ++j) {
        const unsigned char* p = at(0, j);
        const u32x4 y = *reinterpret_cast<const u32x4*>(p + (kHBlocks + wave * 4) * 1024);
        const bf16x8 w0 = widen8(y[0], y[1], 1.f), w1 = widen8(y[2], y[3], 1.f);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          const u32x4 x = read(p, mb);
          f32x16 sum = {};
          sum = mfma32x32x16(w0, widen8(x[0], x[1], 1.f), sum);
          sum = mfma32x32x16(w1, widen8(x[2], x[3], 1.f), sum);
          const float f = reinterpret_cast<const float*>(lds + kScaleAt)[mb * 32 + r] * sw;
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[mb][0][e] = fmaf(sum[e], f, acc[mb][0][e]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  lds_barrier();
  if (kParts > 1) {
    f32x4* const sums = reinterpret_cast<f32x4*>(lds_all) + wave * (MB * 4 * kWave) + lane;
    if (part == 1) {
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          sums[(mb * 4 + g) * kWave] =
              f32x4{acc[mb][0][4 * g], acc[mb][0][4 * g + 1], acc[mb][0][4 * g + 2], acc[mb][0][4 * g + 3]};
    }
    lds_barrier();
    if (part == 1) return;  // the barriers that follow count the waves that are left
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 o = sums[(mb * 4 + g) * kWave];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mb][0][4 * g + e] += o[e];
      }
    lds_barrier();
  }
  tile_epilogue32<MB, 1, NW>(acc, M, V, ntiles, tile, m0, blk0, logits, partials,
                             reinterpret_cast<float(*)[MB * 32]>(lds_all));
}

template <int MB, int NW>
hipError_t launch(const Fp8Plan& p, const void* hidden, const float* hidden_scale, const void* w, const float* w_scale,
                  float* logits, float2* partials, hipStream_t stream) {
  hipLaunchKernelGGL((vocab_fp8_kernel<MB, NW>), dim3((p.ntiles + 7) / 8 * 8 * p.mtiles), dim3(kWaves * kWave), 0, stream,
                     p.M, p.K, p.V, p.ntiles, p.mtiles, static_cast<const uint8_t*>(hidden), hidden_scale,
                     static_cast<const uint8_t*>(w), w_scale, logits, partials);
  return hipGetLastError();
}

}  // namespace

Fp8Plan fp8_plan(int M, int K, int V) {
  Fp8Plan p{M, K, V, 0, 0, 0, 0};
  const int blocks = (M + 31) / 32;
  const int most = (blocks + 4) / 5;  // tiles of at most 160 rows: two stages of two parts' lines fill LDS
  p.nw = (int64_t)(V + 127) / 128 * most <= kCUs ? 4 : 8;
  p.mtiles = p.nw == 4 ? most : (blocks + 6) / 7;
  p.mb = (blocks + p.mtiles - 1) / p.mtiles;
  const int width = 32 * p.nw;
  p.ntiles = (V + width - 1) / width;
  return p;
}

// Of the narrow tiles, whichever are used: it grows with rows and entries.
size_t fp8_logits_bytes(int M, int V) { return (size_t)M * ((V + 127) / 128) * sizeof(float2); }

hipError_t launch_logits_fp8(const Fp8Plan& p, const void* hidden, const float* hidden_scale, const void* w,
                             const float* w_scale, float* logits, float* row_lse, void* ws, hipStream_t stream) {
  float2* partials = static_cast<float2*>(ws);
  hipError_t e = hipErrorInvalidValue;
#define SDV_F(B, N)                                                                               \
  case 16 * B + N:                                                                                \
    e = launch<B, N>(p, hidden, hidden_scale, w, w_scale, logits, partials, stream);              \
    break;
  switch (16 * p.mb + p.nw) {
    SDV_F(1, 4) SDV_F(2, 4) SDV_F(3, 4) SDV_F(4, 4) SDV_F(5, 4)
    SDV_F(1, 8) SDV_F(2, 8) SDV_F(3, 8) SDV_F(4, 8) SDV_F(5, 8) SDV_F(6, 8) SDV_F(7, 8)
    default: break;
  }
#undef SDV_F
  if (e != hipSuccess) return e;
  VocabPlan vp{};
  vp.M = p.M;
  vp.ntiles = p.ntiles;
  return launch_lse_combine(vp, partials, row_lse, stream);
}

}  // namespace sdv
