// Vocabulary projection of 8-bit rows with 8-bit weights (gfx950).
//
//   logits[m][v] = sum_c sa[c][m] * sw[v/128][c] * sum_{k in block c} a[m][k] * w[v][k],
//
// and per row and tile of vocabulary entries the maximum and the sum of
// exponentials, folded into the rows' log-sum-exp by the bf16 projection's kernel.
//
// Bound by the stream of W up to about 200 rows, by the matrix cores past that.
// A row's 128 columns of one scale are one 128-byte line, so W [V][K] and the
// rows [M][K] are streamed as they are, in whole lines by LDS DMA, a line of
// every row of the tile per stage.  Codes widen to bfloat16 exactly on their way
// from LDS into MFMA 32x32x16: the 8-bit matrix instructions would need no
// widening and run twice as fast, but they keep too few bits of their sums
// (measured: 1.4e-5 of a 128-product sum, where bfloat16's products are exact).
// A line's products are summed from zero and then added to the accumulators
// times both scales.
//
// Of a 32-row group (four 1 KB blocks of eight rows), unit u (16 bytes) of row r
// sits at slot 8 r + (u + r / 2) mod 8, so that the 32 rows that a fragment read
// takes of one unit fall on distinct banks.  The line's eight units are read in
// pairs: lanes 0-31 take unit 2 j, lanes 32-63 unit 2 j + 1, which are the 32
// columns of two MFMA steps; both operands permute the columns alike.
#include <algorithm>
#include <atomic>

#include "fp8.h"
#include "vocab_tile.h"

namespace sdv {

namespace {

constexpr int kWaves = 4;
constexpr int kScaleBytes = 1024;  // a stage's row scales: 256 floats

constexpr int stage_bytes(int mb, int nb) { return (4 * mb + 4 * kWaves * nb) * 1024 + kScaleBytes; }
constexpr int stages(int mb, int nb) {
  const int n = 160 * 1024 / stage_bytes(mb, nb);
  return n < 6 ? n : 6;
}

// LDS DMA of four bytes per lane (as line_dma: lane l to lds + 4 l).
__device__ __forceinline__ void word_dma(const float* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(g) : "m0", "memory");
}

template <int MB, int NB>
__global__ __launch_bounds__(kWaves * kWave, 1)
void vocab_fp8_kernel(int M, int K, int V, int ntiles, int mtiles, const uint8_t* __restrict__ hidden,
                      const float* __restrict__ hidden_scale, const uint8_t* __restrict__ w,
                      const float* __restrict__ w_scale, float* __restrict__ logits, float2* __restrict__ partials) {
  constexpr int NW = kWaves;
  constexpr int kHBlocks = 4 * MB;
  constexpr int kStage = stage_bytes(MB, NB);
  constexpr int kScaleAt = kStage - kScaleBytes;
  constexpr int S = stages(MB, NB);
  constexpr int kOps = MB + 4 * NB + 1;  // DMAs per wave and line
  static_assert(S >= 2 && (S - 1) * kOps < 64, "two stages; vmcnt holds 6 bits");
  __shared__ __align__(1024) unsigned char lds[S * kStage];

  // The M-tiles of one vocabulary tile share an XCD (ids 8 apart).
  const int grp = 8 * mtiles;
  const int tile = (blockIdx.x / grp) * 8 + (blockIdx.x & 7);
  if (tile >= ntiles) return;
  const int m0 = ((blockIdx.x % grp) >> 3) * MB * 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int blk0 = (tile * NW + wave) * NB;
  const int nlines = (K + kColBlock - 1) / kColBlock;
  const int last_units = (K - (nlines - 1) * kColBlock) / 16;  // 2, 4, 6 or 8

  // Lane l of block q of a group brings unit (l % 8) - r / 2 of row r = 8 q + l
  // / 8.  Rows past V and past M repeat the last row; units past the last line's
  // end repeat earlier ones and are not read.
  auto unit = [&](int q) { return ((lane & 7) - 4 * (q & 1) - (lane >> 4)) & 7; };
  const char* wsrc[NB][4];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = min((blk0 + nb) * 32 + 8 * q + (lane >> 3), V - 1);
      wsrc[nb][q] = reinterpret_cast<const char*>(w + (int64_t)row * K) + unit(q) * 16;
    }
  const char* hsrc[MB];  // block `wave` of every 32-row group
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    const int row = min(m0 + mb * 32 + 8 * wave + (lane >> 3), M - 1);
    hsrc[mb] = reinterpret_cast<const char*>(hidden + (int64_t)row * K) + unit(wave) * 16;
  }
  const float* ssrc = hidden_scale + min(m0 + (int)threadIdx.x, M - 1);
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  // DMA j of line c into stage s.
  auto issue_op = [&](int j, int s, int c) {
    const uint32_t dst = lds_base + (uint32_t)s * kStage;
    const bool part = last_units < 8 && c == nlines - 1;
    const int64_t o = (int64_t)c * kLineBytes;
    if (j < MB) {
      const int u = unit(wave);
      line_dma<false>(hsrc[j] + o + (part && u >= last_units ? (u % last_units - u) * 16 : 0), dst + (4 * j + wave) * 1024);
    } else if (j < MB + 4 * NB) {
      const int nb = (j - MB) >> 2, q = (j - MB) & 3;
      const int u = unit(q);
      line_dma<true>(wsrc[nb][q] + o + (part && u >= last_units ? (u % last_units - u) * 16 : 0),
                     dst + (kHBlocks + (wave * NB + nb) * 4 + q) * 1024);
    } else {
      word_dma(ssrc + (int64_t)c * M, dst + kScaleAt + wave * 256);
    }
  };
  // Units 2 j and 2 j + 1 of the rows of W block nb, of hidden block mb.
  const int r = lane & 31;
  auto slot = [&](int s, int j) {
    return lds + s * kStage + (r >> 3) * 1024 + (r & 7) * 128 + ((2 * j + (lane >> 5) + (r >> 1)) & 7) * 16;
  };
  auto read_w = [&](int s, int nb, int j) {
    return *reinterpret_cast<const u32x4*>(slot(s, j) + (kHBlocks + (wave * NB + nb) * 4) * 1024);
  };
  auto read_h = [&](int s, int mb, int j) { return *reinterpret_cast<const u32x4*>(slot(s, j) + 4 * mb * 1024); };

  f32x16 acc[MB][NB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[mb][nb][e] = 0.f;

  // A wave's entries lie in one block of 128: lane j holds its scale of line c0 + j.
  const float* wsc = w_scale + (int64_t)min(blk0 * 32 / kColBlock, (V - 1) / kColBlock) * nlines;
  float sw_all = 0.f;

#pragma unroll
  for (int c = 0; c < S - 1; ++c)
    if (c < nlines) {
#pragma unroll
      for (int j = 0; j < kOps; ++j) issue_op(j, c, c);
    }
  int s = 0;
  for (int c = 0; c < nlines; ++c) {
    if ((c & 63) == 0) sw_all = wsc[min(c + lane, nlines - 1)];
    // Line c is in once only the lines after it are in flight; past the barrier
    // every wave's part is, and line c - 1 has been read by all.
    if (c + S - 1 <= nlines)
      wait_vmcnt<(S - 2) * kOps>();
    else
      wait_vmcnt<0>();
    lds_barrier();
    if (c + S - 1 < nlines) {
      const int sp = s == 0 ? S - 1 : s - 1;
#pragma unroll
      for (int j = 0; j < kOps; ++j) issue_op(j, sp, c + S - 1);
    }
    const float sw = lane_f32(sw_all, c & 63);
    const float* sa = reinterpret_cast<const float*>(lds + s * kStage + kScaleAt);
    if (last_units == 8 || c + 1 < nlines) {
      bf16x8 wf[NB][8];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 x = read_w(s, nb, j);
          wf[nb][2 * j] = widen8(x[0], x[1], 1.f);
          wf[nb][2 * j + 1] = widen8(x[2], x[3], 1.f);
        }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        f32x16 sum[NB];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 x = read_h(s, mb, j);
          const bf16x8 h0 = widen8(x[0], x[1], 1.f), h1 = widen8(x[2], x[3], 1.f);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            if (j == 0) {
#pragma unroll
              for (int e = 0; e < 16; ++e) sum[nb][e] = 0.f;
            }
            sum[nb] = mfma32x32x16(wf[nb][2 * j], h0, sum[nb]);
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) sum[nb] = mfma32x32x16(wf[nb][2 * j + 1], h1, sum[nb]);
        }
        const float f = sa[mb * 32 + r] * sw;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[mb][nb][e] = fmaf(sum[nb][e], f, acc[mb][nb][e]);
      }
    } else {
      for (int j = 0; j < last_units / 2; ++j) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const u32x4 y = read_w(s, nb, j);
          const bf16x8 w0 = widen8(y[0], y[1], 1.f), w1 = widen8(y[2], y[3], 1.f);
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            const u32x4 x = read_h(s, mb, j);
            f32x16 sum;
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[e] = 0.f;
            sum = mfma32x32x16(w0, widen8(x[0], x[1], 1.f), sum);
            sum = mfma32x32x16(w1, widen8(x[2], x[3], 1.f), sum);
            const float f = sa[mb * 32 + r] * sw;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[mb][nb][e] = fmaf(sum[e], f, acc[mb][nb][e]);
          }
        }
      }
    }
    s = s + 1 == S ? 0 : s + 1;
  }
  lds_barrier();
  tile_epilogue32<MB, NB, NW>(acc, M, V, ntiles, tile, m0, blk0, logits, partials,
                              reinterpret_cast<float(*)[MB * 32]>(lds));
}

template <int MB, int NB>
hipError_t launch(const Fp8Plan& p, const void* hidden, const float* hidden_scale, const void* w, const float* w_scale,
                  float* logits, float2* partials, hipStream_t stream) {
  hipLaunchKernelGGL((vocab_fp8_kernel<MB, NB>), dim3((p.ntiles + 7) / 8 * 8 * p.mtiles), dim3(kWaves * kWave), 0,
                     stream, p.M, p.K, p.V, p.ntiles, p.mtiles, static_cast<const uint8_t*>(hidden), hidden_scale,
                     static_cast<const uint8_t*>(w), w_scale, logits, partials);
  return hipGetLastError();
}

}  // namespace

Fp8Plan fp8_plan(int M, int K, int V) {
  Fp8Plan p{M, K, V, 0, 0, 0, 0};
  const int blocks = (M + 31) / 32;
  p.mtiles = (blocks + 6) / 7;
  p.mb = (blocks + p.mtiles - 1) / p.mtiles;
  p.nb = V > 32 * 1024 ? 2 : 1;
  const int width = 32 * kWaves * p.nb;
  p.ntiles = (V + width - 1) / width;
  return p;
}

size_t fp8_logits_bytes(const Fp8Plan& p) { return (size_t)p.M * p.ntiles * sizeof(float2); }

hipError_t launch_logits_fp8(const Fp8Plan& p, const void* hidden, const float* hidden_scale, const void* w,
                             const float* w_scale, float* logits, float* row_lse, void* ws, hipStream_t stream) {
  float2* partials = static_cast<float2*>(ws);
  hipError_t e = hipErrorInvalidValue;
#define SDV_F(B)                                                                                             \
  case B:                                                                                                    \
    e = p.nb == 2 ? launch<B, 2>(p, hidden, hidden_scale, w, w_scale, logits, partials, stream)              \
                  : launch<B, 1>(p, hidden, hidden_scale, w, w_scale, logits, partials, stream);             \
    break;
  switch (p.mb) {
    SDV_F(1) SDV_F(2) SDV_F(3) SDV_F(4) SDV_F(5) SDV_F(6) SDV_F(7)
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
