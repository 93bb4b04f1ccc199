// Norms of queries and keys for each head and the position rotation (gfx950).
//
//   y = x * weight / sqrt(mean(x^2) + eps);  of each pair (a, b), t = position * inv_freq:
//   (a cos t - b sin t, a sin t + b cos t).
//
// A workgroup takes a row (or a share of its heads): the row's angles are computed once,
// by as many threads as it has, and kept in LDS; a thread holds eight columns of a head.
// Angles are reduced in float64, in revolutions: a float32 product of a far position
// would be off by whole radians.
//
// Bound by memory: 9,001 bf16 rows of 64 + 8 heads, D = 128 (332 MB), take 65 us, 5.1 TB/s (a large copy reaches
// 4.7-4.9), 4,500 float32 ones 72.5 us, 4.6 TB/s; 320 rows of 32 + 32 heads 4.1-4.9 us, a launch's latency, a trip to memory
// and the angles.  Rows of few heads leave threads idle: 9,001 rows of 8 + 1 heads (41 MB) take 17.6 us, 2.4 TB/s.
#include <algorithm>

#include "fp4.h"

namespace sdv {

namespace {

constexpr int kRopeThreads = 256;
// Workgroups up to which a row's heads are shared among several: 320 rows of 64 heads take 4.1 us in 1,280 of them, 5.4
// in 320.
constexpr int kRopeGroups = 2048;

// Sum over the threads of a head.
template <int D>
__device__ __forceinline__ float head_sum(float v) {
  v += dpp_f32<kDppXor1>(v);
  v += dpp_f32<kDppXor2>(v);
  v += dpp_f32<kDppRowHalfMirror>(v);
  return D == 128 ? v + dpp_f32<kDppRowMirror>(v) : v;
}
template <int D>
__device__ __forceinline__ double head_sum(double v) {
  v += dpp_f64<kDppXor1>(v);
  v += dpp_f64<kDppXor2>(v);
  v += dpp_f64<kDppRowHalfMirror>(v);
  return D == 128 ? v + dpp_f64<kDppRowMirror>(v) : v;
}

// x * weight / rms.  Sums of squares near the ends of float32's range are taken again in
// float64 (a wave at a time: rows of ordinary numbers never come here).
template <int D>
__device__ __forceinline__ void normed(float (&x)[8], const float (&w)[8], float eps) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
  sum = head_sum<D>(sum);
  const bool plain = sum > 1e-25f && sum < 1e30f;
  if (__builtin_expect(__ballot(!plain) == 0, 1)) {
    const float r = 1.f / sqrtf(sum * (1.f / D) + eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
    return;
  }
  double wide = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) wide += (double)x[i] * (double)x[i];
  const double r = 1.0 / sqrt(head_sum<D>(wide) / D + (double)eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)((double)x[i] * r * (double)w[i]);
}

// Eight of a weight's columns, which every head reads again.
__device__ __forceinline__ void load_weight(const uint16_t* p, float (&w)[8]) {
  const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[2 * i] = __uint_as_float(r[i] << 16);
    w[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load_weight(const float* p, float (&w)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = a[i];
    w[4 + i] = b[i];
  }
}

template <typename T, int D, bool INTERLEAVED, bool NORM>
__global__ __launch_bounds__(kRopeThreads)
void qk_rope_kernel(RopeArgs a, const T* q, const T* k, const int32_t* __restrict__ positions,
                    const float* __restrict__ inv_freq, const T* __restrict__ q_weight,
                    const T* __restrict__ k_weight, T* q_out, T* k_out) {
  constexpr int TPR = D / 8;
  __shared__ __align__(16) float2 turn[D / 2];  // cos and sin of each pair's angle
  const int row = blockIdx.x, t = threadIdx.x;
  const int half = a.rotary / 2, heads = a.Hq + a.Hkv;
  if (t < half) {
    const double rev = (double)positions[row] * (double)inv_freq[t] * 0.15915494309189535;
    float s, c;
    sincospif(2.f * (float)(rev - rint(rev)), &s, &c);
    turn[t] = make_float2(c, s);
  }
  __syncthreads();
  const int col = t % TPR * 8;
  const bool turned = col < a.rotary, low = INTERLEAVED || col < half;
  // Half-split pairs: the other column of this thread's lies in this thread.
  const int other = (t & ~(TPR - 1)) + (turned ? (low ? col + half : col - half) / 8 : col / 8);
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int pair = INTERLEAVED ? (col + i) / 2 : (low ? col : col - half) + i;
    const float2 cs = turn[turned ? pair : 0];
    c[i] = turned ? cs.x : 1.f;
    s[i] = !turned ? 0.f : (INTERLEAVED ? i % 2 == 0 : low) ? -cs.y : cs.y;
  }
  const int per = kRopeThreads / TPR;
  for (int h0 = blockIdx.y * per; h0 < heads; h0 += per * gridDim.y) {
    const int h = h0 + t / TPR;
    const bool mine = h < heads, is_k = h >= a.Hq;
    const int hc = mine ? (is_k ? h - a.Hq : h) : 0;  // any head of the row's is read in its place
    const T* src = (mine && is_k ? k + row * a.k_stride : q + row * a.q_stride) + hc * D + col;
    float x[8];
    load_row8(src, x);
    float y[8];
    if (NORM) {
      const T* weight = mine && is_k ? k_weight : q_weight;
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.f;
      if (weight != nullptr) load_weight(weight + col, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i];
      normed<D>(y, w, a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = weight != nullptr ? y[i] : x[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = INTERLEAVED ? x[i ^ 1] : __shfl(x[i], other & 63);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = turned ? fmaf(x[i], c[i], y[i] * s[i]) : x[i];
    if (mine) store_row8((is_k ? k_out + row * a.k_out_stride : q_out + row * a.q_out_stride) + hc * D + col, x);
  }
}

}  // namespace

hipError_t launch_qk_rope(const RopeArgs& a, int D, bool f32, bool interleaved, const void* q, const void* k,
                          const int32_t* positions, const float* inv_freq, const void* q_weight, const void* k_weight,
                          void* q_out, void* k_out, hipStream_t stream) {
  const int64_t passes = (a.Hq + a.Hkv + kRopeThreads * 8 / D - 1) / (kRopeThreads * 8 / D);
  const int64_t shares = std::max<int64_t>(1, std::min({passes, int64_t(kRopeGroups) / a.rows, int64_t(65535)}));
  const dim3 grid(a.rows, static_cast<unsigned>(shares)), block(kRopeThreads);
  const bool norm = q_weight != nullptr || k_weight != nullptr;
#define SDV_ROPE(T, DIM, INTER, NORM)                                                                             \
  hipLaunchKernelGGL((qk_rope_kernel<T, DIM, INTER, NORM>), grid, block, 0, stream, a, static_cast<const T*>(q),         \
                     static_cast<const T*>(k), positions, inv_freq, static_cast<const T*>(q_weight),               \
                     static_cast<const T*>(k_weight), static_cast<T*>(q_out), static_cast<T*>(k_out))
#define SDV_ROPE_DIM(T, DIM)        \
  if (interleaved && norm) {        \
    SDV_ROPE(T, DIM, true, true);   \
  } else if (interleaved) {         \
    SDV_ROPE(T, DIM, true, false);  \
  } else if (norm) {                \
    SDV_ROPE(T, DIM, false, true);  \
  } else {                          \
    SDV_ROPE(T, DIM, false, false); \
  }
  if (f32 && D == 128) {
    SDV_ROPE_DIM(float, 128)
  } else if (f32) {
    SDV_ROPE_DIM(float, 64)
  } else if (D == 128) {
    SDV_ROPE_DIM(uint16_t, 128)
  } else {
    SDV_ROPE_DIM(uint16_t, 64)
  }
#undef SDV_ROPE_DIM
#undef SDV_ROPE
  return hipGetLastError();
}

}  // namespace sdv
