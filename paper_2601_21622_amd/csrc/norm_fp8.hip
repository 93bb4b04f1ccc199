// Residual addition, root-mean-square norm and 8-bit output (gfx950).
//
//   h = x + residual,  y = h * weight / sqrt(mean(h^2) + eps),
//   per 128 columns: s = max(max|y| / 448, 2^-126), code = e4m3(y / s).
//
// One workgroup per row: a thread holds R groups of eight columns in registers,
// so that the row is read once; 16 lanes hold the 128 columns of a scale.  Bound
// by memory: bf16 rows read 4 bytes and write 3 per column; 9,001 rows of 8,192 take
// 92 us, 5.6 TB/s (a large copy reaches 4.9), 48 rows of 4,096 3.4 us, a launch's
// latency and two trips to memory.  Squares are summed in float64: float32 squares
// of values past 1.8e19 overflow, and the conversions hide behind the loads.
#include <algorithm>

#include "fp8.h"

namespace sdv {

namespace {

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float (&v)[8]) {
  const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r[i] << 16);
    v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <>
__device__ __forceinline__ void store8<uint16_t>(uint16_t* p, const float (&v)[8]) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (__bf16)v[i];
  *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, r);
}
template <>
__device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// Maximum over the 16 lanes of a DPP row.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_f32<kDppXor1>(v));
  v = fmaxf(v, dpp_f32<kDppXor2>(v));
  v = fmaxf(v, dpp_f32<kDppRowHalfMirror>(v));
  return fmaxf(v, dpp_f32<kDppRowMirror>(v));
}

// y / s, rounded to nearest, with the rounded reciprocal of s: the remainder of the
// first product is exact and corrects it (Markstein's division step).  Its sign is
// taken so that a zero keeps y's.  2,000 rows of 4,096: 12.7 us so, 12.3 with the product
// alone, 14.7 with the division's instructions.
__device__ __forceinline__ float quotient(float y, float s, float to) {
  const float q = y * to;
  return fmaf(-fmaf(q, s, -y), to, q);
}

template <typename T, int THREADS, int R>
__global__ __launch_bounds__(THREADS)
void residual_norm_kernel(int scale_stride, int width, float eps, const T* x, const T* residual, const T* __restrict__ weight,
                          T* new_residual, uint8_t* __restrict__ out, float* __restrict__ out_scale) {
  constexpr int NW = THREADS / kWave;
  __shared__ double sums[NW];
  const int row = blockIdx.x, t = threadIdx.x;
  const int groups = width / 8;
  const int64_t base = (int64_t)row * width;
  float h[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int g = min(t + i * THREADS, groups - 1);  // lanes past the row read its last group, unused
    load8(x + base + g * 8, h[i]);
  }
  if (residual != nullptr) {
    float r[R][8];
#pragma unroll
    for (int i = 0; i < R; ++i) load8(residual + base + min(t + i * THREADS, groups - 1) * 8, r[i]);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += r[i][e];
  }
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (t + i * THREADS < groups) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma((double)h[i][e], (double)h[i][e], sum);
    }
  sum = wave_sum_f64(sum);
  if (NW > 1) {
    if ((t & 63) == 0) sums[t >> 6] = sum;
    __syncthreads();
    sum = sums[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += sums[w];
  }
  // 1/rms as inv * up, up a power of two: h * up is exact, and codes are those of
  // v / (max|v| / 448), v = h * up * weight: three roundings, and inv enters the scale
  // alone.  Rows of subnormal numbers are lifted first.  Infinities, NaN, and zeros with
  // eps 0: h * up is 0 or NaN as h / rms is.
  const double by = 1.0 / sqrt(sum / (double)width + (double)eps);
  const bool number = by > 0.0 && by < (double)INFINITY;
  const int e = number ? max(ilogb(by), -126) : 0;
  const bool lift = e > 126;
  const float up = number ? ldexpf(1.f, lift ? e - 64 : e) : (float)by;
  const float inv = number ? (float)ldexp(by, -e) : 1.f;
  const float least = 0x1p-126f / inv;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int g = t + i * THREADS;
    const bool live = g < groups;
    if (live && new_residual != nullptr) store8(new_residual + base + g * 8, h[i]);
    if (lift) {
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] *= 0x1p64f;
    }
    float w[8], v[8], most = 0.f;
    load8(weight + min(g, groups - 1) * 8, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = h[i][e] * up * w[e];
      most = fmaxf(most, live ? fabsf(v[e]) : 0.f);
    }
    most = row_max(most);
    const float part = most / 448.f, s = fmaxf(part, least);
    const float to = 1.f / s;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = quotient(v[e], s, to);
    if (live) {
      const u32x2 c = {encode4(v[0], v[1], v[2], v[3]), encode4(v[4], v[5], v[6], v[7])};
      *reinterpret_cast<u32x2*>(out + base + g * 8) = c;
      if ((t & 15) == 0) out_scale[(int64_t)(g / 16) * scale_stride + row] = fmaxf(part * inv, 0x1p-126f);
    }
  }
}

}  // namespace

hipError_t launch_residual_norm(bool f32, int rows, int width, float eps, const void* x, const void* residual,
                                const void* weight, void* new_residual, uint8_t* out, float* out_scale,
                                hipStream_t stream) {
  const int groups = width / 8;
  // Few groups per thread, few idle threads.  30,000 rows of 4,096: 149 us with 256
  // threads of two groups, 154 with 512 of one, 155 with 128 of four; of 8,192: 296 with 512
  // of two, 302 with 256 of four, 312 with 1,024 of one.
  // A launch's threads number less than 2^32, so that many rows are several launches.
#define SDV_NORM(T, N, R)                                                                                             \
  for (int r0 = 0; r0 < rows; r0 += (1 << 30) / N) {                                                                  \
    const int64_t at = (int64_t)r0 * width;                                                                           \
    const T* const res = residual != nullptr ? static_cast<const T*>(residual) + at : nullptr;                        \
    T* const next = new_residual != nullptr ? static_cast<T*>(new_residual) + at : nullptr;                           \
    hipLaunchKernelGGL((residual_norm_kernel<T, N, R>), dim3(std::min(rows - r0, (1 << 30) / N)), dim3(N), 0, stream, \
                       rows, width, eps, static_cast<const T*>(x) + at, res, static_cast<const T*>(weight), next,     \
                       out + at, out_scale + r0);                                                                     \
  }
#define SDV_NORM_SIZES(T)                            \
  if (groups <= 64) SDV_NORM(T, 64, 1)               \
  else if (groups <= 256) SDV_NORM(T, 256, 1)        \
  else if (groups <= 512) SDV_NORM(T, 256, 2)        \
  else if (groups <= 1024) SDV_NORM(T, 512, 2)       \
  else if (groups <= 2048) SDV_NORM(T, 1024, 2)      \
  else SDV_NORM(T, 1024, 4)
  if (f32) {
    SDV_NORM_SIZES(float)
  } else {
    SDV_NORM_SIZES(uint16_t)
  }
#undef SDV_NORM_SIZES
#undef SDV_NORM
  return hipGetLastError();
}

}  // namespace sdv
