// What the kernels over pages share (paged.cu, paged_tree.cu, paged_keep.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

namespace aatc {
namespace paged {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float2 widen(__nv_bfloat16, uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 widen(__half, uint32_t w) {
  __half2 h;
  *reinterpret_cast<uint32_t*>(&h) = w;
  return __half22float2(h);
}
__device__ __forceinline__ uint32_t narrow(__nv_bfloat16, float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t narrow(__half, float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void raise(int32_t* err, int32_t bits) {
  if (err) atomicOr(err, bits);
}

// a / b of values that are not negative, of 32 bits or mostly so
__device__ __forceinline__ int quotient(int a, int b) { return static_cast<unsigned>(a) / static_cast<unsigned>(b); }
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (a | b) >> 32 ? a / b : static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
}

__device__ __forceinline__ float exp2_of(float x) {            // (-inf: 0)
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh x = 1 - 2 / (e^(2 x) + 1), and where that cancels its Taylor series: either within 4e-7 of its value
__device__ __forceinline__ float tanh_of(float x) {
  const float a = fabsf(x), x2 = x * x;
  const float big = 1.0f - __fdividef(2.0f, exp2_of(2.0f * kLog2e * a) + 1.0f);
  const float small = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  return a < 0.25f ? x * small : copysignf(a > 20.0f ? 1.0f : big, x);
}
// cap tanh(s / cap) of a score, given y = s / cap too, in the same way, but the series times s itself: for caps so large that y has
// left the normal numbers it is s.
constexpr float kSeries = 0.25f;                               // of y, up to which the series holds
__device__ __forceinline__ float series_of(float s, float y) {
  const float y2 = y * y;
  return s * fmaf(y2, fmaf(y2, fmaf(y2, fmaf(y2, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
}
__device__ __forceinline__ float capped_of(float s, float y, float cap) {
  const float a = fabsf(y), big = cap * (1.0f - __fdividef(2.0f, exp2_of(2.0f * kLog2e * a) + 1.0f));
  return a < kSeries ? series_of(s, y) : copysignf(a > 20.0f ? cap : big, y);
}
// The same of N scores S, unit S and far_in S being s and y: mostly all of a warp's are in the series' range.
template <int N>
__device__ __forceinline__ void cap_far(uint32_t (&x)[N], float unit, float far_in, float cap) {
  float most = 0.0f;
#pragma unroll
  for (int j = 0; j < N; ++j) most = fmaxf(most, fabsf(__uint_as_float(x[j])));
  if (!__any_sync(0xffffffffu, most * fabsf(far_in) >= kSeries)) {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = __float_as_uint(series_of(__uint_as_float(x[j]) * unit, __uint_as_float(x[j]) * far_in));
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = __float_as_uint(capped_of(__uint_as_float(x[j]) * unit, __uint_as_float(x[j]) * far_in, cap));
  }
}

}  // namespace paged
}  // namespace aatc
