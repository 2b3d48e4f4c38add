// A cache in 8 bits: e4m3 numbers, and a power of two for each page and head.
#pragma once

#include <cuda_fp8.h>

#include "../common.cuh"
#include "serve.h"

namespace retrace {

template <>
__device__ __forceinline__ float to_f32<__nv_fp8_e4m3>(__nv_fp8_e4m3 x) { return (float)x; }

namespace {

constexpr int kMostExponent = 40;  // of a page, of either sign
constexpr float kMostE4m3 = 448.f;

__device__ __forceinline__ int clamp_exponent(int e) { return min(max(e, -kMostExponent), kMostExponent); }
// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ int page_exponent(const AttendArgs& a, const int8_t* exps, int page, int head) {
  return clamp_exponent(exps[page * a.exp_page + head * a.exp_head]);
}

// The least e in [-40, 40] with a <= 448 2^e, a not negative and no NaN: 448 is 1.75 * 2^8.
__device__ __forceinline__ int exponent_for(float a) {
  const uint32_t bits = __float_as_uint(a);
  return clamp_exponent((int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u));
}

// Two e4m3 numbers, the first in the low byte.
__device__ __forceinline__ float2 e4m3_floats(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(__half2(h));
}
// To the nearest, ties to even; beyond 448 the largest, NaN stays.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}

}  // namespace
}  // namespace retrace
