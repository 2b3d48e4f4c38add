// Two fp32 operations as one instruction.
#pragma once

#include <stdint.h>

namespace retrace {
namespace {

__device__ __forceinline__ uint64_t bits2(float2 v) {
  uint64_t x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(v.x), "f"(v.y));
  return x;
}
__device__ __forceinline__ float2 floats2(uint64_t x) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(x));
  return v;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return floats2(y);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(bits2(a)), "l"(bits2(b)));
  return floats2(y);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t y;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(bits2(a)), "l"(bits2(b)));
  return floats2(y);
}

}  // namespace
}  // namespace retrace
