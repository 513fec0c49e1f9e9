// Arithmetic on two 32-bit numbers at a time, which sm_100 and on do in one instruction.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace aiq {
#ifdef __CUDACC__
// Pairs of 32-bit numbers, an instruction for both.
struct Two {
  uint64_t v;
  Two() = default;
  __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ explicit Two(float2 x) : Two(x.x, x.y) {}
  __device__ __forceinline__ float2 parts() const {
    float2 x;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x.x), "=f"(x.y) : "l"(v));
    return x;
  }
};
__device__ __forceinline__ Two add_rd(Two a, Two b) {
  asm("add.rm.f32x2 %0, %1, %2;" : "=l"(a.v) : "l"(a.v), "l"(b.v));
  return a;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(a.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return a;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(a.v) : "l"(a.v), "l"(b.v));
  return a;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a.v) : "l"(a.v), "l"(b.v));
  return a;
}
__device__ __forceinline__ Two sub2(Two a, Two b) { return fma2(b, Two(-1.f, -1.f), a); }  // (exact but for the difference's rounding)
#endif
}  // namespace aiq
