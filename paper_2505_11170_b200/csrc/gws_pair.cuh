// FP32 arithmetic on pairs: one instruction for two numbers.
#pragma once
#include <stdint.h>

namespace {

// Two FP32 numbers in a register pair: one instruction rounds both as the scalar ones do.
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 two(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 both(float a) { return two(a, a); }
__device__ __forceinline__ float first_of(F2 a) {
  float x;
  asm("mov.b64 {%0, _}, %1;" : "=f"(x) : "l"(a.v));
  return x;
}
__device__ __forceinline__ float second_of(F2 a) {
  float y;
  asm("mov.b64 {_, %0}, %1;" : "=f"(y) : "l"(a.v));
  return y;
}
// Two additions: add.rn.f32x2 would be fused with a mul.rn.f32x2 before it, under -fmad=false too.
__device__ __forceinline__ F2 add2(F2 a, F2 b) { return two(__fadd_rn(first_of(a), first_of(b)), __fadd_rn(second_of(a), second_of(b))); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

}  // namespace
