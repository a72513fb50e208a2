// FP32 arithmetic on two numbers at a time, and their square roots.
#pragma once

#include <cuda_runtime.h>

namespace fpq {

// two numbers at a time, each operation rounded on its own
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(__fmul_rn(a.x, b.x), __fmul_rn(a.y, b.y)); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(__fmaf_rn(a.x, b.x, c.x), __fmaf_rn(a.y, b.y, c.y)); }
__device__ __forceinline__ float2 both2(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 minus(float2 v) { return make_float2(-v.x, -v.y); }

// The square roots of two numbers, rounded to nearest, for v = 0 and 2^-96 <= v < infinity, without a branch: one step of
// Goldschmidt's iteration from an approximate 1 / sqrt(v), then Markstein's correction of the result by its exact remainder
// (P. Markstein, IBM J. Res. Dev. 34, 1990).  tests/test_adamw_table.py compares every such FP32 number.
__device__ __forceinline__ float2 roots_of(float2 v)
{
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(v.x, 1e-30f)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(v.y, 1e-30f)));
    float2 g = mul2(v, y), h = mul2(y, both2(0.5f));
    const float2 d = fma2(minus(h), g, both2(0.5f));
    g = fma2(g, d, g);
    h = fma2(h, d, h);
    return fma2(fma2(minus(g), g, v), h, g);
}

}  // namespace fpq
