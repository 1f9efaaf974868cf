// Pairs of fp32 values (internal).
#pragma once
#include "octet.cuh"

namespace hn {

// two fp32 values in one instruction each
typedef float2 f2;
__device__ __forceinline__ f2 make2(float x, float y) { return make_float2(x, y); }
__device__ __forceinline__ void split2(f2 a, float &x, float &y) { x = a.x; y = a.y; }
__device__ __forceinline__ f2 pair(float x) { return make_float2(x, x); }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float sum2(f2 a) { float x, y; split2(a, x, y); return x + y; }
__device__ __forceinline__ f2 widen2(unsigned w) { f2 f; unpack2(w, f.x, f.y); return f; }
__device__ __forceinline__ unsigned narrow2(f2 a) { float x, y; split2(a, x, y); return pack2(x, y); }
__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float rcp(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

}  // namespace hn
