// Pairs of fp32 values: one instruction for two additions, products or multiply-adds (rounded to nearest, each by itself).
#pragma once
#include "common.cuh"

namespace ddg {

namespace {

struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float lo, float hi) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ F2 f2(float both) { return f2(both, both); }
__device__ __forceinline__ float2 parts(F2 a) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v)); return r; }
__device__ __forceinline__ F2 operator+(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 operator*(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ float sum2(F2 a) { const float2 p = parts(a); return p.x + p.y; }

// two bf16 values in a word, the first in its low half
__device__ __forceinline__ F2 bf16_pair(uint32_t w) { return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t to_bf16_pair(F2 a) {
    const float2 p = parts(a);
    const __nv_bfloat162 h = __floats2bfloat162_rn(p.x, p.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

}  // namespace

}  // namespace ddg
