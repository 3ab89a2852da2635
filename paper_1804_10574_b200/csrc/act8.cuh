// Rows of 8-bit codes with a scale each: m = max(max |x|, 127 2^-126), scale = m / 127 rounded to fp32, code = 127 x / m
// rounded once, halves to even.  The maximum's lower bound keeps the scale a normal number, so that its reciprocal is finite; the
// scale of an fp32 row up to FLT_MAX is rounded down, so that 127 scale is finite.
// A row that holds a NaN or an infinity has scale NaN and codes 0: all that is made of it is NaN.
#pragma once
#include "common.cuh"

namespace ddg {

namespace {

constexpr float kAct8Least = 127.f * 1.17549435e-38f;  // 127 x 2^-126, exact
constexpr float kAct8MostScale = 8454659.f * 0x1p98f;  // FLT_MAX / 127 rounded down

struct Act8Row { float top, inv; };  // inv: NaN row 0, so that codes are 0

// From a row's largest magnitude as bits, which order as numbers do, infinity and NaN above them.
__device__ __forceinline__ Act8Row act8_row(uint32_t top_bits, float &scale) {
    if (top_bits >= 0x7f800000u) {
        scale = __int_as_float(0x7fffffff);
        return Act8Row{1.f, 0.f};
    }
    const float top = fmaxf(__uint_as_float(top_bits), kAct8Least);
    scale = fminf(__fdiv_rn(top, 127.f), kAct8MostScale);
    return Act8Row{top, __fdiv_rn(127.f, top)};
}

// The code of x.  x inv is off by less than 2^-15 of a step; only where that could decide between two codes is the quotient
// formed in 64 bits, whose distance from a border that it is not exactly on is 2^-33 at least (24-bit x and m).
__device__ __forceinline__ int act8_code(float x, const Act8Row &r) {
    if (r.inv == 0.f) return 0;
    const float t = x * r.inv, n = rintf(t);
    if (fabsf(t - n) > 0.5f - 0x1p-13f) return (int)rint(127.0 * (double)x / (double)r.top);
    return (int)n;
}

__device__ __forceinline__ uint32_t act8_pack4(int a, int b, int c, int d) {
    return __byte_perm(__byte_perm((uint32_t)a, (uint32_t)b, 0x0040), __byte_perm((uint32_t)c, (uint32_t)d, 0x0040), 0x5410);
}

// What a code stands for, in the element type.
template <typename T> __device__ __forceinline__ float act8_value(int code, float scale) { return to_f(from_f<T>((float)code * scale)); }

}  // namespace

}  // namespace ddg
