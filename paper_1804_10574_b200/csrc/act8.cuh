// Rows of 8-bit codes with a scale each: m = max(max |x|, 127 2^-126), scale = m / 127 rounded to fp32, code = 127 x / m
// rounded once, halves to even.  The maximum's lower bound keeps the scale a normal number, so that its reciprocal is finite; the
// scale of an fp32 row up to FLT_MAX is rounded down, so that 127 scale is finite.
// A row that holds a NaN or an infinity has scale NaN and codes 0: all that is made of it is NaN.
#pragma once
#include "f32x2.cuh"

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

// N codes at once, in the words' bytes.  t = 127 x / m rounded by adding 1.5 x 2^23, which leaves the whole number in the sum's
// low byte.
//   kBf16 (x and m are bf16 values): 127 x is exact (here 127 / 128 x, and m / 128), and the quotient corrected by its remainder
//     (Markstein, 1990) is exactly a border where it is one, as x = m / 2 is, and else nearer to the quotient than any border
//     (2^-17 at least).
//   kF32: x inv, with one test for all of them whether a border is so near that it could decide; then they are formed in 64 bits.
//   kNear: x inv, less than 2^-15 of a step off, where x is itself a rounded result.
enum Act8Kind { kBf16, kF32, kNear };
template <Act8Kind KIND, int N> __device__ __forceinline__ void act8_codes(const F2 (&x)[N / 2], const Act8Row &r, uint32_t (&w)[(N + 3) / 4]) {
    constexpr float kRound = 12582912.f;
    const F2 inv = f2(r.inv), up = f2(kRound);
    uint32_t n[N];
    float off = 0.f;
    const F2 inv_m = f2(r.inv * (128.f / 127.f)), neg_m = f2(-r.top * 0x1p-7f), by = f2(127.f * 0x1p-7f);  // all by 2^-7: nothing overflows
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        F2 t;
        if (KIND == kBf16) {
            const F2 x127 = x[k] * by;
            t = x127 * inv_m;
            t = fma2(fma2(t, neg_m, x127), inv_m, t);
        } else {
            t = x[k] * inv;
        }
        const F2 s = t + up;
        const float2 sp = parts(s);
        n[2 * k] = __float_as_uint(sp.x);
        n[2 * k + 1] = __float_as_uint(sp.y);
        if (KIND == kF32) {
            const float2 d = parts(fma2(s + f2(-kRound), f2(-1.f), t));
            off = fmaxf(off, fmaxf(fabsf(d.x), fabsf(d.y)));
        }
    }
    if (KIND == kF32 && off > 0.5f - 0x1p-14f) {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
            const float2 p = parts(x[k]);
            n[2 * k] = (uint32_t)act8_code(p.x, r);
            n[2 * k + 1] = (uint32_t)act8_code(p.y, r);
        }
    }
    const uint32_t keep = r.inv == 0.f ? 0u : 0xffffffffu;  // a row of codes 0, whatever stands in it
#pragma unroll
    for (int k = 0; k < N; k += 4)
        w[k / 4] = keep & __byte_perm(__byte_perm(n[k], n[k + 1], 0x0040), N > 2 ? __byte_perm(n[N > 2 ? k + 2 : 0], n[N > 2 ? k + 3 : 0], 0x0040) : 0u, 0x5410);
}

// VEC codes, 1, 4 or 8, on a boundary of as many bytes.
template <Act8Kind KIND, int VEC> __device__ __forceinline__ void act8_store(int8_t *to, const float (&v)[VEC], const Act8Row &r) {
    if constexpr (VEC == 1) {
        *to = (int8_t)act8_code(v[0], r);
    } else {
        F2 x[VEC / 2];
        uint32_t w[VEC / 4];
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) x[j] = f2(v[2 * j], v[2 * j + 1]);
        act8_codes<KIND, VEC>(x, r, w);
        if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(to) = w[0];
    }
}

// A thread's pairs (see row_ring.cuh) to a row of codes.
template <Act8Kind KIND, int VEC, int ITER> __device__ __forceinline__ void act8_share_store(int8_t *row, int C, int threads, const F2 (&v)[VEC * ITER / 2], const Act8Row &r) {
    if constexpr (VEC > 1) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * threads + threadIdx.x) * VEC;
            F2 x[VEC / 2];
            uint32_t w[VEC / 4];
#pragma unroll
            for (int j = 0; j < VEC / 2; ++j) x[j] = v[i * VEC / 2 + j];
            act8_codes<KIND, VEC>(x, r, w);
            if (c >= C) continue;
            if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(row + c) = w[0];
        }
    } else {
        uint32_t w[(ITER + 3) / 4];
        act8_codes<KIND, ITER>(v, r, w);
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = i * threads + threadIdx.x;
            if (c < C) row[c] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
        }
    }
}

// What a code stands for, in the element type.
template <typename T> __device__ __forceinline__ float act8_value(int code, float scale) { return to_f(from_f<T>((float)code * scale)); }

}  // namespace

}  // namespace ddg
