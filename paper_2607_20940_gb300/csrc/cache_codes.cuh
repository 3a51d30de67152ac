// What the 4-bit cache's attention kernels have in common: conversions of codes
// and scales, rows of queries in f16, divisions of shares, the join.
#pragma once

#include <stdint.h>

#include "cache.h"
#include "ptx.cuh"

namespace msf {
namespace codes {

// Byte I of w as two f16: the lower code in the lower half. (On a GB300 at
// least 42 lanes a clock and SM; taking sign and magnitude apart with shifts and
// logic reaches 22.)
template <int I>
__device__ __forceinline__ uint32_t e2m1_f16x2(uint32_t w) {
    uint32_t r;
    if constexpr (I == 0)
        asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %1;\ncvt.rn.f16x2.e2m1x2 %0, a;\n}" : "=r"(r) : "r"(w));
    else if constexpr (I == 1)
        asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %1;\ncvt.rn.f16x2.e2m1x2 %0, b;\n}" : "=r"(r) : "r"(w));
    else if constexpr (I == 2)
        asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %1;\ncvt.rn.f16x2.e2m1x2 %0, c;\n}" : "=r"(r) : "r"(w));
    else
        asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %1;\ncvt.rn.f16x2.e2m1x2 %0, d;\n}" : "=r"(r) : "r"(w));
    return r;
}
// Two scales (the lower 16 bits) as two f16.
__device__ __forceinline__ uint32_t e4m3_f16x2(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
    return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float bf(uint32_t x16) { return __uint_as_float(x16 << 16); }

// How a row of queries goes into f16: times the power of two that takes its
// largest value to [2^14, 2^15), so a value loses bits only below 2^-28 of that
// (f16 keeps 24 binary places), far less than an fp32 sum does. `e`: the biased
// exponent of the largest; rows below 2^-99 are taken as that.
__device__ __forceinline__ int row_exponent(uint32_t largest_bf16) { return max((int)(largest_bf16 >> 7), 28); }
__device__ __forceinline__ float row_up(int e) { return __uint_as_float((uint32_t)(268 - e) << 23); }
__device__ __forceinline__ float row_down(int e) { return __uint_as_float((uint32_t)(e - 14) << 23); }
// What takes a score of such a row to base 2; never 0 or infinite, so that a
// masked score stays -infinity and a row of zeros 0.
__device__ __forceinline__ float row_factor(int e, float scale) {
    return fminf(fmaxf(row_down(e) * scale * 1.4426950408889634f, 1.17549435e-38f), 3.0e38f);
}

// n / d, by a 32-bit division where n allows it (a 64-bit one takes hundreds of cycles).
__device__ __forceinline__ long long divide(long long n, long long d) {
    if (((unsigned long long)n | (unsigned long long)d) >> 32) return (long long)((unsigned long long)n / (unsigned long long)d);
    return (long long)((unsigned)n / (unsigned)d);
}

// The joined result's weights: this attention's unnormalised output times own,
// the base's times other. M: running maximum (base 2), L: sum.
struct Join {
    float own, other, lse;
};
__device__ __forceinline__ Join join_of(float M, float L, bool has_base, float base_lse, float unit) {
    Join j;
    j.lse = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : L == 0.f ? -INFINITY : L;
    j.own = L > 0.f ? 1.f / L : 0.f;
    j.other = 0.f;
    if (L != L) j.own = L;  // NaN stays
    if (has_base) {
        const float top = fmaxf(j.lse, base_lse);
        if (top == -INFINITY) {
            j.own = 0.f;
        } else {
            const float a = expf(j.lse - top), b = expf(base_lse - top);
            j.own *= a / (a + b);
            j.other = b / (a + b);
            j.lse = top + logf(a + b);
        }
    }
    j.own *= unit;
    return j;
}

}  // namespace codes
}  // namespace msf
