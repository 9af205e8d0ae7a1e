// How the 8-bit kernels make a row's bytes and scale from its fp32 values.
#pragma once

#include "cats_common.cuh"

namespace cats {

constexpr float kTinyMax = 7.888609052210118e-31f;    // 2^-100: the smallest maximum a scale is made from

// rint(127 v / a) as bytes, v = y rs; |v| <= a, so the result is within 127 whatever rs and a are.
// One bf16 element in a thousand is a tie, 127 v / a an exact half, and v fl(127 / a) puts it on either side of the half (one in 1900
// elements a step off).  So the factor is kept in two parts, hi + lo = 127 / a to 2^-29 or better, and fma(v, hi, v lo) rounds the
// quotient once: one that fp32 holds, a tie among them, is exact.  SwiGLU's values have several roundings behind them and
// no exact ties: they take hi alone (the second part took 7 us more for 4096 x 11008 and its values).  Two instructions per element
// more than hi alone: 22016 x 4096 bf16 and its values 82.6 -> 84.2 us, norm of 8191 x 4096 53.3 either way.
// Rounding to a whole number: the sum with 1.5 * 2^23 leaves it (ties to even) in the low bits; the conversion instruction has
// a sixteenth of the FMA rate and shares its unit with ex2 and rcp.
constexpr float kRintMagic = 12582912.f;
struct Factor { float hi, lo; };
__device__ __forceinline__ Factor factor_127_over(float a) {
    const float hi = 127.f / a;
    return {hi, fmaf(-hi, a, 127.f) * (hi * (1.f / 127.f))};      // the remainder of the division, over a
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

}  // namespace cats
