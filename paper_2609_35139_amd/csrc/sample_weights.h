// What a logit weighs in sampling (gfx950; the host computes the same, for the tests).
#pragma once
#include <cmath>

namespace cr {

typedef unsigned long long u64;

// exp((x - x_0) / T) 2^shift.  With c = 64 log2(e) / T, x c - x_0 c = n + r - f: n whole,
// |r| <= 1/2, f what x_0 c is off a whole number, the same for all tokens.  2^(n / 64)
// comes from a table (with 2^(-f / 64) in it) and the exponent, 2^(r / 64) by its series
// up to the fourth power (relative error 4e-14, below a step for all but the largest).
// Products inside the fused operations are exact, so nothing is lost however far x and x_0
// are from 0.  A pass that forms weights takes a CU 46 us for a row of 151,936 logits and
// issues about 37 vector instructions for a logit, ten of them fp64 (counters of 256 rows
// without a filter, less those of the first token alone).  At four cycles of a SIMD each
// that is 37 us: bound by their number.  Neither the chains of eight logits side by side, a
// stage at a time, nor a table for each bank changed it.
constexpr int kExpTable = 64;
constexpr float kLowestLogit = -3.402823466e38f;      // the type's lowest
// The largest fp32 number that is not above x, but no less than the lowest.
__host__ __device__ __forceinline__ float at_most(double x) {
  const float f = (float)x;
  return fmaxf((double)f > x ? nextafterf(f, -INFINITY) : f, kLowestLogit);
}
struct Weigher {
  static constexpr u64 kOffset = 0x4330000000000000ull;
  const double* table;   // 2^((j - f) / 64) 2^shift
  double c, whole;       // whole: 1.5 2^52 less the whole number next to x_0 c
  // What lies below weighs less than 2^-20 steps.  Rounded downwards, so below top: where
  // floats lie further apart than that (T = 1e-8 from a top of 8 on, T = 1 from 1e9 on), the
  // next float would be top itself, and all of the row would weigh as much as that.
  float lowest;
  __host__ __device__ __forceinline__ u64 operator()(float logit) const {
    const double x = (double)(logit > lowest ? logit : lowest);      // (NaN too)
    const double m = __builtin_fma(x, c, whole);
    // (the float next to the lowest may lie further down; what it weighs is still no step)
    const int low = (int)(bits_of(m) & 0xffffffff), n = low > -80 * kExpTable ? low : -80 * kExpTable;
    const long long b = bits_of(table[n & (kExpTable - 1)]) + ((long long)(n & ~(kExpTable - 1)) * (1ll << 46));
    const double r = __builtin_fma(x, c, whole - m);
    constexpr double y = 0.69314718055994530942 / kExpTable;
    double e = __builtin_fma(r, y * y * y * y / 24., y * y * y / 6.);
    e = __builtin_fma(e, r, y * y / 2.);
    e = __builtin_fma(e, r, y);
    e = __builtin_fma(e, r, 1.);
    // in whole steps: added to 2^52, the bits are kOffset + the weight
    return (u64)bits_of(__builtin_fma(__builtin_bit_cast(double, b), e, 4503599627370496.)) - kOffset;
  }
  __host__ __device__ __forceinline__ static long long bits_of(double x) { return __builtin_bit_cast(long long, x); }
  // of a row whose largest logit is top, finite, |top c| < 2^48, and entry j of its table
  __host__ __device__ __forceinline__ static Weigher of(const double* table, float top, double c) {
    return Weigher{table, c, 6755399441055744. - rint((double)top * c),
                   at_most((double)top - 64. * kExpTable / c)};
  }
  __host__ __device__ __forceinline__ static double entry(int j, float top, double c, double one) {
    const double at_top = (double)top * c;
    const double off = (at_top - rint(at_top)) + __builtin_fma((double)top, c, -at_top);
    return exp2((j - off) / kExpTable) * one;
  }
};
// The smallest logit whose p is at least min_p, which is that of (x - x_0) / T >=
// log(min_p): so min_p is a bound of the logits themselves.
__host__ __device__ __forceinline__ float least_logit(float min_p, double top, double temperature) {
  const double t = temperature * log((double)min_p);
  auto holds = [&](float x) { return (double)x - top >= t; };
  float x = fmaxf((float)(top + t), kLowestLogit);
  for (int i = 0; i < 4 && !holds(x); ++i) x = nextafterf(x, INFINITY);
  for (int i = 0; i < 4 && holds(nextafterf(x, -INFINITY)); ++i) x = nextafterf(x, -INFINITY);
  return fminf(x, (float)top);
}

}  // namespace cr
