// An fp64 exponential for the logits' kernels.
#pragma once

#include <hip/hip_runtime.h>

namespace kvg {

namespace {

// e^x for x below 700, in fp64: x = (64 k + j) ln2 / 64 + r, |r| <= ln2 / 128, so
// e^x = 2^k 2^(j/64) e^r with the table tab[j] = 2^(j/64) and e^r - 1 by its series to r^5
// (the rest is below 4e-17).  Below the smallest subnormal the result is an exact 0, so that a
// logit of -inf weighs what it should.
__device__ __forceinline__ double exp_table(double x, const double* tab) {
  constexpr double kInv = 92.332482616893656877;               // 64 / ln 2
  constexpr double kHi = 0x1.62e42fefa39efp-7, kLo = 0x1.abc9e3b39803fp-62;   // ln 2 / 64
  const double xc = x >= -750.0 ? x : -750.0;      // NaN too: the conversion needs a number
  const double n = __builtin_rint(xc * kInv);
  const double r = fma(-n, kLo, fma(-n, kHi, xc));
  const int m = (int)n;
  const double p = fma(r * r, fma(r, fma(r, fma(r, 1.0 / 120.0, 1.0 / 24.0), 1.0 / 6.0), 0.5), r);
  const double t = tab[m & 63];
  const double y = __builtin_ldexp(fma(t, p, t), m >> 6);
  return x >= -750.0 ? y : x < -750.0 ? 0.0 : x;
}

}  // namespace

}  // namespace kvg
