// What the distillation kernels share: a row's list as a table that the sweeps look its tokens up
// in, and the arithmetic of the loss on the classes {listed tokens, everything else}.
//
// The sums are kept in units of log2: with c = log2(e) / temperature a logit z has the exponent
// z c, a reference R is itself a rounded exponent, and exp2(fma(z, c, -R)) rounds once; what R
// rounds off cancels, because total = 2^R sum is formed with the same R.
#pragma once

#include "cis_tok_row.h"

namespace cis {

// Lowest reference of a row's sum: finite where there is nothing but -inf.
constexpr float kMinExp = -0x1p126f;
constexpr float kLn2 = 0.693147180559945309417f;
// expm1(d) - d >= 0, to a few units in the last place (near 0 by its series, which does not
// cancel: nine terms, the first left out below 2^-24 of the sum up to |d| = 0.6).
__device__ __forceinline__ float expm1_less(float d) {
  if (fabsf(d) > 0.6f) return expm1f(d) - d;
  float s = 1.f / 3628800.f;
  s = __builtin_fmaf(s, d, 1.f / 362880.f);
  s = __builtin_fmaf(s, d, 1.f / 40320.f);
  s = __builtin_fmaf(s, d, 1.f / 5040.f);
  s = __builtin_fmaf(s, d, 1.f / 720.f);
  s = __builtin_fmaf(s, d, 1.f / 120.f);
  s = __builtin_fmaf(s, d, 1.f / 24.f);
  s = __builtin_fmaf(s, d, 1.f / 6.f);
  s = __builtin_fmaf(s, d, 0.5f);
  return s * d * d;
}

// log(rest / (list + rest)), accurate at both ends.
__device__ __forceinline__ float log_rest(float list, float rest) {
  const float total = list + rest;
  return rest > 0.5f * total ? log1pf(-list / total) : logf(rest / total);
}

// A class's part of sum a log(a/b) for log a - log b = d: a log(a/b) - a + b, whose limit at a = 0
// is b.
__device__ __forceinline__ float kl_part(float a, float d, float b) {
  return a > 0.f ? a * expm1_less(-d) : b;
}

// What sweep 2 needs of a row: a gradient of sgn exp2(fma(z, c, -b2)) where the token is not listed.
struct RestGrad {
  float b2;
  uint32_t neg;
};
__device__ __forceinline__ RestGrad rest_grad(float coef, float R, float total) {
  const float b2 = coef != 0.f ? (R + log2f(total)) - log2f(fabsf(coef)) : INFINITY;
  return RestGrad{b2, coef < 0.f ? 1u : 0u};
}

// Gradient coefficients (before scale * weight / temperature) of a listed token and, of p_j, of the
// others.
__device__ __forceinline__ float listed_grad(bool reverse, float p, float q, float d, float kl) {
  if (reverse) return p > 0.f ? p * (d - kl) : 0.f;
  return q > 0.f && d < 1.f ? q * expm1f(d) : p - q;   // (p - q cancels where they are close)
}
__device__ __forceinline__ float others_grad(bool reverse, float p_rest, float q_rest, float d,
                                             float kl) {
  if (!(p_rest > 0.f)) return 0.f;
  if (reverse) return d - kl;
  return q_rest > 0.f ? -expm1f(-d) : 1.f;
}

}  // namespace cis
