// What the distillation kernels share: a row's list as a table that the sweeps look its tokens up
// in, and the arithmetic of the loss on the classes {listed tokens, everything else}.
//
// Every exponent is that of a difference of logits, (z - m) c with c = log2(e) / temperature and m the
// largest logit of the sum: as large as the difference is, wherever the logits lie, and finite sums for
// every temperature. (fma(z, c, -m c) is an instruction less, but m c rounds at its own size: 3e-6 of
// every value for logits near 100, and sums of 0 or inf once it is off by 128, at temperatures of 1e-8.)
#pragma once

#include "cis_tok_row.h"

namespace cis {

constexpr float kLn2 = 0.693147180559945309417f;
// expm1(d) - d for |d| <= kNearLog by its series (which does not cancel): nine terms, the first left
// out below 2^-24 of the sum.
constexpr float kNearLog = 0.6f;
__device__ __forceinline__ float expm1_less(float d) {
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

// Log of the share of a token x below the largest, of a total of 2^L. (In units of log2, that of the
// type's lowest logit would be past float32.) Teacher and student round alike here: shares of the same
// logits are the same bits.
__device__ __forceinline__ float log_share(float x, float inv_t, float L) {
#pragma clang fp contract(off)
  return x * inv_t - L * kLn2;
}

// log(rest / (list + rest)), accurate at both ends; x = log rest (which may be far below what rest can be),
// 2^L = list + rest.
__device__ __forceinline__ float log_rest(float list, float rest, float x, float L) {
  const float total = list + rest;
  if (rest > 0.5f * total) return log1pf(-list / total);
  return rest > 0x1p-64f * total ? logf(rest / total) : x - L * kLn2;
}

// A class's part of sum a log(a/b) for log a - log b = d: a log(a/b) - a + b >= 0, where a and b are
// near each other from the series, since the terms cancel there; b at a = 0.
__device__ __forceinline__ float kl_part(float a, float d, float b) {
  if (!(a > 0.f)) return b;
  return fabsf(d) <= kNearLog ? a * expm1_less(-d) : __builtin_fmaf(a, d, b - a);
}

// The gradient of a class as a factor for its tokens, whose exponentials relative to m sum up to s. A
// factor above 1 leaves its power of two to the exponent: only a gradient below 2^-126 is flushed.
__device__ __forceinline__ RestGrad rest_grad(float grad, float m, float s) {
  const float g = grad == 0.f || s == 0.f ? 0.f : grad / s;
  int up = __builtin_amdgcn_frexp_expf(g);   // (0 for inf and NaN)
  up = up > 0 ? up : 0;
  return RestGrad{m, (float)up, __builtin_amdgcn_ldexpf(g, -up)};
}

// cf exp(l) f for the log l of a share, which may lie far below float32 where the product does not:
// the factors' powers of two join the exponent. cf = mant 2^up.
__device__ __forceinline__ float share_grad(float l, float f, float mant, int up) {
  up += __builtin_amdgcn_frexp_expf(f);
  return fast_exp2(__builtin_fmaf(l, kLog2e, (float)up)) * (mant * __builtin_amdgcn_frexp_mantf(f));
}
// Gradient of a class, by cf = mant 2^up = scale * weight / temperature: a listed token's, or that of
// all others, each of which has it in proportion to its exponential. (lp, lq: logs of its shares)
__device__ __forceinline__ float class_grad(bool reverse, float lp, float lq, float kl, float mant,
                                            int up) {
  const float d = lp - lq;
  if (reverse) return lp > -INFINITY ? share_grad(lp, d - kl, mant, up) : 0.f;
  if (fabsf(d) <= kNearLog)   // (p - q cancels near 0)
    return share_grad(lq, d + expm1_less(d), mant, up);
  return share_grad(lp, 1.f, mant, up) - share_grad(lq, 1.f, mant, up);
}

// ------------------------------------------------------------------------------------------
// A row's list in LDS, and the loss on it by one wave (KMAX entries at most; lane l has entries l,
// l + 64, ...).
// ------------------------------------------------------------------------------------------
constexpr uint32_t kNone = 0xFFFFFFFFu;

template <int KMAX>
struct ListShared {
  int32_t id[KMAX];       // -1: no entry
  float z[KMAX];          // the student's logits
  float lq[KMAX];         // the teacher's logits; from teacher_list() on log q
  float q[KMAX];
  uint32_t grad[KMAX];    // gradient, in the logits' format
};

// Both lists' sums, in every lane.
struct Teacher {
  float q_rest, log_rest;   // the tail's share, and its log
  bool finite;
};
struct Student {
  float term;
  RestGrad rest;
  bool finite;
};

// A lane's share of a sum over the entries.
template <class F>
__device__ __forceinline__ void each_entry(const int32_t* id, int K, int lane, F&& f) {
  for (int k = lane; k < K; k += 64)
    if (id[k] >= 0) f(k);
}

__device__ __forceinline__ float row_tail(const DistillArgs& a, int64_t row) {
  return a.tail ? sload(a.tail + row) : -INFINITY;
}
__device__ __forceinline__ float row_weight(const DistillArgs& a, int64_t row) {
  return a.weight ? sload(a.weight + row) : 1.f;
}

// log q of the listed tokens, and of the tail.
template <int KMAX>
__device__ __forceinline__ Teacher teacher_list(const DistillArgs& a, float tail,
                                                ListShared<KMAX>& sh, int lane) {
  float m = -INFINITY;
  each_entry(sh.id, a.K, lane, [&](int k) { m = fmaxf(m, sh.lq[k]); });
  m = wave_max(m);
  // the tail beside the list's largest: their difference in double, since each is rounded at its own
  // size. Where the tail is the larger one, all are relative to it.
  float t = tail < INFINITY ? m > -INFINITY ? (float)((double)tail - (double)m * a.inv_t64)
                              : tail > -INFINITY ? 0.f : -INFINITY
                            : NAN;
  const float above = t > 0.f ? t : 0.f;
  if (t > 0.f) t = 0.f;
  m = sum_ref(m);
  float s = 0.f;
  const float c = a.c, up = above * kLog2e;
  each_entry(sh.id, a.K, lane, [&](int k) { s += fast_exp2((sh.lq[k] - m) * c - up); });
  s = wave_sum(s);
  const float rest = fast_exp2(t * kLog2e), total = s + rest, L = log2f(total);
  each_entry(sh.id, a.K, lane, [&](int k) {
    const float x = sh.lq[k] - m;
    sh.q[k] = fast_exp2((x * c - up) - L);
    sh.lq[k] = log_share(x, a.inv_t, L) - above;
  });
  return Teacher{rest / total, log_rest(s, rest, t, L), total > 0.f && total < INFINITY};
}

// The loss of a row whose listed logits are at sh.z and whose other tokens' exponentials relative to
// m_rest sum up to s_rest, and with BWD its gradient: of the listed tokens at sh.grad.
template <class E, bool BWD, int KMAX>
__device__ __forceinline__ Student student_list(const DistillArgs& a, float weight,
                                                ListShared<KMAX>& sh, int lane, const Teacher& t,
                                                float m_rest, float s_rest) {
  const float c = a.c;
  const bool reverse = a.reverse != 0;
  float m = -INFINITY;
  each_entry(sh.id, a.K, lane, [&](int k) { m = fmaxf(m, sh.z[k]); });
  m = fmaxf(m_rest, wave_max(m));
  float s = 0.f;
  each_entry(sh.id, a.K, lane, [&](int k) { s += fast_exp2((sh.z[k] - m) * c); });
  s = wave_sum(s);
  const float rest = s_rest * fast_exp2((m_rest - m) * c);
  const float total = s + rest, L = log2f(total);
  const float p_rest = rest / total,
              lp_rest = log_rest(s, rest, (m_rest - m) * a.inv_t + logf(s_rest), L),
              d_rest = lp_rest - t.log_rest;
  // (the logits' logs are formed once more for the gradient: nothing of an entry is kept)
  float kl = 0.f;
  each_entry(sh.id, a.K, lane, [&](int k) {
    const float x = sh.z[k] - m, d = log_share(x, a.inv_t, L) - sh.lq[k], q = sh.q[k],
                p = fast_exp2(x * c - L);
    kl += reverse ? kl_part(p, d, q) : kl_part(q, -d, p);
  });
  kl = wave_sum(kl);
  kl += reverse ? kl_part(p_rest, d_rest, t.q_rest) : kl_part(t.q_rest, -d_rest, p_rest);
  // (kl_part takes a NaN share for 0)
  if (!(total > 0.f && total < INFINITY) || !t.finite) kl = NAN;
  const float w = a.scale * weight;
  Student out;
  out.term = w == 0.f ? 0.f : w * kl;
  out.finite = isfinite(kl) && isfinite(out.term);
  out.rest = RestGrad{0.f, 0.f, 0.f};
  if (BWD) {
    const float cf = w / a.temperature, mant = __builtin_amdgcn_frexp_mantf(cf);
    const int up = __builtin_amdgcn_frexp_expf(cf);
    each_entry(sh.id, a.K, lane, [&](int k) {
      const float lp = log_share(sh.z[k] - m, a.inv_t, L);
      sh.grad[k] =
          E::bits_of(cf == 0.f ? 0.f : class_grad(reverse, lp, sh.lq[k], kl, mant, up));
    });
    out.rest = rest_grad(
        cf == 0.f ? 0.f : class_grad(reverse, lp_rest, t.log_rest, kl, mant, up), m_rest, s_rest);
  }
  return out;
}

// The row's results, by one thread.
__device__ __forceinline__ void put_row(const DistillArgs& a, int64_t row, float term, bool valid,
                                        bool bad, bool finite) {
  if (a.terms_user) a.terms_user[row] = term;
  a.terms_ws[row] = term;
  a.flags_ws[row] = (valid ? kFlagValid : 0) | (bad ? kFlagBadId : 0) |
                    (valid && !finite ? kFlagNonFinite : 0);
  a.logk_ws[row] = 0.f;
  a.excess_ws[row] = 0.f;
}

// The gradient of a vector of logits none of which is listed.
template <class E>
__device__ __forceinline__ u32x4 rest_vec(u32x4 z, float c, const RestGrad& g) {
  float f[E::kPerVec];
  E::unpack(z, f);
#pragma unroll
  for (int e = 0; e < E::kPerVec; ++e) f[e] = fast_exp2(__builtin_fmaf(f[e] - g.m, c, g.up)) * g.g;
  return E::pack(f);
}

}  // namespace cis
