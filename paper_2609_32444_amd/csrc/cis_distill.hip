// Distillation kernels (gfx950).
#include "cis_distill.h"

namespace cis {

// ------------------------------------------------------------------------------------------
// One workgroup per row. The list goes into a table in LDS, hashed by the 16-byte vector that a
// token lies in, with chains; a sweep looks every vector up (one LDS read), leaves the listed
// tokens out of its sum and notes their logits, and the gradient sweep puts theirs in.
// ------------------------------------------------------------------------------------------
constexpr int kDistillTable = 8192;
constexpr uint32_t kNone = 0xFFFFFFFFu;
struct DistillShared {
  uint32_t head[kDistillTable];
  uint32_t next[CIS_TOP_MAX_K];
  int32_t id[CIS_TOP_MAX_K];
  float z[CIS_TOP_MAX_K];        // the student's logits
  float lq[CIS_TOP_MAX_K];       // log q
  uint32_t grad[CIS_TOP_MAX_K];  // gradient, in the logits' format
  float f[16];
  u64 u[16];
};

template <class E, bool BWD>
__global__ __launch_bounds__(kTokBlock) void cis_distill_kernel(const DistillArgs a) {
  constexpr int BLOCK = kTokBlock, NW = BLOCK / 64, EPV = E::kPerVec;
  __shared__ DistillShared sh;
  const int tid = threadIdx.x;
  const int V = a.r.V, nvec = a.r.nvec, K = a.K;
  const float c = kLog2e / a.temperature;
  const bool reverse = a.reverse != 0, ragged = V % EPV != 0;
  for (int i = tid; i < kDistillTable; i += BLOCK) sh.head[i] = kNone;
  __syncthreads();
  auto sum = [&](float x) {
    const float s = block_sum<NW>(x, sh.f);
    __syncthreads();
    return s;
  };
  auto max = [&](float x) {
    const float m = block_max<NW>(x, sh.f);
    __syncthreads();
    return m;
  };
  for (int64_t row = blockIdx.x; row < a.r.T; row += gridDim.x) {
    const bool on = tok_on(a.r, row);
    const int32_t* ids = a.ids + row * a.ld_top;
    const float* values = a.values + row * a.ld_top;
    // the table
    u64 seen = 0;   // entries, and above them ids out of range or repeated
    if (on)
      for (int k = tid; k < K; k += BLOCK) {
        const int32_t id = ids[k];
        const bool in = id >= 0 && id < V;
        sh.id[k] = in ? id : -1;
        sh.next[k] = kNone;
        if (in) sh.next[k] = atomicExch(&sh.head[(id / EPV) & (kDistillTable - 1)], (uint32_t)k);
        seen += in ? 1 : id == -1 ? 0 : u64(1) << 32;
      }
    __syncthreads();
    if (on)
      for (int k = tid; k < K; k += BLOCK)
        if (sh.id[k] >= 0)
          for (uint32_t o = sh.next[k]; o != kNone; o = sh.next[o])
            if (sh.id[o] == sh.id[k]) seen += u64(1) << 32;
    seen = block_sum<NW>(seen, sh.u);
    const bool bad = (seen >> 32) != 0, valid = on && !bad && seen != 0;
    const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
    RestGrad g{INFINITY, 0u};
    float term = 0.f;
    bool nonfinite = false;
    if (valid) {
      // sweep 1: the tokens that are not listed
      float R = kMinExp, s = 0.f;
      for (int v = tid; v < nvec; v += BLOCK) {
        float f[EPV];
        tok_vec<E>(rs, v, V, f);
        for (uint32_t k = sh.head[v & (kDistillTable - 1)]; k != kNone; k = sh.next[k]) {
          const int id = sh.id[k];
          if (id / EPV != v) continue;
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (id % EPV == e) {
              sh.z[k] = f[e];
              f[e] = -INFINITY;
            }
        }
        float m = f[0];
#pragma unroll
        for (int e = 1; e < EPV; ++e) m = fmaxf(m, f[e]);
        const float Rn = fmaxf(R, m * c);
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < EPV; ++e) part += fast_exp2(__builtin_fmaf(f[e], c, -Rn));
        s = s * fast_exp2(R - Rn) + part;
        R = Rn;
      }
      const float Rr = max(R);
      float rest = sum(s * fast_exp2(R - Rr));
      // the list: the student's sums, and the teacher's
      float zm = -INFINITY, vm = -INFINITY;
      for (int k = tid; k < K; k += BLOCK)
        if (sh.id[k] >= 0) {
          zm = fmaxf(zm, sh.z[k]);
          vm = fmaxf(vm, values[k]);
        }
      const float Rs = fmaxf(Rr, max(zm) * c);
      rest *= fast_exp2(Rr - Rs);
      const float tail = a.tail ? a.tail[row] * kLog2e : -INFINITY;
      const float Rt = fmaxf(fmaxf(max(vm) * c, tail), kMinExp);
      float es = 0.f, et = 0.f;
      for (int k = tid; k < K; k += BLOCK)
        if (sh.id[k] >= 0) {
          es += fast_exp2(__builtin_fmaf(sh.z[k], c, -Rs));
          et += fast_exp2(__builtin_fmaf(values[k], c, -Rt));
        }
      es = sum(es);
      et = sum(et);
      const float tr = fast_exp2(tail - Rt);
      const float total = es + rest, ttotal = et + tr;
      const float Ls = log2f(total), Lt = log2f(ttotal);
      const float p_rest = rest / total, q_rest = tr / ttotal;
      const float d_rest = log_rest(es, rest) - log_rest(et, tr);
      auto lp_of = [&](int k) { return (__builtin_fmaf(sh.z[k], c, -Rs) - Ls) * kLn2; };
      auto lq_of = [&](int k) { return (__builtin_fmaf(values[k], c, -Rt) - Lt) * kLn2; };
      float kl = 0.f;
      for (int k = tid; k < K; k += BLOCK)
        if (sh.id[k] >= 0) {
          const float lp = lp_of(k), lq = lq_of(k), p = expf(lp), q = expf(lq);
          kl += reverse ? kl_part(p, lp - lq, q) : kl_part(q, lq - lp, p);
        }
      kl = sum(kl);
      kl += reverse ? kl_part(p_rest, d_rest, q_rest) : kl_part(q_rest, -d_rest, p_rest);
      // (kl_part takes a NaN share for 0)
      const bool sums = total > 0.f && total < INFINITY && ttotal > 0.f && ttotal < INFINITY;
      if (!sums) kl = NAN;
      const float w = a.scale * (a.weight ? a.weight[row] : 1.f);
      term = w == 0.f ? 0.f : w * kl;
      nonfinite = !(isfinite(kl) && isfinite(term));
      if (BWD) {
        const float cf = w / a.temperature;
        for (int k = tid; k < K; k += BLOCK)
          if (sh.id[k] >= 0) {
            const float lp = lp_of(k), lq = lq_of(k);
            const float x = cf == 0.f ? 0.f : cf * listed_grad(reverse, expf(lp), expf(lq), lp - lq, kl);
            sh.grad[k] = E::bits_of(x);
          }
        g = rest_grad(cf == 0.f ? 0.f : cf * others_grad(reverse, p_rest, q_rest, d_rest, kl), Rs,
                      total);
        __syncthreads();
      }
    }
    if (tid == 0) {
      if (a.terms_user) a.terms_user[row] = term;
      a.terms_ws[row] = term;
      a.flags_ws[row] = (valid ? kFlagValid : 0) | (on && bad ? kFlagBadId : 0) |
                        (nonfinite ? kFlagNonFinite : 0);
      a.logk_ws[row] = 0.f;
      a.excess_ws[row] = 0.f;
    }
    if (BWD) {
      void* grow = (char*)a.dlogits + row * a.grow_bytes;
      const __amdgpu_buffer_rsrc_t ws = make_rsrc(grow, (uint32_t)(nvec - (ragged ? 1 : 0)) * 16u);
      const uint32_t sgn = g.neg ? E::kSignMask : 0u;
      for (int v = tid; v < nvec; v += BLOCK) {
        u32x4 out{0u, 0u, 0u, 0u};
        if (valid) {
          float f[EPV];
          tok_vec<E>(rs, v, V, f);
#pragma unroll
          for (int e = 0; e < EPV; ++e) f[e] = fast_exp2(__builtin_fmaf(f[e], c, -g.b2));
          out = E::pack(f) ^ u32x4{sgn, sgn, sgn, sgn};
          for (uint32_t k = sh.head[v & (kDistillTable - 1)]; k != kNone; k = sh.next[k])
            if (sh.id[k] / EPV == v) out = E::set(out, sh.id[k] % EPV, sh.grad[k]);
        }
        bstore(out, ws, (uint32_t)v * 16u, 0u);
        if (ragged && v == nvec - 1)
          for (int e = 0; e < V - v * EPV; ++e) E::store_elem(grow, v * EPV + e, E::elem_bits(out, e));
      }
      __syncthreads();
    }
    if (on)
      for (int k = tid; k < K; k += BLOCK)
        if (sh.id[k] >= 0) sh.head[(sh.id[k] / EPV) & (kDistillTable - 1)] = kNone;
    __syncthreads();
  }
}

const void* distill_kernel(int dtype, bool bwd) {
  if (dtype == CIS_BF16)
    return bwd ? (const void*)&cis_distill_kernel<Bf16, true>
               : (const void*)&cis_distill_kernel<Bf16, false>;
  return bwd ? (const void*)&cis_distill_kernel<F32, true>
             : (const void*)&cis_distill_kernel<F32, false>;
}

}  // namespace cis
