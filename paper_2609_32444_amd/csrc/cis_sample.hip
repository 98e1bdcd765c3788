// Sampling kernels (gfx950): one workgroup per row, which it reads as often as its cuts take.
#include "cis_tok_row.h"

namespace cis {

// ------------------------------------------------------------------------------------------
// One token per row. The cuts give one pair (key, ties); the draw sums the kept weights in pieces
// of the row in order of the ids, finds the piece that the random number falls into and then the
// token, all in whole numbers.
// ------------------------------------------------------------------------------------------
struct SampleShared {
  CutShared cut;
  float f[16];
  u64 u[16];
  double d[16];
  u64 mass[kChunks];
  uint32_t ties[kChunks];
};

template <class E>
__global__ __launch_bounds__(kTokBlock) void cis_sample_kernel(const SampleArgs a) {
  constexpr int BLOCK = kTokBlock, NW = BLOCK / 64, EPV = E::kPerVec;
  __shared__ SampleShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int V = a.r.V, nvec = a.r.nvec;
  for (int64_t row = blockIdx.x; row < a.r.T; row += gridDim.x) {
    const float u = a.u[row];
    const float temp = a.temperature ? a.temperature[row] : a.prm.temperature;
    const int top_k = a.top_k ? a.top_k[row] : a.prm.top_k;
    const float top_p = a.top_p ? a.top_p[row] : a.prm.top_p;
    const float min_p = a.min_p ? a.min_p[row] : a.prm.min_p;
    bool draw = tok_on(a.r, row) && u >= 0.f && u < 1.f && temp >= 0.f && temp < INFINITY &&
                top_k >= 0 && top_p > 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f;
    const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
    RowFacts facts{};
    if (draw) {
      facts = row_facts<E, BLOCK>(rs, nvec, V, sh.f, sh.u);
      draw = facts.finite && facts.tokens > 0;
    }
    if (!draw) {
      if (tid == 0) {
        a.ids[row] = -1;
        if (a.logp) a.logp[row] = 0.f;
        if (a.logp_kept) a.logp_kept[row] = 0.f;
      }
      continue;
    }
    const float M = facts.M;
    float c = kLog2e / temp;
    u64 k = top_k > 0 ? (u64)top_k : facts.tokens;
    if (!(c < INFINITY)) {   // greedy
      c = kLog2e;
      k = 1;
    }
    Cut cut{kNoToken, 0};    // keeps every token
    auto weight = [&](float f) { return draw_weight(f, M, c); };
    if (k < facts.tokens)
      cut = radix_cut<E, BLOCK>(rs, nvec, V, k, 0u, [](float) { return 1u; }, sh.cut);
    if (top_p < 1.f && k > 1) {
      u64 s = 0;
      for (int v = tid; v < nvec; v += BLOCK) {
        float f[EPV];
        tok_vec<E>(rs, v, V, f);
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (order_key(f[e]) > cut.key) s += weight(f[e]);
      }
      s = block_sum<NW>(s, sh.u);
      if (cut.ties > 0) s += cut.ties * weight(key_value(cut.key));
      const double want = ceil((double)top_p * (double)s);
      const Cut p = radix_cut<E, BLOCK>(rs, nvec, V, (u64)want, cut.key, weight, sh.cut);
      // the sum that the key's tokens have to bring, as a count of them
      const u64 w = weight(key_value(p.key));
      if (w > 0) cut = Cut{p.key, (p.ties + w - 1) / w};
    }
    const uint32_t least_w = (uint32_t)ceil((double)min_p * kDrawOne);
    // the kept weights by pieces
    const int cv = chunk_vecs(nvec);
    for (int ch = wid; ch < kChunks; ch += NW) {
      u64 s = 0;
      uint32_t t = 0;
      for (int v = ch * cv + lane; v < min((ch + 1) * cv, nvec); v += 64) {
        float f[EPV];
        tok_vec<E>(rs, v, V, f);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const uint32_t key = order_key(f[e]);
          if (key > cut.key) {
            const uint32_t w = weight(f[e]);
            s += w >= least_w ? w : 0;
          }
          t += key == cut.key ? 1 : 0;
        }
      }
      s = wave_sum(s);
      t = wave_sum(t);
      if (lane == 0) {
        sh.mass[ch] = s;
        sh.ties[ch] = t;
      }
    }
    // the row's own log-sum-exp, relative to the largest logit and without its term (one of them,
    // where there are several): the sums keep what is left of a confident row to full accuracy
    double rest = 0.0;
    u64 largest = 0;
    for (int v = tid; v < nvec; v += BLOCK) {
      float f[EPV], s = 0.f;
      tok_vec<E>(rs, v, V, f);
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        s += f[e] == M ? 0.f : fast_exp2((f[e] - M) * kLog2e);
        largest += f[e] == M ? 1 : 0;
      }
      rest += s;
    }
    rest = block_sum<NW>(rest, sh.d) + (double)(block_sum<NW>(largest, sh.u) - 1);
    if (wid == 0) {
      uint32_t wt = cut.ties > 0 ? weight(key_value(cut.key)) : 0;
      if (wt < least_w) wt = 0;
      // piece 4 l + i of lane l
      u64 ties[4], mass[4], nt = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) nt += ties[i] = sh.ties[4 * lane + i];
      u64 tb = wave_scan(nt, lane) - nt, s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u64 left = cut.ties > tb ? cut.ties - tb : 0;
        mass[i] = sh.mass[4 * lane + i] + (ties[i] < left ? ties[i] : left) * wt;
        tb += ties[i];
        s += mass[i];
      }
      const u64 upto = wave_scan(s, lane), N = __shfl(upto, 63, 64);
      u64 at = (u64)((double)u * (double)N);
      if (at >= N) at = N - 1;
      const int who = __ffsll(__ballot(upto > at)) - 1;
      // the piece, what is before it, and the ties before it
      u64 before = upto - s, tbefore = wave_scan(nt, lane) - nt;
      int ch = 4 * lane;
      for (int i = 0; i < 3 && before + mass[i] <= at; ++i) {
        before += mass[i];
        tbefore += ties[i];
        ++ch;
      }
      ch = __shfl(ch, who, 64);
      before = __shfl(before, who, 64);
      tbefore = __shfl(tbefore, who, 64);
      for (int v0 = ch * cv; v0 < nvec; v0 += 64) {
        const int v = v0 + lane;
        float f[EPV];
        if (v < nvec) {
          tok_vec<E>(rs, v, V, f);
        } else {
          for (int e = 0; e < EPV; ++e) f[e] = -INFINITY;
        }
        uint32_t nt = 0;
        for (int e = 0; e < EPV; ++e) nt += order_key(f[e]) == cut.key ? 1 : 0;
        const u64 tupto = tbefore + wave_scan(nt, lane);
        u64 w[EPV], sum = 0, t = tupto - nt;
        for (int e = 0; e < EPV; ++e) {
          const uint32_t key = order_key(f[e]), q = weight(f[e]);
          w[e] = key > cut.key && q >= least_w ? q : 0;
          if (key == cut.key) w[e] = t++ < cut.ties ? wt : 0;
          sum += w[e];
        }
        const u64 supto = before + wave_scan(sum, lane);
        const u64 hit = __ballot(supto > at);
        if (hit) {
          if (lane == __ffsll(hit) - 1) {
            u64 b = supto - sum;
            int e = 0;
            while (b + w[e] <= at) b += w[e++];
            float fy = f[0];
            u64 wy = w[0];
#pragma unroll
            for (int i = 1; i < EPV; ++i) {
              fy = i == e ? f[i] : fy;
              wy = i == e ? w[i] : wy;
            }
            a.ids[row] = (int64_t)v * EPV + e;
            if (a.logp) a.logp[row] = (fy - M) - log1pf((float)rest);
            if (a.logp_kept) a.logp_kept[row] = (float)log((double)wy / (double)N);
          }
          break;
        }
        before = __shfl(supto, 63, 64);
        tbefore = __shfl(tupto, 63, 64);
      }
    }
    __syncthreads();
  }
}

const void* sample_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_sample_kernel<Bf16>
                           : (const void*)&cis_sample_kernel<F32>;
}

}  // namespace cis
