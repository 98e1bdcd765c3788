// Sampling kernels (gfx950).
//
// A row is drawn from the scan (TokScan) in one of four ways, by what its cuts keep at most:
//   * top_k up to kDrawK (and greedy rows): the candidates that RowSelect collects, put in order; the
//     cuts and the draw run on that list.
//   * nothing but min_p cuts: the weights' sums by chunks (cis_weigh_kernel), the chunk that the
//     random number falls into, and the token within it.
//   * top_p without a count: a histogram of the weights over the whole row (cis_hist_kernel) gives the
//     target and the step of 1/64 octave that the cut falls into; cis_weigh_kernel sums up what lies
//     above it and lists the step's tokens, which are put in order here.
//   * otherwise (top_k beyond kDrawK, or a step of more tokens than a list holds) one workgroup makes
//     such a histogram, of the counts too, in passes over the row, sorts the tokens of the step, and
//     sums up by chunks what is kept. Where a step overflows the list (many equal logits), the cut
//     is found byte by byte (radix_cut).
#include "cis_select.h"

namespace cis {

struct RowParams {
  float u, temp, top_p, min_p;
  int64_t top_k;   // V: no limit
  float c;
  bool ok;
  bool counted;    // top_k (V: all of a short row) leaves few enough for a list
  uint32_t least_w;
};
__device__ __forceinline__ RowParams row_params(const SampleArgs& a, int64_t row) {
  RowParams p;
  p.u = sload(a.u + row);
  p.temp = a.temperature ? sload(a.temperature + row) : a.prm.temperature;
  const int k = a.top_k ? sload(a.top_k + row) : a.prm.top_k;
  p.top_p = a.top_p ? sload(a.top_p + row) : a.prm.top_p;
  p.min_p = a.min_p ? sload(a.min_p + row) : a.prm.min_p;
  p.ok = tok_on(a.r, row) && p.u >= 0.f && p.u < 1.f && p.temp >= 0.f && p.temp < INFINITY &&
         k >= 0 && p.top_p > 0.f && p.top_p <= 1.f && p.min_p >= 0.f && p.min_p <= 1.f;
  p.c = kLog2e / p.temp;
  const bool greedy = !(p.c < INFINITY);
  p.top_k = greedy ? 1 : k == 0 || k >= a.r.V ? a.r.V : k;
  if (greedy) p.c = kLog2e;
  p.counted = greedy || (p.top_k <= kDrawK && (p.top_k < a.r.V || p.top_p < 1.f));
  p.least_w = (uint32_t)ceil((double)p.min_p * kDrawOne);
  return p;
}
// Rows that cis_weigh_kernel sums up: those that no count cuts. (The draw adds up the kept part of
// a step by chunks at WideShared::mass.)
__device__ __forceinline__ bool row_stepped(const RowParams& p, const SampleArgs& a) {
  return p.ok && !p.counted && p.top_k == a.r.V && p.top_p < 1.f && a.s.nch <= kFineSteps;
}
__device__ __forceinline__ bool row_weighed(const RowParams& p, const SampleArgs& a) {
  return row_stepped(p, a) || (p.ok && !p.counted && p.top_k == a.r.V && p.top_p == 1.f);
}

// A logit's exponent, and the step of the histogram of weights that it falls into: steps rise as
// logits fall; kFineSteps: no weight.
__device__ __forceinline__ float draw_exponent(float f, float M, float c) { return (f - M) * c; }
__device__ __forceinline__ int draw_step(float e) {
  const float t = e * -(float)kFine;
  return t < (float)kFineSteps ? (int)t : kFineSteps;
}
__device__ __forceinline__ uint32_t exponent_weight(float e) {
  return (uint32_t)(fast_exp2(e) * (float)kDrawOne);
}
// A row's largest logit, by one wave. (-inf: no token.)
__device__ __forceinline__ float row_max(const float* cmax, int nch, int lane) {
  float M = -INFINITY;
  for (int i = lane; i < nch; i += 64) M = fmaxf(M, cmax[i]);
  return wave_max(M);
}

// The first step at which the sum of mass[] reaches top_p of the whole, by one wave.
__device__ __forceinline__ DrawStep step_of_cut(const u64* mass, float top_p, int lane) {
  constexpr int S = kFineSteps / 64;
  static_assert(kFineSteps % 64 == 0 && S <= 64, "a lane has the same number of steps");
  u64 s = 0;
#pragma unroll
  for (int i = 0; i < S; ++i) s += mass[lane * S + i];
  const u64 upto = wave_scan(s, lane), total = __shfl(upto, 63, 64);
  const u64 want = (u64)ceil((double)top_p * (double)total);
  const u64 who = __ballot(upto >= want);
  DrawStep d{0, kFineSteps, 0};
  if (total == 0) return d;   // (a row without weights)
  const int at = __ffsll(who) - 1;   // the first lane that reaches it has the step
  const u64 before = __shfl(upto - s, at, 64);
  const u64 m = lane < S ? mass[at * S + lane] : 0, to = before + wave_scan(m, lane);
  const int in = __ffsll((u64)__ballot(to >= want)) - 1;
  d.step = at * S + in;
  d.left = want - __shfl(to - m, in, 64);
  return d;
}

// ------------------------------------------------------------------------------------------
// The histogram of a row's weights by their exponents, in a part of the row's chunks per workgroup:
// whole numbers in LDS, so that the order of the additions is of no account. Where a row has one
// workgroup, the step of its cut too. Tokens that the cut cannot reach are added up in registers: at
// most V of them have a weight of `lowest` each, and the whole sum is that of the chunks' largest
// logits at least, so that they stay below 1 - top_p of it. Bound by the arithmetic (exp2 takes four
// times as long as the others) and the atomics: 256 rows of V = 262144 in 30 us, 37 with every
// token in LDS.
// ------------------------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(kHistBlock) void cis_hist_kernel(const SampleArgs a) {
  constexpr int NW = kHistBlock / 64, EPV = E::kPerVec;
  __shared__ u64 mass[kFineSteps];
  const int tid = threadIdx.x, lane = tid & 63,
            wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
  const int64_t at = blockIdx.x / a.parts, row = a.row0 + at;
  const int part = (int)(blockIdx.x - at * a.parts), nch = a.s.nch;
  const RowParams p = row_params(a, row);
  if (!row_stepped(p, a)) return;
  for (int i = tid; i < kFineSteps; i += kHistBlock) mass[i] = 0;
  const float* cmax = a.s.cmax + row * nch;
  const float M = row_max(cmax, nch, lane);
  const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
  float least = 0.f;
  for (int i = lane; i < nch; i += 64) least += fast_exp2(draw_exponent(cmax[i], M, p.c));
  least = 0.99f * wave_sum(least);
  const float octaves = log2f((float)a.r.V / ((1.f - p.top_p) * least)),
              lowest = octaves < 29.f ? ceilf(octaves * kFine) * (-1.f / kFine) : -29.f;
  u64 rest = 0;
  __syncthreads();
  for (int ch = part * NW + wid; ch < nch; ch += a.parts * NW) {
    if (!(draw_exponent(cmax[ch], M, p.c) >= -28.f)) continue;
    u32x4 x[kScanSlots];
    load_chunk<E, 0>(rs, a.r, ch, lane, x);
    static_for<kScanSlots>([&](auto I) {
      float f[EPV];
      E::unpack(x[I], f);
      uint32_t vs = 0;   // (8 weights stay below 2^32)
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const float t = draw_exponent(f[e], M, p.c);
        const uint32_t q = exponent_weight(t);
        if (t > lowest)
          atomicAdd(&mass[(int)(t * -(float)kFine)], (u64)q);
        else
          vs += q;
      }
      rest += vs;
      slot_fence();
    });
  }
  rest = wave_sum(rest);
  if (lane == 0 && rest) atomicAdd(&mass[kFineSteps - 1], rest);
  __syncthreads();
  if (a.parts == 1) {
    if (tid < 64) {
      const DrawStep d = step_of_cut(mass, p.top_p, lane);
      if (lane == 0) a.steps[at] = d;
    }
  } else {
    u64* out = a.hist + (int64_t)blockIdx.x * kFineSteps;
    for (int i = tid; i < kFineSteps; i += kHistBlock) out[i] = mass[i];
  }
}

// The step of a row's cut from its parts' histograms.
__global__ __launch_bounds__(kHistBlock) void cis_step_kernel(const SampleArgs a) {
  __shared__ u64 mass[kFineSteps];
  const int64_t at = blockIdx.x, row = a.row0 + at;
  const RowParams p = row_params(a, row);
  if (!row_stepped(p, a)) return;
  const u64* in = a.hist + at * a.parts * kFineSteps;
  for (int i = threadIdx.x; i < kFineSteps; i += kHistBlock) {
    u64 s = 0;
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) s += in[k * kFineSteps + i];
    mass[i] = s;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const DrawStep d = step_of_cut(mass, p.top_p, threadIdx.x);
    if (threadIdx.x == 0) a.steps[at] = d;
  }
}

// ------------------------------------------------------------------------------------------
// A wave's chunks one after the other, of one row in a workgroup: the sum of their weights, of a row
// that top_p cuts those above the step of the cut, whose tokens are listed. A chunk whose largest logit
// does not reach that far is not read. Without STEP, no row is cut by top_p. Bound by some 10
// instructions a logit (24 us) and the second read of the row: 512 rows of V = 151936 in 32 us; with
// STEP 256 rows of V = 262144, half of them peaked, in 21.
// ------------------------------------------------------------------------------------------
template <class E, bool STEP>
__global__ __launch_bounds__(kWeighBlock) void cis_weigh_kernel(const SampleArgs a) {
  constexpr int NW = kWeighBlock / 64, EPV = E::kPerVec;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6, nch = a.s.nch;
  const uint32_t at = blockIdx.x / (uint32_t)a.weigh_parts;
  const int part = (int)(blockIdx.x - at * (uint32_t)a.weigh_parts);
  const int64_t row = a.row0 + at;
  const RowParams p = row_params(a, row);
  if (!row_weighed(p, a)) return;
  const float* cmax = a.s.cmax + row * nch;
  const float M = row_max(cmax, nch, threadIdx.x & 63);
  const int step = STEP && p.top_p < 1.f ? sload(&a.steps[at].step) : kFineSteps;
  // exponents above the step, and in it (multiples of 1 / kFine: exact)
  const float above = step * (-1.f / kFine), within = (step + 1) * (-1.f / kFine);
  for (int ch = part * NW + wid; ch < nch; ch += a.weigh_parts * NW) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // (else what follows from it is kept for all chunks)
    const float top = draw_exponent(cmax[ch], M, p.c);
    u64 s = 0;
    if (top >= -28.f && draw_step(top) <= step) {
      u32x4 x[kScanSlots];
      load_chunk<E, 0>(tok_rsrc(a.r, row), a.r, ch, lane, x);
      // which of the lane's tokens are in the step: a bit each, of 4 vectors to a word, the first
      // token's highest
      constexpr int kBits = 4 * EPV;
      static_assert(kScanSlots == 8, "two words");
      uint32_t in[2] = {0, 0};
      static_for<kScanSlots>([&](auto I) {
        float f[EPV];
        E::unpack(x[I], f);
        uint32_t vs = 0;   // (8 weights stay below 2^32)
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          const float t = draw_exponent(f[e], M, p.c);
          const uint32_t q = exponent_weight(t);
          if (STEP) in[I / 4] = in[I / 4] * 2 + (t > within && t <= above ? 1 : 0);
          vs += (!STEP || t > above) && q >= p.least_w ? q : 0u;
        }
        s += vs;
        if (STEP) asm volatile("" : "+v"(in[I / 4]));   // (else all vectors are unpacked first)
        slot_fence();
      });
      s = wave_sum(s);
      if (STEP && step < kFineSteps && __ballot((in[0] | in[1]) != 0)) {
        const uint32_t mine = __popc(in[0]) + __popc(in[1]), upto = wave_scan(mine, lane);
        uint32_t to = 0;
        if (lane == 63) to = atomicAdd(&a.steps[at].count, upto);
        to = __builtin_amdgcn_readlane(to, 63) + upto - mine;
        uint32_t* ids = a.step_ids + (int64_t)at * a.step_ld;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          for (uint32_t left = in[h]; left;) {
            const int b = 31 - __clz(left), k = kBits - 1 - b;
            left &= ~(1u << b);
            if (to < (uint32_t)a.step_ld)
              ids[to] = (uint32_t)((ch * kScanVecs + (h * 4 + k / EPV) * 64 + lane) * EPV + k % EPV);
            ++to;
          }
      }
    }
    if (lane == 0) a.draw[row * nch + ch] = s;
  }
}

// ------------------------------------------------------------------------------------------
// The draw, by one workgroup per row. Bound by the latency of its steps, each of which waits for the
// one before: a top-k list of one row 16 us (26 barriers), 512 uncut rows 9 us, 256 rows with a step of
// top_p 14 us.
// ------------------------------------------------------------------------------------------
struct WideShared {
  u64 mass[kFineSteps];
  uint32_t count[kFineSteps];
  uint32_t step;
  u64 left;
};

template <class E, int BLOCK, int LIST, bool WIDE>
struct RowDraw {
  static constexpr int NW = BLOCK / 64, EPV = E::kPerVec;
  const SampleArgs& a;
  const RowParams& p;
  RowSelect<E, BLOCK, LIST>& sel;
  SelectShared<LIST>& sh;
  int64_t row;
  float rest;   // sum of exp(z - M) over the row but one of its largest logits
  u64 mass0;    // the sum of chunk `lane`, asked for ahead of what comes before its use

  __device__ __forceinline__ uint32_t weight(float f) const { return draw_weight(f, sel.M, p.c); }

  __device__ __forceinline__ void put_row(int id, float f, u64 w, u64 N) const {
    a.ids[row] = id;
    if (a.logp) a.logp[row] = (f - sel.M) - log1pf(rest);
    if (a.logp_kept) a.logp_kept[row] = (float)log((double)w / (double)N);
  }

  // f(logits of vector v, v) for a thread's vectors of chunk ch, which follow each other.
  static constexpr int kChunkVecs = kScanVecs < BLOCK ? 1 : kScanVecs / BLOCK;
  template <class F>
  __device__ __forceinline__ void each_in_chunk(int ch, F&& f) const {
    const int v0 = threadIdx.x * kChunkVecs;
    if (v0 >= kScanVecs) return;
    u32x4 x[kChunkVecs];
    static_for<kChunkVecs>([&](auto J) {
      x[J] = bload_aux<0>(sel.rs, (uint32_t)(ch * kScanVecs + v0 + J) * 16u);
    });
    static_for<kChunkVecs>([&](auto J) {
      const int v = ch * kScanVecs + v0 + J;
      float l[EPV];
      E::unpack(x[J], l);
      if ((v + 1) * EPV > sel.V) mask_past_end<E>(l, v, sel.V);
      f(l, v);
    });
  }

  // Sum over the row but one largest logit, relative to it: the chunks' sums, except for the
  // first chunk that holds it, which is summed again without it.
  __device__ __forceinline__ void sum_rest() {
    const int tid = threadIdx.x, lane = tid & 63;
    int first = sel.nch;
    double s = 0.0;
    auto each = [&](auto&& f) {   // f(chunk, its largest logit, its sum)
      if (tid < sel.nch) f(tid, sel.cmax0, sel.csum0);
      for (int i = BLOCK + tid; i < sel.nch; i += BLOCK) f(i, sel.cmax[i], sel.csum[i]);
    };
    each([&](int i, float m, double) {
      if (m == sel.M) first = first < i ? first : i;
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      const int o = __shfl_xor(first, off, 64);
      first = first < o ? first : o;
    }
    if (lane == 0) sh.u[tid >> 6] = (u64)first;
    __syncthreads();
    for (int w = 0; w < NW; ++w) first = first < (int)sh.u[w] ? first : (int)sh.u[w];
    each([&](int i, float m, double sum) {
      if (i != first) s += sum * (double)fast_exp2((m - sel.M) * kLog2e);
    });
    u64 n = 0;   // largest ones in the chunk (counted apart: 1 would swallow what is far smaller)
    each_in_chunk(first, [&](const float (&f)[EPV], int) {
      float t = 0.f;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        t += f[e] == sel.M ? 0.f : fast_exp2((f[e] - sel.M) * kLog2e);
        n += f[e] == sel.M ? 1 : 0;
      }
      s += (double)t;
    });
    __syncthreads();
    n = block_sum<NW>(n, sh.u);
    if (tid == 0) s += (double)(n - 1);
    rest = (float)block_sum<NW>(s, sh.d);
  }

  // Draws from the list's first logits in order: at most `n` of them; of those the fewest that
  // reach `want` (0: all), at least least_w each.
  __device__ __forceinline__ void from_list(int n, u64 want) {
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    constexpr int PT = LIST / BLOCK;
    u64 t[PT];
    uint32_t q[PT];
    u64 s = 0;
    static_for<PT>([&](auto J) {
      const int i = tid * PT + J;
      q[J] = 0;
      if (i < n) {
        t[J] = sh.list[i];
        q[J] = weight(token_value(t[J]));
      }
      s += q[J];
    });
    u64 before = wave_scan(s, lane);
    if (lane == 63) sh.u[wid] = before;
    __syncthreads();
    before -= s;
    u64 total = 0;
    for (int w = 0; w < NW; ++w) {
      if (w < wid) before += sh.u[w];
      total += sh.u[w];
    }
    if (p.top_p < 1.f && want == 0) want = (u64)ceil((double)p.top_p * (double)total);
    // the cuts: each keeps a first part
    u64 keep = 0;   // by top_p, and above by min_p
    u64 b = before;
    static_for<PT>([&](auto J) {
      if (tid * PT + J < n) {
        keep += want == 0 || b < want ? 1 : 0;
        keep += q[J] >= p.least_w ? u64(1) << 32 : 0;
      }
      b += q[J];
    });
    __syncthreads();
    keep = block_sum<NW>(keep, sh.u);
    const int np = (int)(uint32_t)keep, nm = (int)(keep >> 32);
    n = n < np ? n : np;
    n = n < nm ? n : nm;
    s = 0;
    static_for<PT>([&](auto J) {
      if (tid * PT + J >= n) q[J] = 0;
      s += q[J];
    });
    __syncthreads();
    const u64 N = block_sum<NW>(s, sh.u);
    u64 at = (u64)((double)p.u * (double)N);
    if (at >= N) at = N - 1;
    // in order of the ids: (id, weight) pairs
    static_for<PT>([&](auto J) {
      const int i = tid * PT + J;
      if (i < n) sh.list[i] = ((u64)(uint32_t)token_id(t[J]) << 32) | q[J];
    });
    __syncthreads();
    if (n > 256) {
      // narrowed to the tokens that share the first bits of the drawn one's id
      int shift = 0;
      while ((sel.V - 1) >> shift >= kSteps) ++shift;
      for (int i = tid; i < kSteps; i += BLOCK) sh.mass[i] = 0;
      if (tid == 0) sh.count = 0;
      __syncthreads();
      static_for<PT>([&](auto J) {
        if (tid * PT + J < n) atomicAdd(&sh.mass[token_id(t[J]) >> shift], (u64)q[J]);
      });
      __syncthreads();
      constexpr int S = kSteps / BLOCK;
      u64 m[S], ms = 0;
      static_for<S>([&](auto J) { ms += m[J] = sh.mass[tid * S + J]; });
      u64 mb = wave_scan(ms, lane);
      if (lane == 63) sh.u[wid] = mb;
      __syncthreads();
      mb -= ms;
      for (int w = 0; w < wid; ++w) mb += sh.u[w];
      static_for<S>([&](auto J) {
        if (mb <= at && at < mb + m[J]) {
          sh.bin = tid * S + J;
          sh.mass[0] = mb;   // (every thread has read its own)
        }
        mb += m[J];
      });
      __syncthreads();
      const uint32_t bin = sh.bin;
      at -= sh.mass[0];
      static_for<PT>([&](auto J) {
        if (tid * PT + J < n && (uint32_t)(token_id(t[J]) >> shift) == bin)
          sh.list[atomicAdd(&sh.count, 1u)] = ((u64)(uint32_t)token_id(t[J]) << 32) | q[J];
      });
      __syncthreads();
      n = (int)sh.count;
    }
    for (int i = tid; i < n; i += BLOCK) {
      const u64 me = sh.list[i];
      u64 upto = 0;
      for (int j = 0; j < n; ++j) {
        const u64 x = sh.list[j];
        upto += x <= me ? (uint32_t)x : 0;   // ids differ: lower ids first
      }
      const uint32_t w = (uint32_t)me;
      if (upto > at && upto - w <= at) {
        // its logit: from the row (the list holds it no more)
        const int id = (int)(me >> 32);
        float f[EPV], fy = 0.f;
        tok_vec<E>(sel.rs, id / EPV, sel.V, f);
#pragma unroll
        for (int e = 0; e < EPV; ++e) fy = id % EPV == e ? f[e] : fy;
        put_row(id, fy, w, N);
      }
    }
  }

  // Draws by the chunks' sums at a.draw, with `ties` (null: none) tokens of the cut's key per
  // chunk of which the row's first cut.ties count.
  __device__ __forceinline__ void from_chunks(const Cut& cut, const uint32_t* ties, uint32_t least) {
    const int tid = threadIdx.x, lane = tid & 63;
    const u64* mass = a.draw + row * sel.nch;
    uint32_t wt = ties && cut.ties > 0 ? weight(key_value(cut.key)) : 0;
    if (wt < least) wt = 0;
    __syncthreads();
    if (tid < 64) {
      // (chunk i0 + lane's kept mass, and the ties up to it)
      auto chunk_mass = [&](int i0, u64& tb, u64& nt) {
        const int i = i0 + lane;
        nt = ties && i < sel.nch ? ties[i] : 0;
        const u64 upto = tb + (ties ? wave_scan(nt, lane) : 0), b = upto - nt;
        const u64 left = cut.ties > b ? cut.ties - b : 0;
        if (ties) tb = __shfl(upto, 63, 64);
        return (i >= sel.nch ? 0 : ties || i0 > 0 ? mass[i] : mass0) + (nt < left ? nt : left) * wt;
      };
      Place at{0, 0, 0, 0, 0};
      u64 tb = 0, nt;
      for (int i0 = 0; i0 < sel.nch; i0 += 64) at.N += wave_sum(chunk_mass(i0, tb, nt));
      at.to = (u64)((double)p.u * (double)at.N);
      if (at.to >= at.N) at.to = at.N - 1;
      tb = 0;
      for (int i0 = 0; i0 < sel.nch; i0 += 64) {
        const u64 tb0 = tb, m = chunk_mass(i0, tb, nt), upto = at.before + wave_scan(m, lane);
        const u64 hit = __ballot(upto > at.to);
        if (hit) {
          const int who = __ffsll(hit) - 1;
          at.ch = i0 + who;
          at.before = __shfl(upto - m, who, 64);
          at.tb = ties ? tb0 + __shfl(wave_scan(nt, lane) - nt, who, 64) : 0;
          break;
        }
        at.before = __shfl(upto, 63, 64);
      }
      if (lane == 0) put_place(at);
    }
    auto above = [&](float f, int) {
      const uint32_t q = weight(f);
      return order_key(f) > cut.key && q >= least ? q : 0u;
    };
    if (ties)
      in_chunk<true>(above, cut, wt);
    else
      in_chunk<false>(above, cut, 0);
  }

  // What the first wave found: the chunk, the sum ahead of it, the draw, the whole sum, and the ties
  // ahead of the chunk.
  struct Place {
    u64 ch, before, to, N, tb;
  };
  __device__ __forceinline__ void put_place(const Place& p) const {
    sh.u[0] = p.ch;
    sh.u[1] = p.before;
    sh.u[2] = p.to;
    sh.u[3] = p.N;
    sh.u[4] = p.tb;
  }

  // Sum over the threads ahead of this one; `u` may be used again after the next barrier.
  __device__ __forceinline__ u64 ahead(u64 x, u64* u) const {
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
    const u64 upto = wave_scan(x, lane);
    if (lane == 63) u[wid] = upto;
    __syncthreads();
    u64 b = upto - x;
    for (int w = 0; w < wid; ++w) b += u[w];
    return b;
  }

  // Draws within a chunk, at put_place's values: weights kept(logit, id) of the tokens. With TIES,
  // tokens of the cut's key weigh wt (kept() gives them 0) as long as they are among its first
  // cut.ties.
  template <bool TIES, class W>
  __device__ __forceinline__ void in_chunk(W&& kept, const Cut& cut, uint32_t wt) const {
    __syncthreads();
    const int ch = (int)sh.u[0];
    const u64 to = sh.u[2], N = sh.u[3];
    u64 before = sh.u[1], t = sh.u[4];
    uint32_t w[kChunkVecs][EPV];
    float l[kChunkVecs][EPV];
    u64 n = 0, sum = 0;
    int j = 0;
    static_for<kChunkVecs>([&](auto J) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) w[J][e] = 0;
    });
    const int v0 = ch * kScanVecs + threadIdx.x * kChunkVecs;
    each_in_chunk(ch, [&](const float (&f)[EPV], int v) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const uint32_t q = kept(f[e], v * EPV + e);
        const bool tie = TIES && order_key(f[e]) == cut.key;
        static_for<kChunkVecs>([&](auto J) {
          if (j == J) {
            w[J][e] = q;
            l[J][e] = f[e];
          }
        });
        n += tie ? 1 : 0;
        sum += q;
      }
      ++j;
    });
    if (TIES) {
      __syncthreads();   // (every thread has read its own)
      t += ahead(n, sh.u);
      static_for<kChunkVecs>([&](auto J) {
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (threadIdx.x * kChunkVecs < kScanVecs && order_key(l[J][e]) == cut.key) {
            w[J][e] = t++ < cut.ties ? wt : 0;
            sum += w[J][e];
          }
      });
    }
    __syncthreads();
    before += ahead(sum, sh.u);
    if (before <= to && to < before + sum) {
      bool found = false;
      static_for<kChunkVecs>([&](auto J) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          if (!found && before + w[J][e] > to) {
            found = true;
            put_row((v0 + J) * EPV + e, l[J][e], w[J][e], N);
          }
          before += w[J][e];
        }
      });
    }
  }

  __device__ __forceinline__ int fine_step(float f) const {
    return draw_step(draw_exponent(f, sel.M, p.c));
  }

  // f(logits of vector v, v) for the row's chunks that hold a weight, whole waves together; then
  // end(chunk), of the others too.
  template <class F, class G>
  __device__ __forceinline__ void each_chunk(F&& f, G&& end) const {
    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
    constexpr int U = 4;   // loads in flight (8: the float32 kernels spill)
    for (int ch = wid; ch < sel.nch; ch += NW) {
      if (draw_exponent(sel.cmax[ch], sel.M, p.c) >= -28.f)
#pragma unroll 1
        for (int v0 = ch * kScanVecs + lane; v0 < (ch + 1) * kScanVecs; v0 += U * 64) {
          u32x4 x[U];
          static_for<U>([&](auto I) { x[I] = bload_aux<0>(sel.rs, (uint32_t)(v0 + I * 64) * 16u); });
          static_for<U>([&](auto I) {
            const int v = v0 + I * 64;
            float l[EPV];
            E::unpack(x[I], l);
            if ((v + 1) * EPV > sel.V) mask_past_end<E>(l, v, sel.V);
            f(l, v);
            slot_fence();
          });
        }
      end(ch);
    }
  }

  // The first step at which the sum of `part(step)` reaches `want`: the step, and what
  // it has to bring.
  template <class G>
  __device__ __forceinline__ void find_step(WideShared& ws, u64 want, G&& part) const {
    const int tid = threadIdx.x, lane = tid & 63;
    __syncthreads();
    if (tid < 64) {
      constexpr int S = kFineSteps / 64;
      u64 s = 0;
      for (int i = 0; i < S; ++i) s += part(lane * S + i);
      const u64 upto = wave_scan(s, lane);
      u64 before = upto - s;
      if (before < want && want <= upto) {
        int i = 0;
        while (before + part(lane * S + i) < want) before += part(lane * S + i++);
        ws.step = lane * S + i;
        ws.left = want - before;
      }
    }
    __syncthreads();
  }

  // The tokens of a step, in order; false where the list does not hold them.
  __device__ __forceinline__ bool collect_step(int step) {
    const int lane = threadIdx.x & 63;
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    each_chunk(
        [&](const float (&f)[EPV], int v) {
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const bool take = fine_step(f[e]) == step;
            const uint32_t at = take_place(take, &sh.count, lane);
            if (take && at < LIST) sh.list[at] = token_of(f[e], v * EPV + e);
          }
        },
        [](int) {});
    __syncthreads();
    sel.count = (int)sh.count;
    if (sel.count > LIST) return false;
    sort_list<BLOCK>(sh.list, sel.count);
    return true;
  }

  // The cut from a histogram over the row.
  __device__ __forceinline__ Cut wide_cut(WideShared& ws) {
    const int tid = threadIdx.x;
    const bool by_count = p.top_k < sel.V;
    for (int i = tid; i < kFineSteps; i += BLOCK) {
      ws.mass[i] = 0;
      ws.count[i] = 0;
    }
    __syncthreads();
    each_chunk(
        [&](const float (&f)[EPV], int) {
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const int st = fine_step(f[e]);
            if (st < kFineSteps) {
              atomicAdd(&ws.mass[st], (u64)weight(f[e]));
              if (by_count) atomicAdd(&ws.count[st], 1u);
            }
          }
        },
        [](int) {});
    __syncthreads();
    // the list's first n logits as a cut
    auto cut_at = [&](int n) {
      const uint32_t key = (uint32_t)(sh.list[n - 1] >> 32);
      u64 ties = 0;
      for (int i = tid; i < n; i += BLOCK) ties += (uint32_t)(sh.list[i] >> 32) == key ? 1 : 0;
      __syncthreads();
      return Cut{key, block_sum<NW>(ties, sh.u)};
    };
    // how many of the list's logits it takes to reach `want`
    auto reach = [&](u64 want) {
      constexpr int PT = LIST / BLOCK;
      const int lane = tid & 63, wid = tid >> 6;
      u64 s = 0, n = 0;
      for (int j = 0; j < PT && tid * PT + j < sel.count; ++j)
        s += weight(token_value(sh.list[tid * PT + j]));
      u64 b = wave_scan(s, lane);
      __syncthreads();
      if (lane == 63) sh.u[wid] = b;
      __syncthreads();
      b -= s;
      for (int w = 0; w < wid; ++w) b += sh.u[w];
      for (int j = 0; j < PT && tid * PT + j < sel.count; ++j) {
        n += b < want ? 1 : 0;
        b += weight(token_value(sh.list[tid * PT + j]));
      }
      __syncthreads();
      n = block_sum<NW>(n, sh.u);
      return (int)n;
    };
    auto radix = [&](u64 want, uint32_t least, auto&& weigh) {
      return radix_cut<E, BLOCK>(sel.rs, sel.nvec, sel.V, want, least, weigh, sh.cut);
    };
    auto mass = [&](int i) { return ws.mass[i]; };
    auto count = [&](int i) { return (u64)ws.count[i]; };
    Cut cut{kNoToken, 0};
    u64 sum = 0;       // the mass that the count leaves
    int kstep = -1;    // the step that the list holds
    u64 n = 0;
    for (int i = tid; i < kFineSteps; i += BLOCK) {
      sum += ws.mass[i];
      n += ws.count[i];
    }
    sum = block_sum<NW>(sum, sh.u);
    __syncthreads();
    n = block_sum<NW>(n, sh.u);
    if (by_count && (u64)p.top_k < n) {   // (else every token with a weight is kept)
      find_step(ws, (u64)p.top_k, count);
      const int step = ws.step;
      const int left = (int)ws.left;
      if (collect_step(step)) {
        kstep = step;
        cut = cut_at(left);
      } else {
        cut = radix((u64)p.top_k, 0u, [](float) { return 1u; });
      }
      u64 s = 0;
      if (kstep >= 0) {
        for (int i = tid; i < step; i += BLOCK) s += ws.mass[i];
        for (int i = tid; i < left; i += BLOCK) s += weight(token_value(sh.list[i]));
      } else {   // (the step's tokens above the key are not known: the row again)
        for (int v = tid; v < sel.nvec; v += BLOCK) {
          float f[EPV];
          tok_vec<E>(sel.rs, v, sel.V, f);
          for (int e = 0; e < EPV; ++e)
            if (order_key(f[e]) > cut.key) s += weight(f[e]);
        }
        if (tid == 0) s += cut.ties * weight(key_value(cut.key));
      }
      __syncthreads();
      sum = block_sum<NW>(s, sh.u);
    }
    if (p.top_p < 1.f) {
      const u64 want = (u64)ceil((double)p.top_p * (double)sum);
      find_step(ws, want, mass);
      const int step = ws.step;
      const u64 left = ws.left;
      if (step == kstep || collect_step(step)) {
        cut = cut_at(reach(left));
      } else {
        const Cut c = radix(want, cut.key, [&](float f) { return weight(f); });
        const u64 w = weight(key_value(c.key));
        if (w > 0) cut = Cut{c.key, (c.ties + w - 1) / w};
      }
    }
    return cut;
  }

  // The kept weights' sums and ties by chunks, and the draw from them.
  __device__ __forceinline__ void from_cut(const Cut& cut) {
    const int lane = threadIdx.x & 63;
    u64* mass = a.draw + row * sel.nch;
    uint32_t* ties = a.ties + row * sel.nch;
    u64 s = 0;
    uint32_t t = 0;
    each_chunk(
        [&](const float (&f)[EPV], int) {
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const uint32_t key = order_key(f[e]);
            if (key > cut.key) {
              const uint32_t w = weight(f[e]);
              s += w >= p.least_w ? w : 0;
            }
            t += key == cut.key ? 1 : 0;
          }
        },
        [&](int ch) {
          s = wave_sum(s);
          t = wave_sum(t);
          if (lane == 0) {
            mass[ch] = s;
            ties[ch] = t;
          }
          s = 0;
          t = 0;
        });
    __syncthreads();
    from_chunks(cut, ties, p.least_w);
  }

  // Draws a row whose cut falls into a step: the step's kept tokens join the chunks' sums above it.
  // False where the list does not hold the step.
  __device__ __forceinline__ bool from_step(WideShared& ws) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t which = row - a.row0;
    const uint32_t n_step = a.steps[which].count;
    const u64 left = a.steps[which].left;
    if (n_step > (uint32_t)a.step_ld || n_step > LIST) return false;
    const int count = (int)n_step, step = a.steps[which].step;
    const uint32_t* ids = a.step_ids + which * a.step_ld;
    for (int i = tid; i < count; i += BLOCK) {
      const int id = (int)ids[i];
      float f[EPV], fy = 0.f;
      tok_vec<E>(sel.rs, id / EPV, sel.V, f);
#pragma unroll
      for (int e = 0; e < EPV; ++e) fy = id % EPV == e ? f[e] : fy;
      sh.list[i] = token_of(fy, id);
    }
    for (int i = tid; i < sel.nch; i += BLOCK) ws.mass[i] = a.draw[row * sel.nch + i];
    __syncthreads();
    sort_list<BLOCK>(sh.list, count);
    // the first tokens that reach `left`, of min_p's weight at least
    const int per = (count + BLOCK - 1) / BLOCK, i0 = tid * per,
              i1 = i0 + per < count ? i0 + per : count;
    u64 s = 0;
    for (int i = i0; i < i1; ++i) s += weight(token_value(sh.list[i]));
    u64 b = ahead(s, sh.u), keep = 0;
    for (int i = i0; i < i1; ++i) {
      const uint32_t q = weight(token_value(sh.list[i]));
      if (b < left && q >= p.least_w) {
        ++keep;
        atomicAdd(&ws.mass[token_id(sh.list[i]) / (EPV * kScanVecs)], (u64)q);
      }
      b += q;
    }
    __syncthreads();
    keep = block_sum<NW>(keep, sh.u);
    const u64 last = keep > 0 ? sh.list[keep - 1] : ~u64(0);
    __syncthreads();
    if (tid < 64) {
      Place at{0, 0, 0, 0, 0};
      for (int i = lane; i < sel.nch; i += 64) at.N += ws.mass[i];
      at.N = wave_sum(at.N);
      at.to = (u64)((double)p.u * (double)at.N);
      if (at.to >= at.N) at.to = at.N - 1;
      for (int i0 = 0; i0 < sel.nch; i0 += 64) {
        const u64 m = i0 + lane < sel.nch ? ws.mass[i0 + lane] : 0,
                  upto = at.before + wave_scan(m, lane), hit = __ballot(upto > at.to);
        if (hit) {
          const int who = __ffsll(hit) - 1;
          at.ch = i0 + who;
          at.before = __shfl(upto - m, who, 64);
          break;
        }
        at.before = __shfl(upto, 63, 64);
      }
      if (lane == 0) put_place(at);
    }
    auto kept = [&](float f, int id) {
      const float t = draw_exponent(f, sel.M, p.c);
      const int st = draw_step(t);
      const uint32_t q = exponent_weight(t);
      const bool in = st < step ? q >= p.least_w : st == step && token_of(f, id) >= last;
      return in ? q : 0u;
    };
    in_chunk<false>(kept, Cut{}, 0);
    return true;
  }

  __device__ __forceinline__ void run(WideShared* ws) {
    const int tid = threadIdx.x;
    sum_rest();
    const int64_t V = sel.V;
    const int k = (int)p.top_k;
    if (p.counted) {
      if (sel.collect(k)) {
        sel.order(k);
        from_list(sel.count < k ? sel.count : k, 0);
        return;
      }
    } else if (p.top_k == V) {
      if (p.top_p == 1.f) {
        __syncthreads();
        from_chunks(Cut{kNoToken, 0}, nullptr, p.least_w);
        return;
      }
      if constexpr (WIDE) {
        if (row_stepped(p, a) && from_step(*ws)) return;
      }
    }
    if constexpr (WIDE) {
      __syncthreads();
      from_cut(wide_cut(*ws));
    } else {
      // a row of many equal logits
      __syncthreads();
      Cut cut = radix_cut<E, BLOCK>(sel.rs, sel.nvec, sel.V, (u64)k, 0u,
                                    [](float) { return 1u; }, sh.cut);
      if (p.top_p < 1.f) {
        u64 s = 0;
        for (int v = tid; v < sel.nvec; v += BLOCK) {
          float f[EPV];
          tok_vec<E>(sel.rs, v, sel.V, f);
          for (int e = 0; e < EPV; ++e)
            if (order_key(f[e]) > cut.key) s += weight(f[e]);
        }
        if (tid == 0) s += cut.ties * weight(key_value(cut.key));
        s = block_sum<NW>(s, sh.u);
        __syncthreads();
        const Cut c = radix_cut<E, BLOCK>(
            sel.rs, sel.nvec, sel.V, (u64)ceil((double)p.top_p * (double)s), cut.key,
            [&](float f) { return weight(f); }, sh.cut);
        const u64 w = weight(key_value(c.key));
        if (w > 0) cut = Cut{c.key, (c.ties + w - 1) / w};
      }
      from_cut(cut);
    }
  }
};

// WIDE: any parameters; else top_k in [1, LIST / 8] for every row, or nothing to cut but min_p.
template <class E, int BLOCK, int LIST, bool WIDE>
__global__ __launch_bounds__(BLOCK) __attribute__((amdgpu_waves_per_eu(4))) void cis_sample_kernel(
    const SampleArgs a) {
  __shared__ SelectShared<LIST> sh;
  __shared__ std::conditional_t<WIDE, WideShared, uint32_t> ws;
  const int64_t row = a.row0 + blockIdx.x;
  const RowParams p = row_params(a, row);
  const int lane = threadIdx.x & 63;
  u64 mass0 = 0;
  if (row_weighed(p, a) && lane < a.s.nch) mass0 = a.draw[row * a.s.nch + lane];
  RowSelect<E, BLOCK, LIST> sel(sh, a.r, a.s, row, p.ok, p.counted);
  if (!p.ok || !sel.tokens()) {
    if (threadIdx.x == 0) {
      a.ids[row] = -1;
      if (a.logp) a.logp[row] = 0.f;
      if (a.logp_kept) a.logp_kept[row] = 0.f;
    }
    return;
  }
  RowDraw<E, BLOCK, LIST, WIDE> draw{a, p, sel, sh, row, 0.f, mass0};
  if constexpr (WIDE)
    draw.run(&ws);
  else
    draw.run(nullptr);
}

const void* weigh_kernel(int dtype, bool step) {
#define CIS_WEIGH(E) \
  (step ? (const void*)&cis_weigh_kernel<E, true> : (const void*)&cis_weigh_kernel<E, false>)
  return dtype == CIS_BF16 ? CIS_WEIGH(Bf16) : CIS_WEIGH(F32);
#undef CIS_WEIGH
}
const void* hist_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_hist_kernel<Bf16>
                           : (const void*)&cis_hist_kernel<F32>;
}
const void* step_kernel() { return (const void*)&cis_step_kernel; }
const void* sample_kernel(int dtype, bool wide) {
  if (dtype == CIS_BF16)
    return wide ? (const void*)&cis_sample_kernel<Bf16, kTokBlock, 8192, true>
                : (const void*)&cis_sample_kernel<Bf16, kTopBlock, 1024, false>;
  return wide ? (const void*)&cis_sample_kernel<F32, kTokBlock, 8192, true>
              : (const void*)&cis_sample_kernel<F32, kTopBlock, 1024, false>;
}

}  // namespace cis
