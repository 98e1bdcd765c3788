// Selection of a row's largest logits by one workgroup, from the scan of the row (TokScan): shared by
// the top-logits and the sampling kernels.
#pragma once

#include "cis_tok_row.h"

namespace cis {

// The logits' format as whole numbers.
template <class E>
using elem_t = std::conditional_t<E::kPerVec == 8, uint16_t, uint32_t>;

// A vector's first n elements, and -inf for the others (n <= 0: all of them).
template <class E>
__device__ __forceinline__ u32x4 tail_vec(u32x4 x, int n) {
  constexpr int per = E::kPerVec / 4;   // elements per word
  const u32x4 none = E::neg_inf_vec();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t keep = n > k * per ? ~0u : 0u;
    if (per == 2 && n == 2 * k + 1) keep = 0xFFFFu;
    x[k] = (x[k] & keep) | (none[k] & ~keep);
  }
  return x;
}

// A chunk's vectors, 8 per lane; past the row's end -inf.
constexpr int kScanSlots = kScanVecs / 64;
template <class E, int AUX>
__device__ __forceinline__ void load_chunk(__amdgpu_buffer_rsrc_t rs, const TokRows& r, int ch,
                                           int lane, u32x4 (&x)[kScanSlots]) {
  const int v0 = ch * kScanVecs + lane;
  static_for<kScanSlots>([&](auto I) { x[I] = bload_aux<AUX>(rs, (uint32_t)(v0 + I * 64) * 16u); });
  if ((ch + 1) * kScanVecs * E::kPerVec > r.V)
    static_for<kScanSlots>([&](auto I) {
      x[I] = tail_vec<E>(x[I], r.V - (v0 + I * 64) * E::kPerVec);
    });
}

constexpr int kSteps = 1024;         // fine steps
constexpr int kStepMost = 128;       // logits of one step that are ranked against each other
constexpr int kGroupRegs = 16;       // groups that a thread keeps
template <int LIST>
struct SelectShared {
  u64 list[LIST];             // key << 32 | ~id: falls in the order of the tokens
  union {
    uint32_t group[LIST / 2];
    uint32_t step[kSteps];
    u64 mass[kSteps];
    CutShared cut;
  };
  uint32_t hist[256];
  float f[16];
  double d[16];
  u64 u[16];
  uint32_t groups, count, bin;
};

// Steps of `scale` below M, at most `most`; rises as f falls.
__device__ __forceinline__ int below(float f, float M, float scale, float most) {
  return (int)fminf((M - f) * scale, most);
}
__device__ __forceinline__ u64 token_of(float f, int id) {
  return ((u64)order_key(f) << 32) | (uint32_t)~(uint32_t)id;
}
__device__ __forceinline__ float token_value(u64 t) { return key_value((uint32_t)(t >> 32)); }
__device__ __forceinline__ int token_id(u64 t) { return (int)~(uint32_t)t; }

// A place in a list for every lane that takes one.
__device__ __forceinline__ uint32_t take_place(bool take, uint32_t* counter, int lane) {
  const u64 who = __ballot(take);
  uint32_t at = 0;
  if (who) {
    if (lane == 0) at = atomicAdd(counter, (uint32_t)__popcll(who));
    at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((u64(1) << lane) - 1));
  }
  return at;
}

// The list in falling order of its different entries: by counting those above each where there are
// few (29 entries by 16 waves: 2.8 us in steps, 0.5 us counted), else a bitonic sort of the list's next
// power of two (0 sorts last).
template <int BLOCK>
__device__ __forceinline__ void sort_list(u64* list, int count) {
  const int tid = threadIdx.x;
  if (count <= 256) {
    __syncthreads();
    const u64 x = tid < count ? list[tid] : 0;
    int at = 0;
    if (tid < count)
      for (int j = 0; j < count; ++j) at += list[j] > x ? 1 : 0;
    __syncthreads();
    if (tid < count) list[at] = x;
    __syncthreads();
    return;
  }
  int P = 1;
  while (P < count) P <<= 1;
  for (int i = count + tid; i < P; i += BLOCK) list[i] = 0;
  for (int size = 2; size <= P; size <<= 1)
    for (int step = size >> 1; step > 0; step >>= 1) {
      __syncthreads();
      for (int h = tid; h < P / 2; h += BLOCK) {
        const int i = 2 * h - (h & (step - 1)), j = i + step;
        const u64 x = list[i], y = list[j];
        if (((i & size) == 0) == (x < y)) {
          list[i] = y;
          list[j] = x;
        }
      }
    }
  __syncthreads();
}

template <class E, int BLOCK, int LIST>
struct RowSelect {
  static constexpr int NW = BLOCK / 64, EPV = E::kPerVec;
  SelectShared<LIST>& sh;
  __amdgpu_buffer_rsrc_t rs;
  int V, nvec, ngrp, gv, nch;
  const elem_t<E>* gm;
  const float* cmax;
  const double* csum;
  float cmax0;      // of chunk `tid`
  double csum0;
  float gr[kGroupRegs];
  bool kept;
  float M;          // the row's largest logit
  bool bad;         // a NaN or a +inf in it
  float top, least; // the last collect() took the logits from `least`; few of them lie above `top`
  uint32_t bin;     // 256: it took every logit
  int count;        // logits in the list

  __device__ __forceinline__ RowSelect(SelectShared<LIST>& s, const TokRows& r, const TokScan& t,
                                       int64_t row, bool on, bool groups)
      : sh(s), rs(tok_rsrc(r, row)), V(r.V), nvec(r.nvec), ngrp(t.ngrp), gv(t.gv), nch(t.nch),
        gm((const elem_t<E>*)t.gmax + row * t.ngrp), cmax(t.cmax + row * t.nch),
        csum(t.csum + row * t.nch) {
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    // the groups' largest logits, kept where a thread has few of them
    kept = ngrp <= kGroupRegs * BLOCK;
    if (on && groups && kept)
      static_for<kGroupRegs>([&](auto I) {
        const int g = tid + I * BLOCK;
        gr[I] = I * BLOCK < ngrp && g < ngrp ? group_max(g) : -INFINITY;
      });
    cmax0 = -INFINITY;
    csum0 = 0.0;
    if (on && tid < nch) {
      cmax0 = cmax[tid];
      csum0 = csum[tid];
    }
    M = cmax0;
    bad = !(csum0 < INFINITY);
    if (on)
      for (int i = BLOCK + tid; i < nch; i += BLOCK) {
        M = fmaxf(M, cmax[i]);
        bad |= !(csum[i] < INFINITY);
      }
    if (tid < 256) sh.hist[tid] = 0;
    M = wave_max(__ballot(bad) ? INFINITY : M);   // (no row that counts holds +inf)
    if (lane == 0) sh.f[wid] = M;
    __syncthreads();
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sh.f[w]);
    bad = M == INFINITY;
  }
  __device__ __forceinline__ bool tokens() const { return M > -INFINITY && !bad; }
  __device__ __forceinline__ float group_max(int g) const {
    return __uint_as_float(EPV == 8 ? (uint32_t)gm[g] << 16 : (uint32_t)gm[g]);
  }
  // f(group, its largest logit) for a thread's groups, whole waves together
  template <class F>
  __device__ __forceinline__ void each_group(F&& f) const {
    const int tid = threadIdx.x;
    if (kept) {
      static_for<kGroupRegs>([&](auto I) {
        if (I * BLOCK < ngrp) f(tid + I * BLOCK, gr[I]);
        slot_fence();
      });
    } else {
      for (int g0 = 0; g0 < ngrp; g0 += BLOCK)
        f(g0 + tid, g0 + tid < ngrp ? group_max(g0 + tid) : -INFINITY);
    }
  }

  // The logits that reach the K-th largest of the groups' largest ones (about: within a step), or all
  // of a row with fewer groups: the K largest logits are among them. False, where the list does
  // not hold them.
  __device__ __forceinline__ bool collect(int K) {
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    // 256 steps below `top`, of the groups that do not lie above it; those that do are `prior`. From
    // pass to pass the step that holds the K-th group is looked at more closely, or what lies
    // beyond the steps.
    float scale = 16.f;
    uint32_t prior = 0;
    top = M;
    for (;;) {
      each_group([&](int, float x) {
        if (x > -INFINITY && x <= top) atomicAdd(&sh.hist[below(x, top, scale, 255.f)], 1u);
      });
      __syncthreads();
      if (tid < 64) {
        uint32_t b[4], s = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) s += b[i] = sh.hist[4 * tid + i];
        const uint32_t upto = wave_scan(s, tid) + prior, total = __shfl(upto, 63, 64);
        uint32_t before = upto - s;
        if (total < (uint32_t)K) {   // every logit is taken
          if (tid == 0) sh.bin = 256;
        } else if (before < (uint32_t)K && (uint32_t)K <= upto) {
          int i = 0;
          while (before + b[i] < (uint32_t)K) before += b[i++];
          sh.bin = 4 * tid + i;
          sh.groups = before + b[i];
          sh.count = before;
        }
      }
      __syncthreads();
      bin = sh.bin;
      const uint32_t reach = sh.groups, before = sh.count;
      // too coarse a step takes in many more groups than it has to
      const bool finer = bin < 255 && reach > 2u * (uint32_t)K + 64 && scale < 0x1p40f;
      const bool coarser = bin == 255 && scale > 0x1p-140f;
      float hi = -INFINITY, lo = INFINITY;   // of the step's groups
      if (finer || coarser) {
        each_group([&](int, float x) {
          if (x > -INFINITY && x <= top && (uint32_t)below(x, top, scale, 255.f) == bin) {
            hi = fmaxf(hi, x);
            lo = fminf(lo, x);
          }
        });
        hi = wave_max(hi);
        lo = -wave_max(-lo);
        if (lane == 0) {
          sh.f[wid] = hi;
          sh.d[wid] = lo;
        }
      }
      __syncthreads();
      if (tid == 0) sh.groups = sh.count = 0;
      if (tid < 256) sh.hist[tid] = 0;
      if (finer || coarser)
        for (int w = 0; w < NW; ++w) {
          hi = fmaxf(hi, sh.f[w]);
          lo = fminf(lo, (float)sh.d[w]);
        }
      __syncthreads();
      if (!(finer || coarser) || hi == lo) {
        least = hi == lo ? lo : -FLT_MAX;   // (the last step has no end)
        break;
      }
      top = hi;
      prior = before;
      scale *= finer ? 16.f : 0.25f;
    }
    // what is taken reaches the steps' end, or falls a few roundings short of it: no group of the
    // steps is left out
    if (bin < 255) {
      const float end = top - (float)(bin + 1) / scale * (1.f + 0x1p-20f);
      least = fmaxf(end - fabsf(end) * 0x1p-22f, -FLT_MAX);
    }
    {
      uint32_t mine = 0;
      each_group([&](int, float x) { mine += x >= least ? 1 : 0; });
      const uint32_t upto = wave_scan(mine, lane);
      uint32_t at = 0;
      if (lane == 63 && upto) at = atomicAdd(&sh.groups, upto);
      at = __builtin_amdgcn_readlane(at, 63) + upto - mine;
      if (mine)
        each_group([&](int g, float x) {
          if (x >= least) {
            if (at < LIST / 2) sh.group[at] = (uint32_t)g;
            ++at;
          }
        });
    }
    __syncthreads();
    const uint32_t ng = sh.groups;
    if (ng > LIST / 2) return false;
    const int nv = (int)ng * gv;   // vectors of the groups
    constexpr int U = 4;           // loads in flight (8: fewer waves fit, 132 us became 179)
    for (int i0 = 0; i0 < nv; i0 += U * BLOCK) {
      u32x4 x[U];
      int v[U];
      static_for<U>([&](auto J) {
        const int i = i0 + J * BLOCK + tid;
        v[J] = nvec;
        if (i < nv) v[J] = gv == 1 ? (int)sh.group[i] : (int)sh.group[i >> 3] * 8 + (i & 7);
        x[J] = bload_aux<0>(rs, v[J] < nvec ? (uint32_t)v[J] * 16u : kOutOfRange);
      });
      // places for all that a wave takes at once
      uint32_t mine = 0;
      static_for<U>([&](auto J) {
        float f[EPV];
        E::unpack(x[J], f);
        if ((v[J] + 1) * EPV > V) {
          mask_past_end<E>(f, v[J], V);
          x[J] = E::pack(f);
        }
#pragma unroll
        for (int e = 0; e < EPV; ++e) mine += f[e] >= least ? 1 : 0;
        slot_fence();
      });
      const uint32_t upto = wave_scan(mine, lane);
      uint32_t at = 0;
      if (lane == 63 && upto) at = atomicAdd(&sh.count, upto);
      at = __builtin_amdgcn_readlane(at, 63) + upto - mine;
      if (mine)
        static_for<U>([&](auto J) {
          float f[EPV];
          E::unpack(x[J], f);
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (f[e] >= least) {
              if (at < LIST) sh.list[at] = token_of(f[e], v[J] * EPV + e);
              ++at;
            }
          slot_fence();
        });
    }
    __syncthreads();
    count = (int)sh.count;
    __syncthreads();
    return count <= LIST;
  }

  // The first K of the collected list in order: counted into fine steps (a quarter of them above
  // `top`), moved to the steps' places, and ranked among the few that share a step.
  __device__ __forceinline__ void order(int K) {
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    constexpr int R = LIST / BLOCK, S = kSteps / BLOCK;
    bool ranked = bin < 256;
    if (ranked) {
      const int first = top < M ? kSteps / 4 : 0;
      const float above = (float)first / fmaxf(M - top, FLT_MIN),
                  fine = (float)(kSteps - first) / fmaxf(top - least, FLT_MIN);
      auto step_of = [&](u64 t) {
        const float f = token_value(t);
        return f > top ? below(f, M, above, (float)(first - 1))
                       : first + below(f, top, fine, (float)(kSteps - first - 1));
      };
      for (int i = tid; i < kSteps; i += BLOCK) sh.step[i] = 0;
      __syncthreads();
      u64 t[R];
      static_for<R>([&](auto J) {
        const int i = tid + J * BLOCK;
        if (i < count) {
          t[J] = sh.list[i];
          atomicAdd(&sh.step[step_of(t[J])], 1u);
        }
        slot_fence();
      });
      __syncthreads();
      uint32_t b[S], s = 0, most = 0;   // thread i has steps S i ..
      static_for<S>([&](auto J) {
        b[J] = sh.step[tid * S + J];
        s += b[J];
        most = most > b[J] ? most : b[J];
      });
      ranked = !__syncthreads_or(most > kStepMost);
      if (ranked) {
        const uint32_t upto = wave_scan(s, lane);
        if (lane == 63) sh.u[wid] = upto;
        __syncthreads();
        uint32_t at = upto - s;
        for (int w = 0; w < wid; ++w) at += (uint32_t)sh.u[w];
        static_for<S>([&](auto J) {
          sh.step[tid * S + J] = at;
          at += b[J];
        });
        __syncthreads();
        static_for<R>([&](auto J) {
          if (tid + J * BLOCK < count) sh.list[atomicAdd(&sh.step[step_of(t[J])], 1u)] = t[J];
        });
        __syncthreads();   // step[i] is now the end of step i
        uint32_t to[R];
        static_for<R>([&](auto J) {
          const int i = tid + J * BLOCK;
          to[J] = LIST;
          if (i >= count) return;
          t[J] = sh.list[i];
          const int st = step_of(t[J]);
          const uint32_t lo = st > 0 ? sh.step[st - 1] : 0, hi = sh.step[st];
          if (lo >= (uint32_t)K) return;
          uint32_t r = lo;
          for (uint32_t j = lo; j < hi; ++j) r += sh.list[j] > t[J] ? 1 : 0;
          to[J] = r;
        });
        __syncthreads();
        static_for<R>([&](auto J) {
          if (to[J] < (uint32_t)K) sh.list[to[J]] = t[J];
        });
        __syncthreads();
      }
    }
    if (!ranked) sort_list<BLOCK>(sh.list, count);
  }
};

}  // namespace cis
