// The scan of rows of logits that the top-logits and sampling kernels start from, and the top-logits
// kernel (gfx950).
#include "cis_tok_row.h"

namespace cis {

// ------------------------------------------------------------------------------------------
// One wave per chunk of kScanVecs vectors, 8 of them per lane: the chunk's largest logit, the sum of
// its exponentials relative to that, and the groups' largest logits (TokScan). Reads the logits
// once; the workgroups are short-lived and many, which suits a read-only stream here.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ double row16_sum(double x) {
  auto step = [](double x, auto ctrl) {
    constexpr int C = ctrl;
    const u64 b = __builtin_bit_cast(u64, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, C, 0xF, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), C, 0xF, 0xF, false);
    return x + __builtin_bit_cast(double, ((u64)hi << 32) | lo);
  };
  x = step(x, std::integral_constant<int, kDppXor1>{});
  x = step(x, std::integral_constant<int, kDppXor2>{});
  x = step(x, std::integral_constant<int, kDppHalfMirror>{});
  return step(x, std::integral_constant<int, kDppRowMirror>{});
}
__device__ __forceinline__ double lane_double(double x, int lane) {
  const u64 b = __builtin_bit_cast(u64, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane);
  return __builtin_bit_cast(double, ((u64)hi << 32) | lo);
}

template <class E, int GV>
__global__ __launch_bounds__(kScanBlock) void cis_scan_kernel(const ScanArgs a) {
  constexpr int EPV = E::kPerVec, K = kScanVecs / 64, NW = kScanBlock / 64;
  typedef std::conditional_t<EPV == 8, uint16_t, uint32_t> elem;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
  const int V = a.r.V, nch = a.s.nch, ngrp = a.s.ngrp;
  const int64_t total = a.r.T * (int64_t)nch;
  for (int64_t w = (int64_t)blockIdx.x * NW + wid; w < total; w += (int64_t)gridDim.x * NW) {
    const int64_t row = w / nch;
    const int ch = (int)(w - row * nch);
    if (!tok_on(a.r, row)) continue;
    const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
    const int v0 = ch * kScanVecs + lane;
    u32x4 x[K];
    static_for<K>([&](auto I) { x[I] = bload_aux<kAuxNT>(rs, (uint32_t)(v0 + I * 64) * 16u); });
    if ((ch + 1) * kScanVecs * EPV > V)   // past the row's end: -inf
      static_for<K>([&](auto I) {
        const int v = v0 + I * 64;
        if (v >= a.r.nvec - 1) x[I] = v < a.r.nvec ? E::mask_tail(x[I], V - v * EPV) : E::neg_inf_vec();
      });
    float m8[K], m = -INFINITY;
    static_for<K>([&](auto I) {
      float f[EPV];
      E::unpack(x[I], f);
      m8[I] = f[0];
#pragma unroll
      for (int e = 1; e < EPV; ++e) m8[I] = fmaxf(m8[I], f[e]);
      m = fmaxf(m, m8[I]);
      slot_fence();
    });
    opaque(x);   // (unpacked again below, rather than kept unpacked)
    m = wave_max(m);
    const float R = fmaxf(m * a.c, kMinExp);
    double s = 0.0;
    static_for<K>([&](auto I) {
      float f[EPV];
      E::unpack(x[I], f);
      s += (double)vec_sum<E>(f, a.c, R);
      slot_fence();
    });
    s = row16_sum(s);
    s = (lane_double(s, 0) + lane_double(s, 16)) + (lane_double(s, 32) + lane_double(s, 48));
    if (lane == 0) {
      a.s.cmax[w] = m;
      a.s.csum[w] = s;
    }
    elem* gm = (elem*)a.s.gmax + row * ngrp;
    if (GV == 1) {
      static_for<K>([&](auto I) {
        const int g = v0 + I * 64;
        if (g < ngrp) gm[g] = (elem)E::bits_of(m8[I]);
      });
    } else {
      // 8 lanes' vectors are a group; lane l stores slot l % 8 of its eight lanes
      float mine = 0.f;
      static_for<K>([&](auto I) {
        float g = m8[I];
        g = fmaxf(g, dpp16<kDppXor1>(g));
        g = fmaxf(g, dpp16<kDppXor2>(g));
        g = fmaxf(g, dpp16<kDppHalfMirror>(g));
        mine = (lane & 7) == I ? g : mine;
      });
      const int g = ch * (kScanVecs / 8) + (lane & 7) * 8 + (lane >> 3);
      if (g < ngrp) gm[g] = (elem)E::bits_of(mine);
    }
  }
}

const void* scan_kernel(int dtype, int32_t gv) {
  if (dtype == CIS_BF16)
    return gv == 1 ? (const void*)&cis_scan_kernel<Bf16, 1> : (const void*)&cis_scan_kernel<Bf16, 8>;
  return gv == 1 ? (const void*)&cis_scan_kernel<F32, 1> : (const void*)&cis_scan_kernel<F32, 8>;
}

// ------------------------------------------------------------------------------------------
// The K largest logits of a row, by one workgroup, from the scan:
//   1. a threshold that at least K groups reach, from a histogram of the groups' largest logits by
//      their distance from the row's largest (in 256 steps, whose size follows the row);
//   2. the logits of those groups that reach it (every logit of the row that does is among
//      them), into a list in LDS;
//   3. the list put in order: counted into fine steps of the distance, moved to the steps' places,
//      and ranked among the few that share a step;
//   4. the log-sum-exp of the others: the chunks' sums without the vectors that hold listed
//      tokens, and what those vectors hold besides. The sums are in double and a vector's sum is
//      the same bits wherever it is formed, so that nothing of the listed tokens is left over;
//      where less than 2^-28 of the row remains, the row is summed again without them.
// Where the list overflows (a row of many equal logits) the cut is found in passes over the row.
// ------------------------------------------------------------------------------------------
constexpr int kSteps = 1024;         // fine steps
constexpr int kStepMost = 128;       // logits of one step that are ranked against each other
constexpr int kGroupRegs = 16;       // groups that a thread keeps (of rows of up to 4096)
template <int LIST>
struct TopShared {
  u64 list[LIST];             // key << 32 | ~id: falls in the order of the tokens
  union {
    uint32_t group[LIST / 2];
    uint32_t step[kSteps];
    CutShared cut;
  };
  uint32_t hist[256];
  float f[16];
  double d[16];
  uint32_t u[16];
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

// Bitonic sort, falling, of the list's next power of two (0 sorts last).
template <int BLOCK>
__device__ __forceinline__ void sort_list(u64* list, int count) {
  const int tid = threadIdx.x;
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
__global__ __launch_bounds__(BLOCK) __attribute__((amdgpu_waves_per_eu(4))) void cis_top_kernel(
    const TopArgs a) {
  constexpr int NW = BLOCK / 64, EPV = E::kPerVec;
  typedef std::conditional_t<EPV == 8, uint16_t, uint32_t> elem;
  __shared__ TopShared<LIST> sh;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int V = a.r.V, nvec = a.r.nvec, K = a.K, gv = a.s.gv, ngrp = a.s.ngrp;
  const float c = a.c;
  const int64_t row = a.row0 + blockIdx.x;
  const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
  const bool on = tok_on(a.r, row);
  const float* cmax = a.s.cmax + row * a.s.nch;
  const double* csum = a.s.csum + row * a.s.nch;
  // the groups' largest logits, kept where a thread has few of them
  const elem* gm = (const elem*)a.s.gmax + row * ngrp;
  auto group_max = [&](int g) {
    return __uint_as_float(EPV == 8 ? (uint32_t)gm[g] << 16 : (uint32_t)gm[g]);
  };
  const bool kept = ngrp <= kGroupRegs * BLOCK;
  float gr[kGroupRegs];
  if (on && kept)
    static_for<kGroupRegs>([&](auto I) {
      const int g = tid + I * BLOCK;
      gr[I] = I * BLOCK < ngrp && g < ngrp ? group_max(g) : -INFINITY;
    });
  // f(group, its largest logit) for a thread's groups, whole waves together
  auto each_group = [&](auto&& f) {
    if (kept) {
      static_for<kGroupRegs>([&](auto I) {
        if (I * BLOCK < ngrp) f(tid + I * BLOCK, gr[I]);
        slot_fence();
      });
    } else {
      for (int g0 = 0; g0 < ngrp; g0 += BLOCK)
        f(g0 + tid, g0 + tid < ngrp ? group_max(g0 + tid) : -INFINITY);
    }
  };
  float M = -INFINITY;
  bool bad = false;
  if (on)
    for (int i = tid; i < a.s.nch; i += BLOCK) {
      M = fmaxf(M, cmax[i]);
      bad |= !(csum[i] < INFINITY);
    }
  if (tid < 256) sh.hist[tid] = 0;
  M = wave_max(__ballot(bad) ? INFINITY : M);   // (no row that counts holds +inf)
  if (lane == 0) sh.f[wid] = M;
  __syncthreads();
  for (int w = 0; w < NW; ++w) M = fmaxf(M, sh.f[w]);
  bad = M == INFINITY;
  const bool any = M > -INFINITY && !bad;
  int n = 0;   // listed
  if (any) {
    // 1. the threshold
    float scale = 16.f;
    uint32_t bin;
    for (;;) {
      each_group([&](int, float x) {
        if (x > -INFINITY) atomicAdd(&sh.hist[below(x, M, scale, 255.f)], 1u);
      });
      __syncthreads();
      if (tid < 64) {
        uint32_t b[4], s = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) s += b[i] = sh.hist[4 * tid + i];
        const uint32_t upto = wave_scan(s, tid), total = __shfl(upto, 63, 64);
        uint32_t before = upto - s;
        if (total < (uint32_t)K) {   // every logit is taken
          if (tid == 0) sh.bin = 256;
        } else if (before < (uint32_t)K && (uint32_t)K <= upto) {
          int i = 0;
          while (before + b[i] < (uint32_t)K) before += b[i++];
          sh.bin = 4 * tid + i;
          sh.groups = before + b[i];
        }
      }
      __syncthreads();
      bin = sh.bin;
      // too coarse a step takes in many more groups than it has to
      const bool finer = bin < 15 && sh.groups > 2u * (uint32_t)K + 64 && scale < 0x1p40f;
      const bool coarser = bin == 255 && scale > 0x1p-140f;
      __syncthreads();
      if (tid == 0) sh.groups = sh.count = 0;
      if (tid < 256) sh.hist[tid] = 0;
      __syncthreads();
      if (!finer && !coarser) break;
      scale *= finer ? 16.f : 0.0625f;
    }
    // what is taken reaches the smallest of the groups' largest logits within the steps
    float least = INFINITY;
    if (bin == 256)
      least = -FLT_MAX;
    else
      each_group([&](int, float x) {
        if (x > -INFINITY && (uint32_t)below(x, M, scale, 255.f) <= bin) least = fminf(least, x);
      });
    least = -wave_max(-least);
    if (lane == 0) sh.f[wid] = least;
    __syncthreads();
    for (int w = 0; w < NW; ++w) least = fminf(least, sh.f[w]);
    // a place in a list for every lane that takes one
    auto place = [&](bool take, uint32_t* counter) {
      const u64 who = __ballot(take);
      uint32_t at = 0;
      if (who) {
        if (lane == 0) at = atomicAdd(counter, (uint32_t)__popcll(who));
        at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((u64(1) << lane) - 1));
      }
      return at;
    };
    // 2. the list
    each_group([&](int g, float x) {
      const bool take = x >= least;
      const uint32_t at = place(take, &sh.groups);
      if (take && at < LIST / 2) sh.group[at] = (uint32_t)g;
    });
    __syncthreads();
    const uint32_t ng = sh.groups;
    bool fits = ng <= LIST / 2;
    if (fits) {
      const int nv = (int)ng * gv;   // vectors of the groups
      constexpr int U = 4;           // loads in flight
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
      fits = sh.count <= LIST;
    }
    int count = (int)sh.count;
    // 3. in order
    bool ranked = false;
    if (fits && bin < 256) {
      const float fine = scale * ((float)kSteps / (float)(bin + 1));
      constexpr int R = LIST / BLOCK;
      auto step_of = [&](u64 t) { return below(token_value(t), M, fine, (float)(kSteps - 1)); };
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
      // the steps' first places: thread i has steps 4 i ..
      uint32_t b[kSteps / BLOCK], s = 0, most = 0;
      static_for<kSteps / BLOCK>([&](auto J) {
        b[J] = sh.step[tid * (kSteps / BLOCK) + J];
        s += b[J];
        most = most > b[J] ? most : b[J];
      });
      ranked = !__syncthreads_or(most > kStepMost);
      if (ranked) {
        const uint32_t upto = wave_scan(s, lane);
        if (lane == 63) sh.u[wid] = upto;
        __syncthreads();
        uint32_t at = upto - s;
        for (int w = 0; w < wid; ++w) at += sh.u[w];
        static_for<kSteps / BLOCK>([&](auto J) {
          sh.step[tid * (kSteps / BLOCK) + J] = at;
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
    if (!fits) {
      // the cut from passes over the row, then everything above it and the first of the ties
      __syncthreads();
      const Cut cut =
          radix_cut<E, BLOCK>(rs, nvec, V, (u64)K, 0u, [](float) { return 1u; }, sh.cut);
      if (tid == 0) sh.count = 0;
      __syncthreads();
      for (int v = tid; v < nvec; v += BLOCK) {
        float f[EPV];
        tok_vec<E>(rs, v, V, f);
        for (int e = 0; e < EPV; ++e)
          if (order_key(f[e]) > cut.key)
            sh.list[atomicAdd(&sh.count, 1u)] = token_of(f[e], v * EPV + e);
      }
      __syncthreads();
      count = (int)sh.count;
      if (tid < 64) {   // in order of the ids, by one wave, as many as there are to be
        u64 left = cut.ties;
        for (int v0 = 0; v0 < nvec && left > 0; v0 += 64) {
          float f[EPV];
          if (v0 + lane < nvec) {
            tok_vec<E>(rs, v0 + lane, V, f);
          } else {
            for (int e = 0; e < EPV; ++e) f[e] = -INFINITY;
          }
          uint32_t nt = 0;
          for (int e = 0; e < EPV; ++e) nt += order_key(f[e]) == cut.key ? 1 : 0;
          const uint32_t upto = wave_scan(nt, lane), all = __shfl(upto, 63, 64);
          uint32_t t = upto - nt;
          for (int e = 0; e < EPV; ++e)
            if (order_key(f[e]) == cut.key) {
              if (t < left)
                sh.list[count + (int)(cut.ties - left) + t] = token_of(f[e], (v0 + lane) * EPV + e);
              ++t;
            }
          left -= all < left ? all : left;
        }
        if (tid == 0) sh.count = (uint32_t)(count + (int)(cut.ties - left));
      }
      __syncthreads();
      count = (int)sh.count;
    }
    if (!ranked) sort_list<BLOCK>(sh.list, count);
    n = count < K ? count : K;
  }
  if (a.tail && any) {
    // 4. what is not listed
    const u64 last = sh.list[n - 1];
    const float R = fmaxf(M * c, kMinExp);
    double s = 0.0, whole = 0.0;
    for (int i = tid; i < a.s.nch; i += BLOCK)
      whole += csum[i] * (double)fast_exp2(fmaxf(cmax[i] * c, kMinExp) - R);
    for (int k = tid; k < n; k += BLOCK) {
      const int id = (int)~(uint32_t)sh.list[k], v = id / EPV, ch = v / kScanVecs;
      const float Rc = fmaxf(cmax[ch] * c, kMinExp);
      float f[EPV];
      tok_vec<E>(rs, v, V, f);
      const float all = vec_sum<E>(f, c, Rc);
      int first = -1;   // the vector's first listed token brings in the vector
#pragma unroll
      for (int e = EPV - 1; e >= 0; --e)
        if (token_of(f[e], v * EPV + e) >= last) {
          first = e;
          f[e] = -INFINITY;
        }
      if (first == id % EPV)
        s += ((double)vec_sum<E>(f, c, Rc) - (double)all) * (double)fast_exp2(Rc - R);
    }
    whole = block_sum<NW>(whole, sh.d);
    __syncthreads();
    s = whole + block_sum<NW>(s, sh.d);
    float top = M, tail = -INFINITY;
    if (!(s > whole * 0x1p-28)) {
      top = -INFINITY;
      for (int v = tid; v < nvec; v += BLOCK) {
        float f[EPV];
        tok_vec<E>(rs, v, V, f);
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (token_of(f[e], v * EPV + e) < last) top = fmaxf(top, f[e]);
      }
      __syncthreads();
      top = block_max<NW>(top, sh.f);
      s = 0.0;
      if (top > -INFINITY)
        for (int v = tid; v < nvec; v += BLOCK) {
          float f[EPV], x = 0.f;
          tok_vec<E>(rs, v, V, f);
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            x += token_of(f[e], v * EPV + e) < last ? fast_exp2((f[e] - top) * c) : 0.f;
          s += x;
        }
      __syncthreads();
      s = block_sum<NW>(s, sh.d);
      if (top > -INFINITY) tail = top / a.temperature + logf((float)s);
    } else {
      tail = (float)((double)R * 0.693147180559945309417 + log(s));
    }
    if (tid == 0) a.tail[row] = tail;
  } else if (tid == 0 && a.tail) {
    a.tail[row] = bad ? NAN : -INFINITY;
  }
  for (int k = tid; k < K; k += BLOCK) {
    const u64 x = k < n ? sh.list[k] : 0;
    a.ids[row * K + k] = k < n ? (int32_t)~(uint32_t)x : -1;
    a.values[row * K + k] = k < n ? token_value(x) : -INFINITY;
  }
}

// The list holds 8 K logits at least: all of a row of fewer groups than K.
int top_block(int64_t K) { return K <= 256 ? kTopBlock : kTokBlock; }
const void* top_kernel(int dtype, int64_t K) {
#define CIS_TOP(E)                                                                \
  (K <= 128 ? (const void*)&cis_top_kernel<E, kTopBlock, 1024>                    \
   : K <= 256 ? (const void*)&cis_top_kernel<E, kTopBlock, 2048>                  \
              : (const void*)&cis_top_kernel<E, kTokBlock, 8192>)
  return dtype == CIS_BF16 ? CIS_TOP(Bf16) : CIS_TOP(F32);
#undef CIS_TOP
}

}  // namespace cis
