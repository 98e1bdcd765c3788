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
    static_for<K>([&](auto I) { x[I] = bload_aux<0>(rs, (uint32_t)(v0 + I * 64) * 16u); });
    // past the row's end: -inf
    const bool tail = (ch + 1) * kScanVecs * EPV > V;
    auto vec = [&](auto I, float (&f)[EPV]) {
      E::unpack(x[I], f);
      if (tail) mask_past_end<E>(f, v0 + I * 64, V);
    };
    float m8[K], m = -INFINITY;
    static_for<K>([&](auto I) {
      float f[EPV];
      vec(I, f);
      m8[I] = f[0];
#pragma unroll
      for (int e = 1; e < EPV; ++e) m8[I] = fmaxf(m8[I], f[e]);
      m = fmaxf(m, m8[I]);
    });
    opaque(x);   // (unpacked again below, rather than kept unpacked)
    m = wave_max(m);
    const float R = fmaxf(m * a.c, kMinExp);
    double s = 0.0;
    static_for<K>([&](auto I) {
      float f[EPV];
      vec(I, f);
      s += (double)vec_sum<E>(f, a.c, R);
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
//      them), into a list in LDS, and the list sorted;
//   3. the log-sum-exp of the others: the chunks' sums without the vectors that hold listed
//      tokens, and what those vectors hold besides. The sums are in double and a vector's sum is
//      the same bits wherever it is formed, so that nothing of the listed tokens is left over;
//      where less than 2^-28 of the row remains, the row is summed again without them.
// Where the list overflows (a row of many equal logits) the cut is found in passes over the row.
// ------------------------------------------------------------------------------------------
constexpr int kTopList = 4096, kTopGroups = 4096;
struct TopShared {
  u64 list[kTopList];         // key << 32 | ~id: falls in the order of the tokens
  union {
    uint32_t group[kTopGroups];
    CutShared cut;
  };
  uint32_t hist[256];
  float f[4];
  double d[4];
  uint32_t groups, count, bin;
};

// Steps of `scale` below M, at most 255; rises as f falls.
__device__ __forceinline__ int below(float f, float M, float scale) {
  return (int)fminf((M - f) * scale, 255.f);
}

template <class E>
__global__ __launch_bounds__(kTopBlock) void cis_top_kernel(const TopArgs a) {
  constexpr int BLOCK = kTopBlock, NW = BLOCK / 64, EPV = E::kPerVec;
  typedef std::conditional_t<EPV == 8, uint16_t, uint32_t> elem;
  __shared__ TopShared sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int V = a.r.V, nvec = a.r.nvec, K = a.K, gv = a.s.gv;
  const float c = a.c;
  for (int64_t row = blockIdx.x; row < a.r.T; row += gridDim.x) {
    const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
    const bool on = tok_on(a.r, row);
    const float* cmax = a.s.cmax + row * a.s.nch;
    const double* csum = a.s.csum + row * a.s.nch;
    float M = -INFINITY, bad = 0.f;
    if (on)
      for (int i = tid; i < a.s.nch; i += BLOCK) {
        M = fmaxf(M, cmax[i]);
        if (!(csum[i] < INFINITY)) bad = 1.f;
      }
    M = block_max<NW>(M, sh.f);
    __syncthreads();
    bad = block_max<NW>(bad, sh.f);
    const bool any = M > -INFINITY && bad == 0.f;
    int n = 0;   // listed
    if (any) {
      // 1. the threshold
      const elem* gm = (const elem*)a.s.gmax + row * a.s.ngrp;
      auto gmax = [&](int g) {
        return __uint_as_float(EPV == 8 ? (uint32_t)gm[g] << 16 : (uint32_t)gm[g]);
      };
      float scale = 16.f;
      uint32_t bin;
      for (;;) {
        __syncthreads();
        if (tid < 256) sh.hist[tid] = 0;
        __syncthreads();
        for (int g = tid; g < a.s.ngrp; g += BLOCK) {
          const float x = gmax(g);
          if (x > -INFINITY) atomicAdd(&sh.hist[below(x, M, scale)], 1u);
        }
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
        if (bin < 15 && sh.groups > 2u * (uint32_t)K + 64 && scale < 0x1p40f)
          scale *= 16.f;
        else if (bin == 255 && scale > 0x1p-140f)
          scale *= 0.0625f;
        else
          break;
      }
      __syncthreads();
      if (tid == 0) sh.groups = sh.count = 0;
      __syncthreads();
      auto in = [&](float f) { return f > -INFINITY && (uint32_t)below(f, M, scale) <= bin; };
      // 2. the list
      for (int g0 = 0; g0 < a.s.ngrp; g0 += BLOCK) {
        const int g = g0 + tid;
        const bool take = g < a.s.ngrp && in(gmax(g));
        const u64 who = __ballot(take);
        uint32_t at = 0;
        if (lane == 0 && who) at = atomicAdd(&sh.groups, (uint32_t)__popcll(who));
        at = __shfl(at, 0, 64) + __popcll(who & ((u64(1) << lane) - 1));
        if (take && at < kTopGroups) sh.group[at] = (uint32_t)g;
      }
      __syncthreads();
      const uint32_t ng = sh.groups;
      bool fits = ng <= kTopGroups;
      if (fits) {
        const int nv = (int)ng * gv;   // vectors of the groups
        for (int i0 = 0; i0 < nv; i0 += BLOCK) {
          const int i = i0 + tid;
          float f[EPV];
          int v = 0;
          if (i < nv) v = gv == 1 ? (int)sh.group[i] : (int)sh.group[i >> 3] * 8 + (i & 7);
          const bool mine = i < nv && v < nvec;
          if (mine) {
            tok_vec<E>(rs, v, V, f);
          } else {
#pragma unroll
            for (int e = 0; e < EPV; ++e) f[e] = -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const bool take = in(f[e]);
            const u64 who = __ballot(take);
            if (!who) continue;
            uint32_t at = 0;
            if (lane == 0) at = atomicAdd(&sh.count, (uint32_t)__popcll(who));
            at = __shfl(at, 0, 64) + __popcll(who & ((u64(1) << lane) - 1));
            if (take && at < kTopList)
              sh.list[at] = ((u64)order_key(f[e]) << 32) | (uint32_t)~(uint32_t)(v * EPV + e);
          }
        }
        __syncthreads();
        fits = sh.count <= kTopList;
      }
      int count = (int)sh.count;
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
              sh.list[atomicAdd(&sh.count, 1u)] =
                  ((u64)order_key(f[e]) << 32) | (uint32_t)~(uint32_t)(v * EPV + e);
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
                  sh.list[count + (int)(cut.ties - left) + t] =
                      ((u64)cut.key << 32) | (uint32_t)~(uint32_t)((v0 + lane) * EPV + e);
                ++t;
              }
            left -= all < left ? all : left;
          }
          if (tid == 0) sh.count = (uint32_t)(count + (int)(cut.ties - left));
        }
        __syncthreads();
        count = (int)sh.count;
      }
      // bitonic sort, falling, of the next power of two (0 sorts last)
      int P = 1;
      while (P < count) P <<= 1;
      for (int i = count + tid; i < P; i += BLOCK) sh.list[i] = 0;
      for (int size = 2; size <= P; size <<= 1)
        for (int step = size >> 1; step > 0; step >>= 1) {
          __syncthreads();
          for (int h = tid; h < P / 2; h += BLOCK) {
            const int i = 2 * h - (h & (step - 1)), j = i + step;
            const u64 x = sh.list[i], y = sh.list[j];
            if (((i & size) == 0) == (x < y)) {
              sh.list[i] = y;
              sh.list[j] = x;
            }
          }
        }
      __syncthreads();
      n = count < K ? count : K;
    }
    if (a.tail && any) {
      // 3. what is not listed
      const u64 last = sh.list[n - 1];
      auto token = [&](float f, int id) {
        return ((u64)order_key(f) << 32) | (uint32_t)~(uint32_t)id;
      };
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
          if (token(f[e], v * EPV + e) >= last) {
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
            if (token(f[e], v * EPV + e) < last) top = fmaxf(top, f[e]);
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
              x += token(f[e], v * EPV + e) < last ? fast_exp2((f[e] - top) * c) : 0.f;
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
      a.tail[row] = bad != 0.f ? NAN : -INFINITY;
    }
    for (int k = tid; k < K; k += BLOCK) {
      const u64 x = k < n ? sh.list[k] : 0;
      a.ids[row * K + k] = k < n ? (int32_t)~(uint32_t)x : -1;
      a.values[row * K + k] = k < n ? key_value((uint32_t)(x >> 32)) : -INFINITY;
    }
    __syncthreads();
  }
}

const void* top_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_top_kernel<Bf16> : (const void*)&cis_top_kernel<F32>;
}

}  // namespace cis
