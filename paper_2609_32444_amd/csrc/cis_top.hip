// The scan of rows of logits that the top-logits and sampling kernels start from, and the top-logits
// kernel (gfx950).
#include "cis_select.h"

namespace cis {

// ------------------------------------------------------------------------------------------
// One wave per chunk of kScanVecs vectors, 8 of them per lane: the chunk's largest logit, the sum of
// its exponentials relative to that, and the groups' largest logits (TokScan). Reads the logits
// once; the workgroups are short-lived and many, which suits a read-only stream here. Bound by the
// memory: 6000 rows of V = 151936 in 299 us (6.1 TB/s), 512 rows in 25 us (6.2 TB/s). Loads of more
// logits than the memory-side cache holds are marked as not used again (6000 rows, K = 256: 54 us
// less); those of fewer are not (512 uncut rows, which are read again: 70 to 65 us).
// ------------------------------------------------------------------------------------------
template <class E, int GV, int AUX, bool DRAFTS>
__global__ __launch_bounds__(kScanBlock) void cis_scan_kernel(const ScanArgs a) {
  constexpr int EPV = E::kPerVec, K = kScanSlots, NW = kScanBlock / 64;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
  const int nch = a.s.nch, ngrp = a.s.ngrp;
  const int64_t total = a.r.T * (int64_t)nch;
  for (int64_t w = (int64_t)blockIdx.x * NW + wid; w < total; w += (int64_t)gridDim.x * NW) {
    const int64_t row = w / nch;
    const int ch = (int)(w - row * nch);
    if (DRAFTS ? !tok_seq_on(a.r, row) : !tok_on(a.r, row)) continue;
    const __amdgpu_buffer_rsrc_t rs = tok_rsrc<DRAFTS>(a.r, row);
    const int v0 = ch * kScanVecs + lane;
    u32x4 x[K];
    load_chunk<E, AUX>(rs, a.r, ch, lane, x);
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
    const float ref = sum_ref(m);
    double s = 0.0;
    static_for<K>([&](auto I) {
      float f[EPV];
      E::unpack(x[I], f);
      s += (double)vec_sum<E>(f, a.c, ref);
      slot_fence();
    });
    s = wave_sum(s);
    if (lane == 0) {
      a.s.cmax[w] = m;
      a.s.csum[w] = s;
    }
    elem_t<E>* gm = (elem_t<E>*)a.s.gmax + row * ngrp;
    if (GV == 0) continue;
    if (GV == 1) {
      static_for<K>([&](auto I) {
        const int g = v0 + I * 64;
        if (g < ngrp) gm[g] = (elem_t<E>)E::bits_of(m8[I]);
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
      if (g < ngrp) gm[g] = (elem_t<E>)E::bits_of(mine);
    }
  }
}

template <bool DRAFTS>
const void* scan_kernel_of(int dtype, int32_t gv, bool keep) {
#define CIS_SCAN_G(E, G)                                       \
  (keep ? (const void*)&cis_scan_kernel<E, G, 0, DRAFTS>       \
        : (const void*)&cis_scan_kernel<E, G, kAuxNT, DRAFTS>)
#define CIS_SCAN(E) (gv == 0 ? CIS_SCAN_G(E, 0) : gv == 1 ? CIS_SCAN_G(E, 1) : CIS_SCAN_G(E, 8))
  return dtype == CIS_BF16 ? CIS_SCAN(Bf16) : CIS_SCAN(F32);
#undef CIS_SCAN
#undef CIS_SCAN_G
}
const void* scan_kernel(int dtype, int32_t gv, bool keep, bool drafts) {
  return drafts ? scan_kernel_of<true>(dtype, gv, keep) : scan_kernel_of<false>(dtype, gv, keep);
}

// ------------------------------------------------------------------------------------------
// The K largest logits of a row, by one workgroup, from the scan:
//   1. a threshold that at least K groups reach, from a histogram of the groups' largest logits by
//      their distance from the row's largest (in 256 steps, whose size follows the row);
//   2. the logits of those groups that reach it (every logit of the row that does is among
//      them), into a list in LDS;
//   3. the list put in order (1 to 3: RowSelect);
//   4. the log-sum-exp of the others: the chunks' sums without the vectors that hold listed
//      tokens, and what those vectors hold besides. The sums are in double and a vector's sum is
//      the same bits wherever it is formed, so that nothing of the listed tokens is left over;
//      where less than 2^-28 of the row remains, the row is summed again without them.
// Where the list overflows (a row of many equal logits) the cut is found in passes over the row.
// Bound by the groups' lines, which lie apart: 6000 rows, K = 256, in 136 us (some 600 lines of 128
// bytes a row); and for few rows by the steps' latency: 96 rows, K = 8, in 14 us.
// ------------------------------------------------------------------------------------------
template <class E, int BLOCK, int LIST>
__global__ __launch_bounds__(BLOCK) __attribute__((amdgpu_waves_per_eu(4))) void cis_top_kernel(
    const TopArgs a) {
  constexpr int NW = BLOCK / 64, EPV = E::kPerVec;
  __shared__ SelectShared<LIST> sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int V = a.r.V, nvec = a.r.nvec, K = a.K;
  const float c = a.c;
  const int64_t row = a.row0 + blockIdx.x;
  const bool on = tok_on(a.r, row);
  RowSelect<E, BLOCK, LIST> sel(sh, a.r, a.s, row, on, on);
  const __amdgpu_buffer_rsrc_t rs = sel.rs;
  const float M = sel.M;
  const bool any = sel.tokens(), bad = sel.bad;
  int n = 0;   // listed
  if (any) {
    if (sel.collect(K)) {
      sel.order(K);
      n = sel.count < K ? sel.count : K;
    } else {
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
      int count = (int)sh.count;
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
      n = (int)sh.count;
      sort_list<BLOCK>(sh.list, n);
    }
  }
  if (a.tail && any) {
    // 4. what is not listed
    const u64 last = sh.list[n - 1];
    double s = 0.0, whole = 0.0;
    for (int i = tid; i < a.s.nch; i += BLOCK)
      whole += sel.csum[i] * (double)fast_exp2((sel.cmax[i] - M) * c);
    for (int k = tid; k < n; k += BLOCK) {
      const int id = token_id(sh.list[k]), v = id / EPV, ch = v / kScanVecs;
      const float m = sel.cmax[ch];   // (not -inf: it holds a token)
      float f[EPV];
      tok_vec<E>(rs, v, V, f);
      const float all = vec_sum<E>(f, c, m);
      int first = -1;   // the vector's first listed token brings in the vector
#pragma unroll
      for (int e = EPV - 1; e >= 0; --e)
        if (token_of(f[e], v * EPV + e) >= last) {
          first = e;
          f[e] = -INFINITY;
        }
      if (first == id % EPV)
        s += ((double)vec_sum<E>(f, c, m) - (double)all) * (double)fast_exp2((m - M) * c);
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
      tail = (float)((double)M / (double)a.temperature + log(s));
    }
    if (tid == 0) a.tail[row] = tail;
  } else if (tid == 0 && a.tail) {
    a.tail[row] = bad ? NAN : -INFINITY;
  }
  for (int k = tid; k < K; k += BLOCK) {
    const u64 x = k < n ? sh.list[k] : 0;
    a.ids[row * K + k] = k < n ? token_id(x) : -1;
    a.values[row * K + k] = k < n ? token_value(x) : -INFINITY;
  }
}

// The list holds 8 K logits at least: all of a row of fewer groups than K. (16 waves for few rows, whose
// barriers wait for more of them: 96 rows, K = 8: 21.2 us for 21.5; a draw of one token 21.0 for 19.5.)
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
