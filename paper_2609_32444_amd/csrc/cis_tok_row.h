// What the sampling and top-logits kernels share: the order of a row's logits as whole numbers, the
// weights of a draw, and a workgroup's selection of the point where a cut falls.
//
// A logit's key is its float32 bits mapped to an unsigned integer of the same order (+0 for -0);
// tokens are ordered by (key descending, id ascending). Every cut keeps a first part of that order, so
// it is a pair (key, ties): the tokens of larger keys, and the first `ties` ones of that key.
#pragma once

#include "cis_row.h"
#include "cis_tok.h"

namespace cis {

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k ^ (~(uint32_t)((int32_t)k >> 31) | 0x80000000u));
}
constexpr uint32_t kNoToken = 0x007FFFFFu;   // the key of -inf

// Weight of logit f in a draw, for the row's largest M and c = log2(e) / temperature. -inf (no
// token) has weight 0, whatever c is.
__device__ __forceinline__ uint32_t draw_weight(float f, float M, float c) {
  return (uint32_t)(fast_exp2((f - M) * c) * (float)kDrawOne);
}

// A row's descriptor. DRAFTS: of verification, whose rows from T1 on are the drafts'. (The other operators' kernels
// do not look at what says so: 64 uncut rows of V = 151936 20.5 us a call for 21.1, 256 of 262144 under top_p 84.1 for 85.0.)
template <bool DRAFTS = false>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tok_rsrc(const TokRows& r, int64_t row) {
  const char* p = !DRAFTS || row < r.T1 ? (const char*)r.logits + row * r.row_bytes
                                        : (const char*)r.draft + (row - r.T1) * r.draft_bytes;
  return make_rsrc(p, (uint32_t)r.nvec * 16u);
}
__device__ __forceinline__ bool tok_on(const TokRows& r, int64_t row) {
  return r.mask ? sload_byte(r.mask, row) != 0 : true;
}
// Verification: whether a row is a sequence's, a draft may be one.
__device__ __forceinline__ bool tok_seq_on(const TokRows& r, int64_t row) {
  const int64_t end = sload(r.offsets + r.n_seq);
  return row < r.T1 ? row < end : row - r.T1 < end - 1;
}
// The sequence that a row or a draft belongs to, if any does (else one of them).
__device__ __forceinline__ int64_t tok_seq(const TokRows& r, int64_t row) {
  const bool draft = row >= r.T1;
  const int64_t end = sload(r.offsets + r.n_seq), at = draft ? row - r.T1 : row;
  int64_t lo = 0, hi = r.n_seq - 1;
  while (lo < hi) {   // the last one that starts at the row or ahead of it
    const int64_t mid = (lo + hi + 1) / 2, first = sload(r.offsets + mid);
    if (draft ? first < end && first - mid <= at : first <= at)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}
// Vector v of a row; elements past the row's end are -inf.
template <class E>
__device__ __forceinline__ void tok_vec(__amdgpu_buffer_rsrc_t rs, int v, int V,
                                        float (&f)[E::kPerVec]) {
  E::unpack(bload_aux<0>(rs, (uint32_t)v * 16u), f);
  if ((v + 1) * E::kPerVec > V) mask_past_end<E>(f, v, V);
}

// Sum of exp2((f - m) c) over a vector. Its order is fixed and nothing in it can be contracted: a
// vector gives the same bits wherever it is summed, so that a sum taken out of a larger one (in
// double) leaves exactly the others.
template <class E>
__device__ __forceinline__ float vec_sum(const float (&f)[E::kPerVec], float c, float m) {
  float x[E::kPerVec];
#pragma unroll
  for (int e = 0; e < E::kPerVec; ++e) x[e] = fast_exp2((f[e] - m) * c);
  float s = (x[0] + x[1]) + (x[2] + x[3]);
  if constexpr (E::kPerVec == 8) s += (x[4] + x[5]) + (x[6] + x[7]);
  return s;
}
// The reference of a sum whose largest logit is m: finite where there is nothing but -inf.
__device__ __forceinline__ float sum_ref(float m) { return fmaxf(m, -FLT_MAX); }

// Sums over a wave, in every lane: within rows of 16 lanes by permutations, then over the four rows.
template <class T, class F>
__device__ __forceinline__ T wave_reduce(T x, F&& step) {
  x += step(x, std::integral_constant<int, kDppXor1>{});
  x += step(x, std::integral_constant<int, kDppXor2>{});
  x += step(x, std::integral_constant<int, kDppHalfMirror>{});
  return x + step(x, std::integral_constant<int, kDppRowMirror>{});
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_word(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
__device__ __forceinline__ uint32_t lane_word(uint32_t x, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}
template <class T>
__device__ __forceinline__ T wave_sum(T x) {
  if constexpr (sizeof(T) == 4) {
    x = wave_reduce(x, [](T y, auto ctrl) {
      return __builtin_bit_cast(T, dpp_word<ctrl>(__builtin_bit_cast(uint32_t, y)));
    });
    auto at = [&](int l) { return __builtin_bit_cast(T, lane_word(__builtin_bit_cast(uint32_t, x), l)); };
    return (at(0) + at(16)) + (at(32) + at(48));
  } else {
    auto both = [](T y, auto&& f) {
      const u64 b = __builtin_bit_cast(u64, y);
      return __builtin_bit_cast(T, ((u64)f((uint32_t)(b >> 32)) << 32) | f((uint32_t)b));
    };
    x = wave_reduce(x, [&](T y, auto ctrl) {
      constexpr int C = ctrl;
      return both(y, [](uint32_t w) { return dpp_word<C>(w); });
    });
    auto at = [&](int l) { return both(x, [l](uint32_t w) { return lane_word(w, l); }); };
    return (at(0) + at(16)) + (at(32) + at(48));
  }
}
__device__ __forceinline__ float wave_max(float x) {
  const float m = row16_max(x);
  return fmaxf(fmaxf(lane_value(m, 0), lane_value(m, 16)),
               fmaxf(lane_value(m, 32), lane_value(m, 48)));
}
// A wave's sum of its lanes' sums of exp2((z - R) c): R the largest of their references.
__device__ __forceinline__ void wave_lse(float& R, float& s, float c) {
  const float m = wave_max(R);
  s = wave_sum(s * fast_exp2((R - m) * c));
  R = m;
}
// Sum over the lanes up to this one.
template <class T>
__device__ __forceinline__ T wave_scan(T x, int lane) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  return x;
}

// Sum over a workgroup's NW waves, in a fixed order, in every thread. `sh` may be used again after
// the next barrier.
template <int NW, class T>
__device__ __forceinline__ T block_sum(T x, T* sh) {
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  T s = sh[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) s += sh[w];
  return s;
}
template <int NW>
__device__ __forceinline__ float block_max(float x, float* sh) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  float m = sh[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) m = fmaxf(m, sh[w]);
  return m;
}

// The part of a row that is cut off: keys below `key`, and of that key all but the first `ties`.
struct Cut {
  uint32_t key;
  u64 ties;
};

// Working memory of radix_cut.
struct CutShared {
  u64 bins[256];
  uint32_t byte;
  u64 left;
};

// The key at which the running sum of weigh(f) over a row's tokens, in falling order of their
// keys, reaches `target` (at least 1), and what that key's own tokens have to bring: a byte of
// the key at a time, from a histogram of the byte among the tokens that agree with the bytes
// found. Tokens of keys below `least` are left out. With a target beyond the whole sum, the last
// token's key. Every thread returns the same.
template <class E, int BLOCK, class W>
__device__ __forceinline__ Cut radix_cut(__amdgpu_buffer_rsrc_t rs, int nvec, int V, u64 target,
                                         uint32_t least, W&& weigh, CutShared& sh) {
  constexpr int EPV = E::kPerVec;
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) sh.bins[tid] = 0;
    __syncthreads();
    for (int v = tid; v < nvec; v += BLOCK) {
      float f[EPV];
      tok_vec<E>(rs, v, V, f);
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const uint32_t k = order_key(f[e]);
        const bool in = k > kNoToken && k >= least && (shift == 24 || (k >> (shift + 8)) == prefix);
        if (in) atomicAdd(&sh.bins[(k >> shift) & 255u], (u64)weigh(f[e]));
      }
    }
    __syncthreads();
    if (tid < 64) {   // lane l has bins 255 - 4 l downwards
      u64 b[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) s += b[i] = sh.bins[255 - 4 * tid - i];
      const u64 upto = wave_scan(s, tid), total = __shfl(upto, 63, 64);
      const u64 want = target < total ? target : total;
      u64 before = upto - s;
      if (before < want && want <= upto) {   // one lane, where any bin holds something
        int i = 0;
        while (before + b[i] < want) before += b[i++];
        sh.byte = 255 - 4 * tid - i;
        sh.left = want - before;
      }
      if (total == 0 && tid == 0) {
        sh.byte = 255;
        sh.left = 0;
      }
    }
    __syncthreads();
    prefix = (prefix << 8) | sh.byte;
    target = sh.left;
  }
  __syncthreads();   // the working memory may be used again
  return Cut{prefix, target};
}

}  // namespace cis
