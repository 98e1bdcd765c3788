// Verification of drafted tokens (gfx950), from what the sampling kernels leave of every row's draw
// (RowKept): which tokens it could take, with what weights and sum, and the token that it took.
#include "cis_select.h"

namespace cis {

// Element j of a lane's own row.
template <class E>
__device__ __forceinline__ float lane_elem(const void* rows, int64_t row_bytes, int64_t row, int j) {
  const char* p = (const char*)rows + row * row_bytes;
  if constexpr (E::kPerVec == 8)
    return __uint_as_float((uint32_t)((const uint16_t*)p)[j] << 16);
  else
    return ((const float*)p)[j];
}
// A token's weight in the distribution that a row was drawn from.
__device__ __forceinline__ uint32_t kept_weight(const RowKept& k, float f, int id) {
  const uint32_t q = draw_weight(f, k.M, k.c);
  return token_of(f, id) >= k.last && q >= k.least_w ? q : 0u;
}
__device__ __forceinline__ void put_token(const VerifyArgs& a, int64_t row, int id, float logp,
                                          float logp_kept) {
  a.ids[row] = id;
  if (a.logp) a.logp[row] = logp;
  if (a.logp_kept) a.logp_kept[row] = logp_kept;
}
__device__ __forceinline__ float kept_logp(const RowKept& k, float f) {
  return (f - k.M) - log1pf(k.rest);
}
__device__ __forceinline__ float kept_share(const RowKept& k, uint32_t w) {
  return (float)log((double)w / (double)k.N);
}

// The weights that a draft which was turned down leaves to its row: max(P - floor(Q rho), 0), or P but for
// the draft where it has no distribution.
template <class E>
struct Leftover {
  static constexpr int EPV = E::kPerVec;
  RowKept p, q;
  double rho;
  __amdgpu_buffer_rsrc_t rp, rq;
  int V, draft;
  bool dist;    // the draft has a distribution
  __device__ __forceinline__ Leftover(const VerifyArgs& a, const VerifyStop& s, int64_t seq)
      : p(a.kept[s.row]), rp(tok_rsrc(a.r, s.row)), V(a.r.V), draft(s.draft), dist(a.r.draft != nullptr) {
    rho = 0.0;
    q = p;
    rq = rp;
    if (dist) {
      const int64_t d = a.r.T1 + s.row - seq;
      q = a.kept[d];
      rq = tok_rsrc(a.r, d);
      rho = (double)p.N / (double)q.N;
    }
  }
  // Of vector v's tokens; `whole`: P itself.
  __device__ __forceinline__ void weights(int v, bool whole, uint32_t (&w)[EPV], float (&f)[EPV]) const {
    float g[EPV];
    tok_vec<E>(rp, v, V, f);
    if (dist) tok_vec<E>(rq, v, V, g);
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      const int id = v * EPV + e;
      w[e] = kept_weight(p, f[e], id);
      if (whole) continue;
      if (dist) {
        const double less = floor((double)kept_weight(q, g[e], id) * rho);
        w[e] = less < (double)w[e] ? w[e] - (uint32_t)less : 0u;
      } else if (id == draft) {
        w[e] = 0;
      }
    }
  }
  // A wave's sum over a chunk.
  __device__ __forceinline__ u64 chunk(int ch, bool whole, int lane) const {
    u64 s = 0;
#pragma unroll 2
    for (int i = 0; i < kScanSlots; ++i) {
      uint32_t w[EPV];
      float f[EPV];
      weights(ch * kScanVecs + i * 64 + lane, whole, w, f);
#pragma unroll
      for (int e = 0; e < EPV; ++e) s += w[e];
    }
    return wave_sum(s);
  }
  // Whether a chunk whose largest logit is m can hold a weight.
  __device__ __forceinline__ bool reaches(float m) const {
    return order_key(m) >= (uint32_t)(p.last >> 32) && (m - p.M) * p.c >= -28.f;
  }
};

// ------------------------------------------------------------------------------------------
// A sequence's drafts, by every wave alike, a lane to a row, up to the first that is turned down; then the
// weights of its row by chunks, a wave's in turn.
// ------------------------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(kVerifyBlock) void cis_verify_kernel(const VerifyArgs a) {
  constexpr int NW = kVerifyBlock / 64;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
  const uint32_t at = blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x - at * (uint32_t)a.parts);
  const int64_t seq = a.seq0 + at, T = a.r.T1;
  const int64_t o0 = sload(a.r.offsets + seq), o1 = sload(a.r.offsets + seq + 1);
  const bool writes = part == 0 && wid == 0;
  if (o0 < 0 || o1 < o0 || o1 > T || (o1 > o0 + 1 && (o0 < seq || o1 - 1 - seq > a.D))) {
    if (writes && lane == 0) {
      a.accepted[seq] = -1;
      a.stops[seq].row = -1;
    }
    return;
  }
  const int64_t n = o1 - o0;
  int64_t stop = n;            // where the sequence ends
  bool turned_down = false;
  int draft = 0;
  for (int64_t i0 = 0; i0 < n; i0 += 64) {
    const int64_t i = i0 + lane, row = o0 + i;
    enum { kTake, kDraw, kEnd } what = kEnd;
    int d = 0;
    float lp = 0.f, lk = 0.f;
    if (i < n) {
      const RowKept k = a.kept[row];
      if (k.id < 0) {
      } else if (i == n - 1) {   // after the last draft
        what = kTake;
        d = k.id;
        lp = k.logp;
        lk = k.logp_kept;
      } else {
        const int64_t id = a.draft_ids[row - seq];
        bool ok = id >= 0 && id < a.r.V;
        double share = (double)k.N;
        if (ok && a.r.draft) {
          const RowKept q = a.kept[T + row - seq];
          ok = q.id >= 0;
          if (ok) {
            const uint32_t w = kept_weight(q, lane_elem<E>(a.r.draft, a.r.draft_bytes, row - seq, (int)id),
                                           (int)id);
            share = (double)w * ((double)k.N / (double)q.N);
          }
        }
        if (ok) {
          d = (int)id;
          const float f = lane_elem<E>(a.r.logits, a.r.row_bytes, row, d);
          const uint32_t w = kept_weight(k, f, d);
          what = (double)a.u[row] * share < (double)w ? kTake : kDraw;
          if (what == kTake) {
            lp = kept_logp(k, f);
            lk = kept_share(k, w);
          }
        }
      }
    }
    const u64 ends = __ballot(what != kTake);
    const int first = ends ? __ffsll(ends) - 1 : 64;
    if (writes && lane < first) put_token(a, row, d, lp, lk);
    if (ends) {
      stop = i0 + first;
      turned_down = __shfl((int)what, first, 64) == kDraw;
      draft = __shfl(d, first, 64);
      break;
    }
  }
  if (turned_down) {   // its draw needs a number
    const float ud = sload(a.u + o1 - 1);
    turned_down = ud >= 0.f && ud < 1.f;
  }
  // (a sequence that goes through ends with the token after its last draft)
  if (writes && lane == 0) {
    a.accepted[seq] = (int32_t)(stop < n ? stop : n > 0 ? n - 1 : 0);
    a.stops[seq] = VerifyStop{turned_down ? o0 + stop : -1, draft};
  }
  if (!turned_down) return;
  const VerifyStop s{o0 + stop, draft};
  const Leftover<E> left(a, s, seq);
  const float* cmax = a.cmax + s.row * a.nch;
  for (int ch = part * NW + wid; ch < a.nch; ch += a.parts * NW) {
    const u64 sum = left.reaches(cmax[ch]) ? left.chunk(ch, false, lane) : 0;
    if (lane == 0) a.left[seq * a.nch + ch] = sum;
  }
}

// ------------------------------------------------------------------------------------------
// The draw in place of a draft, by one workgroup per sequence.
// ------------------------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(kVerifyBlock) void cis_verify_draw_kernel(const VerifyArgs a) {
  constexpr int BLOCK = kVerifyBlock, NW = BLOCK / 64, EPV = E::kPerVec, PV = kScanVecs / BLOCK;
  static_assert(kScanVecs % BLOCK == 0, "a thread has the same number of vectors");
  __shared__ u64 sh[NW];
  __shared__ u64 place[3];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t seq = a.seq0 + blockIdx.x;
  const VerifyStop s{a.stops[seq].row, a.stops[seq].draft};
  if (s.row < 0) return;
  const Leftover<E> left(a, s, seq);
  u64* mass = a.left + seq * a.nch;
  u64 total = 0;
  for (int i = tid; i < a.nch; i += BLOCK) total += mass[i];
  total = block_sum<NW>(total, sh);
  const bool whole = total == 0;
  if (whole) {   // nothing is left: the draw is from the row's own distribution
    for (int ch = wid; ch < a.nch; ch += NW) {
      const u64 m = left.chunk(ch, true, lane);
      if (lane == 0) mass[ch] = m;
    }
    total = left.p.N;
    __syncthreads();
  }
  u64 to = (u64)((double)a.u[sload(a.r.offsets + seq + 1) - 1] * (double)total);
  if (to >= total) to = total - 1;
  if (tid < 64) {
    u64 before = 0;
    for (int i0 = 0; i0 < a.nch; i0 += 64) {
      const u64 m = i0 + lane < a.nch ? mass[i0 + lane] : 0, upto = before + wave_scan(m, lane);
      const u64 hit = __ballot(upto > to);
      if (hit) {
        const int who = __ffsll(hit) - 1;
        before = __shfl(upto - m, who, 64);
        if (lane == 0) {
          place[0] = (u64)(i0 + who);
          place[1] = before;
        }
        break;
      }
      before = __shfl(upto, 63, 64);
    }
  }
  __syncthreads();
  const int v0 = (int)place[0] * kScanVecs + tid * PV;
  uint32_t w[PV][EPV];
  float f[PV][EPV];
  u64 sum = 0;
  static_for<PV>([&](auto J) {
    left.weights(v0 + J, whole, w[J], f[J]);
#pragma unroll
    for (int e = 0; e < EPV; ++e) sum += w[J][e];
  });
  const u64 upto = wave_scan(sum, lane);
  if (lane == 63) sh[wid] = upto;
  __syncthreads();
  u64 before = place[1] + upto - sum;
  for (int k = 0; k < wid; ++k) before += sh[k];
  if (before <= to && to < before + sum) {
    bool found = false;
    static_for<PV>([&](auto J) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        if (!found && before + w[J][e] > to) {
          found = true;
          const int id = (v0 + J) * EPV + e;
          put_token(a, s.row, id, kept_logp(left.p, f[J][e]),
                    kept_share(left.p, kept_weight(left.p, f[J][e], id)));
        }
        before += w[J][e];
      }
    });
  }
}

const void* verify_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_verify_kernel<Bf16>
                           : (const void*)&cis_verify_kernel<F32>;
}
const void* verify_draw_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_verify_draw_kernel<Bf16>
                           : (const void*)&cis_verify_draw_kernel<F32>;
}

}  // namespace cis
