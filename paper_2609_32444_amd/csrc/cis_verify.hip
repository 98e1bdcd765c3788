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
// The same for many tokens of a row: those with a logit above `bound`, and of that logit the ids up to
// `most`. CUT: there is one (else no token lies below).
struct KeptRow {
  float M, c, bound;
  uint32_t least_w, most;
  __device__ __forceinline__ explicit KeptRow(const RowKept& k)
      : M(k.M), c(k.c), bound(k.last ? key_value((uint32_t)(k.last >> 32)) : -INFINITY),
        least_w(k.least_w), most(~(uint32_t)k.last) {}
  template <bool CUT>
  __device__ __forceinline__ uint32_t weight(float f, int id) const {
    const uint32_t q = draw_weight(f, M, c);
    const bool in = !CUT || f > bound || (f == bound && (uint32_t)id <= most);
    return in && q >= least_w ? q : 0u;
  }
};
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
      : p(a.kept[s.row]), rp(tok_rsrc<true>(a.r, s.row)), V(a.r.V), draft(s.draft), dist(a.r.draft != nullptr) {
    rho = 0.0;
    q = p;
    rq = rp;
    if (dist) {
      const int64_t d = a.r.T1 + s.row - seq;
      q = a.kept[d];
      rq = tok_rsrc<true>(a.r, d);
      rho = (double)p.N / (double)q.N;
    }
  }
  // Of vector v's tokens; `whole`: P itself.
  template <bool CUT>
  __device__ __forceinline__ void weights(int v, bool whole, uint32_t (&w)[EPV], float (&f)[EPV]) const {
    float g[EPV];
    tok_vec<E>(rp, v, V, f);
    if (dist) tok_vec<E>(rq, v, V, g);
    const KeptRow kp(p), kq(q);
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      const int id = v * EPV + e;
      w[e] = kp.weight<CUT>(f[e], id);
      if (whole) continue;
      if (dist) {
        const uint32_t less =
            (uint32_t)fmin((double)kq.weight<CUT>(g[e], id) * rho, 0x1p32 - 1.0);   // (its floor)
        w[e] -= less < w[e] ? less : w[e];
      } else if (id == draft) {
        w[e] = 0;
      }
    }
  }
  __device__ __forceinline__ bool cut() const { return (p.last | q.last) != 0; }
  // A wave's sum over a piece of the row.
  template <bool CUT>
  __device__ __forceinline__ u64 piece_of(int sub, bool whole, int lane) const {
    u64 s = 0;
    static_for<kLeftVecs / 64>([&](auto I) __attribute__((always_inline)) {
      uint32_t w[EPV], vs = 0;   // (8 weights stay below 2^32)
      float f[EPV];
      weights<CUT>(sub * kLeftVecs + I * 64 + lane, whole, w, f);
#pragma unroll
      for (int e = 0; e < EPV; ++e) vs += w[e];
      s += vs;
    });
    return wave_sum(s);
  }
  __device__ __forceinline__ u64 piece(int sub, bool whole, int lane) const {
    return cut() ? piece_of<true>(sub, whole, lane) : piece_of<false>(sub, whole, lane);
  }
  // Whether a chunk whose largest logit is m can hold a weight.
  __device__ __forceinline__ bool reaches(float m) const {
    return order_key(m) >= (uint32_t)(p.last >> 32) && (m - p.M) * p.c >= -28.f;
  }
};

// ------------------------------------------------------------------------------------------
// What the scan's sums decide of uncut rows at temperature 1, by one workgroup per sequence: drafts that are
// surely accepted or surely turned down, and so which rows have to be looked at: those of the target up
// to the first that is surely turned down, and the drafts' up to there that are not surely accepted.
//
// The scan's S = sum of exp(z - M) is within 2^-16 of what its float32 exponents (28 * 2^-24 and less where
// a weight is not 0), exp2 and sums of 8 add up to, and a token's weight is below 2^28 exp(z - M) by less than
// 1, so that N lies in [2^28 S (1 - 2^-16) - V, 2^28 S (1 + 2^-16)]. What holds for both ends of N and N', with
// 2^-40 for the comparison's own roundings, holds for what they are; all else stays open. A row with a NaN or
// an infinity, or without a token, has a NaN sum, and nothing that is compared with it holds.
// ------------------------------------------------------------------------------------------
struct SumRange {
  float M;
  double lo, hi;
};
__device__ __forceinline__ SumRange sum_range(const VerifyArgs& a, int64_t row, int lane) {
  const float* cmax = a.cmax + row * a.nch;
  const double* csum = a.csum + row * a.nch;
  float M = -INFINITY;
  for (int i = lane; i < a.nch; i += 64) M = fmaxf(M, cmax[i]);
  M = wave_max(M);
  double S = 0.0;
  for (int i = lane; i < a.nch; i += 64)
    S += csum[i] * (double)fast_exp2((cmax[i] - M) * kLog2e);
  S = wave_sum(S) * (double)kDrawOne;
  return SumRange{M, S * (1 - 0x1p-16) - (double)a.r.V, S * (1 + 0x1p-16)};
}
template <class E>
__global__ __launch_bounds__(kVerifyBlock) void cis_verdict_kernel(const VerifyArgs a) {
  constexpr int NW = kVerifyBlock / 64;
  __shared__ int64_t first[NW];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
  const int64_t seq = a.seq0 + blockIdx.x, T = a.r.T1;
  const int64_t o0 = sload(a.r.offsets + seq), o1 = sload(a.r.offsets + seq + 1);
  if (o0 < 0 || o1 <= o0 || o1 > T || (o1 > o0 + 1 && (o0 < seq || o1 - 1 - seq > a.D))) return;
  int64_t stop = o1;   // the first row whose draft is surely turned down
  for (int64_t row = o0 + wid; row < o1 - 1; row += NW) {
    const int64_t id = sload(a.draft_ids + row - seq);
    const float u = sload(a.u + row);
    uint8_t v = kOpen;
    if (id >= 0 && id < a.r.V && u >= 0.f && u < 1.f) {
      const SumRange p = sum_range(a, row, lane);
      const double w = (double)draw_weight(lane_elem<E>(a.r.logits, a.r.row_bytes, row, (int)id), p.M, kLog2e);
      double most = p.hi, least = p.lo;   // of what u is multiplied by
      if (a.r.draft) {
        const SumRange q = sum_range(a, T + row - seq, lane);
        const double wq = (double)draw_weight(
            lane_elem<E>(a.r.draft, a.r.draft_bytes, row - seq, (int)id), q.M, kLog2e);
        most = q.lo > 0.0 ? wq * (p.hi / q.lo) : INFINITY;
        least = wq * (p.lo / q.hi);
      }
      if ((double)u * most * (1 + 0x1p-40) < w) v = kAccepted;
      if (least > 0.0 && (double)u * least * (1 - 0x1p-40) >= w) v = kTurnedDown;
    }
    if (lane == 0) a.verdict[row] = v;
    if (v == kTurnedDown && row < stop) stop = row;
  }
  if (lane == 0) first[wid] = stop;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NW; ++k) stop = first[k] < stop ? first[k] : stop;
  for (int64_t row = o0 + threadIdx.x; row < o1; row += kVerifyBlock) {
    a.need[row] = row <= stop;
    if (row < o1 - 1 && a.r.draft) a.need[T + row - seq] = row <= stop && a.verdict[row] != kAccepted;
  }
}

// ------------------------------------------------------------------------------------------
// A sequence's drafts, a lane to a row, up to the first that is turned down, by the first wave of each of
// its workgroups (of which one writes); then the weights that are left of its row, a piece to a wave: some 30
// instructions a token, two exp2 and a product in double among them. Bound by the latency of both steps: 13 us
// for 64 sequences of 4 drafts over V = 151936, 8 for one, 4.6 where rows are of one token. (Pieces of 512
// vectors 17 and 16 us; judged by every wave, logarithms too, 19.)
// ------------------------------------------------------------------------------------------
template <class E>
__device__ __forceinline__ VerifyStop judge(const VerifyArgs& a, int64_t seq, bool writes) {
  const int lane = threadIdx.x & 63;
  const int64_t o0 = sload(a.r.offsets + seq), o1 = sload(a.r.offsets + seq + 1), T = a.r.T1;
  if (o0 < 0 || o1 < o0 || o1 > T || (o1 > o0 + 1 && (o0 < seq || o1 - 1 - seq > a.D))) {
    if (writes && lane == 0) a.accepted[seq] = -1;
    return VerifyStop{-1, 0};
  }
  const int64_t n = o1 - o0;
  int64_t stop = n;            // where the sequence ends
  bool turned_down = false;
  int draft = 0;
  for (int64_t i0 = 0; i0 < n; i0 += 64) {
    const int64_t i = i0 + lane, row = o0 + i;
    enum { kTake, kDraw, kEnd } what = kEnd;
    int d = 0;
    uint32_t w = 0;
    float f = 0.f;
    RowKept k;
    k.id = -1;
    const bool drafted = i < n - 1;
    int64_t id = -1;
    float u = 0.f;
    if (i < n) k = a.kept[row];
    if (drafted) {
      id = a.draft_ids[row - seq];
      u = a.u[row];
    }
    const uint8_t verdict = drafted && a.verdict ? a.verdict[row] : kOpen;
    if (k.id >= 0 && !drafted) {   // after the last draft
      what = kTake;
      d = k.id;
    } else if (verdict != kOpen) {
      d = (int)id;
      f = lane_elem<E>(a.r.logits, a.r.row_bytes, row, d);
      w = kept_weight(k, f, d);
      what = verdict == kAccepted ? kTake : kDraw;
    } else if (k.id >= 0 && id >= 0 && id < a.r.V) {
      d = (int)id;
      f = lane_elem<E>(a.r.logits, a.r.row_bytes, row, d);
      w = kept_weight(k, f, d);
      double share = (double)k.N;
      bool ok = true;
      if (a.r.draft) {
        const RowKept q = a.kept[T + row - seq];
        const float g = lane_elem<E>(a.r.draft, a.r.draft_bytes, row - seq, d);
        ok = q.id >= 0;
        share = (double)kept_weight(q, g, d) * ((double)k.N / (double)q.N);
      }
      if (ok) what = (double)u * share < (double)w ? kTake : kDraw;
    }
    const u64 ends = __ballot(what != kTake);
    const int first = ends ? __ffsll(ends) - 1 : 64;
    if (writes && lane < first) {
      if (drafted)
        put_token(a, row, d, kept_logp(k, f), kept_share(k, w));
      else
        put_token(a, row, d, k.logp, k.logp_kept);
    }
    if (ends) {
      stop = i0 + first;
      turned_down = __shfl((int)what, first, 64) == kDraw;
      draft = __shfl(d, first, 64);
      break;
    }
  }
  if (turned_down) {
    const RowKept k = a.kept[o0 + stop];
    const float u = sload(a.u + o1 - 1);
    turned_down = u >= 0.f && u < 1.f;   // (its draw needs a number)
    if (turned_down && k.N == kDrawOne) {
      // a distribution of one token: the largest logit's weight, and nothing besides
      if (writes && lane == 0) put_token(a, o0 + stop, k.id, k.logp, k.logp_kept);
      turned_down = false;
    }
  }
  // (a sequence that goes through ends with the token after its last draft)
  if (writes && lane == 0) a.accepted[seq] = (int32_t)(stop < n ? stop : n > 0 ? n - 1 : 0);
  return VerifyStop{turned_down ? o0 + stop : -1, draft};
}

template <class E>
__global__ __launch_bounds__(kVerifyBlock) void cis_verify_kernel(const VerifyArgs a) {
  constexpr int NW = kVerifyBlock / 64;
  __shared__ VerifyStop shared;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x) >> 6;
  const uint32_t at = blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x - at * (uint32_t)a.parts);
  const int64_t seq = a.seq0 + at;
  if (wid == 0) {
    const VerifyStop j = judge<E>(a, seq, part == 0);
    if (lane == 0) {
      shared = j;
      if (part == 0) a.stops[seq] = j;
    }
  }
  __syncthreads();
  const VerifyStop s = shared;
  if (s.row < 0) return;
  const Leftover<E> left(a, s, seq);
  const float* cmax = a.cmax + s.row * a.nch;
  for (int sub = part * NW + wid; sub < a.nsub; sub += a.parts * NW) {
    const u64 sum = left.reaches(cmax[sub / (kScanVecs / kLeftVecs)]) ? left.piece(sub, false, lane) : 0;
    if (lane == 0) a.left[seq * a.nsub + sub] = sum;
  }
}

// ------------------------------------------------------------------------------------------
// The draw in place of a draft, by one workgroup per sequence: 8 us, by the latency of its steps.
// ------------------------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(kVerifyBlock) void cis_verify_draw_kernel(const VerifyArgs a) {
  constexpr int BLOCK = kVerifyBlock, NW = BLOCK / 64, EPV = E::kPerVec;
  static_assert(kLeftVecs <= BLOCK, "a thread has one vector of a piece");
  __shared__ u64 sh[NW];
  __shared__ u64 place[2];   // the piece, and the sum ahead of it
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t seq = a.seq0 + blockIdx.x;
  const VerifyStop s{a.stops[seq].row, a.stops[seq].draft};
  if (s.row < 0) return;
  const Leftover<E> left(a, s, seq);
  u64* mass = a.left + seq * a.nsub;
  u64 total = 0;
  for (int i = tid; i < a.nsub; i += BLOCK) total += mass[i];
  total = block_sum<NW>(total, sh);
  const bool whole = total == 0;
  if (whole) {   // nothing is left: the draw is from the row's own distribution
    for (int sub = wid; sub < a.nsub; sub += NW) {
      const u64 m = left.piece(sub, true, lane);
      if (lane == 0) mass[sub] = m;
    }
    total = left.p.N;
    __syncthreads();
  }
  u64 to = (u64)((double)a.u[sload(a.r.offsets + seq + 1) - 1] * (double)total);
  if (to >= total) to = total - 1;
  if (tid < 64) {
    u64 before = 0;
    for (int i0 = 0; i0 < a.nsub; i0 += 64) {
      const u64 m = i0 + lane < a.nsub ? mass[i0 + lane] : 0, upto = before + wave_scan(m, lane);
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
  uint32_t w[EPV];
  float f[EPV];
  u64 sum = 0;
  const int v = (int)place[0] * kLeftVecs + tid;
  if (tid < kLeftVecs) {
    left.template weights<true>(v, whole, w, f);
#pragma unroll
    for (int e = 0; e < EPV; ++e) sum += w[e];
  }
  const u64 upto = wave_scan(sum, lane);
  if (lane == 63) sh[wid] = upto;
  __syncthreads();
  u64 before = place[1] + upto - sum;
  for (int k = 0; k < wid; ++k) before += sh[k];
  if (before <= to && to < before + sum) {
    bool found = false;
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      if (!found && before + w[e] > to) {
        found = true;
        const int id = v * EPV + e;
        put_token(a, s.row, id, kept_logp(left.p, f[e]),
                  kept_share(left.p, kept_weight(left.p, f[e], id)));
      }
      before += w[e];
    }
  }
}

const void* verdict_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_verdict_kernel<Bf16>
                           : (const void*)&cis_verdict_kernel<F32>;
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
