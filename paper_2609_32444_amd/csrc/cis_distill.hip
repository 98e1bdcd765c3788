// Distillation kernels (gfx950): a fused pass that holds a row on the compute unit, and a pass in
// parts (scan, a wave per row or four, gradient by segments) for the forward direction and for few rows.
#include "cis_distill.h"
#include "cis_select.h"
#include "cis_stats.h"

namespace cis {

// ------------------------------------------------------------------------------------------
// Fused forward and backward: one workgroup per row, which it reads once and holds in registers (the
// first NV vectors of every thread; longer rows read the rest a second time). The list goes into a
// table in LDS, hashed by the vector that a token lies in, with chains, and every thread has a bit for
// each of its vectors that holds one: the first sweep leaves the listed tokens out of its sum and notes
// their logits, the second puts their gradients in. Bound by the memory: 16384 rows of V = 151936 in
// 1.88 ms (5.3 TB/s of reads and writes); the list's table and the loss by one wave lie between the
// sweeps of a row, where the compute unit has no other row's loads to turn to.
// ------------------------------------------------------------------------------------------
template <int BLOCK, int KMAX>
struct FusedShared {
  static constexpr int kTable = BLOCK == 1024 ? 8192 : BLOCK == 512 ? 4096 : BLOCK == 256 ? 2048 : 1024;
  uint32_t head[kTable];
  uint32_t next[KMAX];
  uint32_t mine[BLOCK];   // a thread's vectors (the first 32) with listed tokens
  ListShared<KMAX> list;
  float f[16], g[16];
  uint32_t u[16];
  RestGrad rest;
  Teacher teacher;
};

// A barrier for what lies in LDS: loads of the row stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <class E, int BLOCK, int NV, int KMAX>
__global__ __launch_bounds__(BLOCK) __attribute__((amdgpu_waves_per_eu(4))) void cis_distill_kernel(
    const DistillArgs a) {
  constexpr int NW = BLOCK / 64, EPV = E::kPerVec;
  // vectors that are asked for before the list, and stay in flight ahead of sweep 1 (16384 rows of
  // V = 151936: 4 1903 us, 8 1867, 12 2081; 3001 of V = 50257: 144, 148, 154)
  constexpr int MOST = BLOCK == 1024 ? 8 : 4, FIRST = NV > MOST ? MOST : NV;
  typedef FusedShared<BLOCK, KMAX> Shared;
  __shared__ Shared sh;
  for (int i = threadIdx.x; i < Shared::kTable; i += BLOCK) sh.head[i] = kNone;
  sh.mine[threadIdx.x] = 0;
  // Rows by rounds of the grid. From round to round a workgroup moves on by a few places, so that it does
  // not meet the same place of every response (padding is periodic).
  constexpr uint32_t kShift = 61;
  uint32_t place = blockIdx.x;
  // a thread's first entry of the list is fetched a row ahead
  int32_t id0 = -1;
  float value0 = 0.f;
  auto fetch = [&](int64_t row, int tid) {
    if (row < a.r.T && tid < a.K) {
      id0 = a.ids[row * a.ld_top + tid];
      value0 = a.values[row * a.ld_top + tid];
    }
  };
  fetch(blockIdx.x, threadIdx.x);
  bool old = false;   // the table holds the last row's list
  for (int64_t round = 0; round < a.r.T; round += gridDim.x) {
    const int64_t row = round + place;
    if (row >= a.r.T) break;   // (the last round)
    if (gridDim.x > kShift) {
      place += kShift;
      if (place >= gridDim.x) place -= gridDim.x;
    }
    const int64_t next = round + gridDim.x + place;
    // (what follows from these is formed again for every row: kept, it would take up the registers)
    int tid = threadIdx.x, nvec = a.r.nvec;
    asm volatile("" : "+v"(tid));
    asm volatile("" : "+s"(nvec));
    const int lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid) >> 6;
    const int V = a.r.V, K = a.K;
    const float c = a.c;
    const bool on = tok_on(a.r, row);
    const __amdgpu_buffer_rsrc_t rs =
        make_rsrc((const char*)a.r.logits + row * a.r.row_bytes, on ? (uint32_t)nvec * 16u : 0u);
    u32x4 r[NV];
    static_for<FIRST>([&](auto I) {
      r[I] = bload(rs, (uint32_t)(I * BLOCK + tid) * 16u, 0u);
      slot_fence();
    });
    const float tail = row_tail(a, row), weight = row_weight(a, row);
    // the table
    uint32_t seen = 0, wrong = 0;   // entries; ids out of range or repeated
    lds_barrier();   // (nobody looks the last row's vectors up any more)
    if (old)
      for (int k = tid; k < K; k += BLOCK)
        if (sh.list.id[k] >= 0) sh.head[(sh.list.id[k] / EPV) & (Shared::kTable - 1)] = kNone;
    old = on;
    lds_barrier();
    if (on)
      for (int k = tid; k < K; k += BLOCK) {
        const int32_t id = k < BLOCK ? id0 : a.ids[row * a.ld_top + k];
        sh.list.lq[k] = k < BLOCK ? value0 : a.values[row * a.ld_top + k];
        const bool in = id >= 0 && id < V;
        sh.list.id[k] = in ? id : -1;
        sh.next[k] = kNone;
        if (in) {
          const int v = id / EPV;
          sh.next[k] = atomicExch(&sh.head[v & (Shared::kTable - 1)], (uint32_t)k);
          if (v < NV * BLOCK) atomicOr(&sh.mine[v & (BLOCK - 1)], 1u << (v / BLOCK));
        }
        seen |= in ? 1u : 0u;
        wrong |= in || id == -1 ? 0u : 1u;
      }
    lds_barrier();
    if (on)
      for (int k = tid; k < K; k += BLOCK)
        if (sh.list.id[k] >= 0)
          for (uint32_t o = sh.next[k]; o != kNone; o = sh.next[o])
            wrong |= sh.list.id[o] == sh.list.id[k] ? 1u : 0u;
    if (lane == 0) sh.u[wid] = 0;
    if (__ballot(seen | wrong)) {
      const uint32_t any = (__ballot(seen) ? 1u : 0u) | (__ballot(wrong) ? 2u : 0u);
      if (lane == 0) sh.u[wid] = any;
    }
    lds_barrier();
    uint32_t any = 0;
    for (int w = 0; w < NW; ++w) any |= sh.u[w];
    const bool bad = (any & 2u) != 0, valid = on && any == 1u;
    // f(entry, element) for the listed tokens of vector v
    auto each_listed = [&](int v, auto&& f) {
      for (uint32_t k = sh.head[v & (Shared::kTable - 1)]; k != kNone; k = sh.next[k])
        if (sh.list.id[k] / EPV == v) f(k, sh.list.id[k] % EPV);
    };
    const uint32_t mine = sh.mine[tid];
    // sweep 1: the tokens that are not listed
    float R = -FLT_MAX, s = 0.f;   // the largest of them, and the sum of exponentials relative to it
    auto fold = [&](int v, u32x4 x, bool listed, bool last) {
      float f[EPV];
      E::unpack(x, f);
      if (last) mask_past_end<E>(f, v, V);
      if (listed)
        each_listed(v, [&](uint32_t k, int at) {
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (at == e) {
              sh.list.z[k] = f[e];
              f[e] = -INFINITY;
            }
        });
      float m = f[0];
#pragma unroll
      for (int e = 1; e < EPV; ++e) m = fmaxf(m, f[e]);
      const float Rn = fmaxf(R, m);
      float part = 0.f;
#pragma unroll
      for (int e = 0; e < EPV; ++e) part += fast_exp2((f[e] - Rn) * c);
      s = s * fast_exp2((R - Rn) * c) + part;
      R = Rn;
    };
    if (valid && wid == 0) {
      const Teacher t = teacher_list(a, tail, sh.list, lane);
      if (lane == 0) sh.teacher = t;   // (rather than in every thread's registers)
    }
    // (a row that does not count has no records: nothing is read)
    static_for<NV>([&](auto I) {
      if constexpr (I + FIRST < NV) {
        r[I + FIRST] = bload(rs, (uint32_t)((I + FIRST) * BLOCK + tid) * 16u, 0u);
        slot_fence();
      }
      if (valid && I * BLOCK < nvec)
        fold(I * BLOCK + tid, r[I], mine >> I & 1, (I + 1) * BLOCK * EPV > V);
      slot_fence();
    });
    if (valid) {
      for (int v = NV * BLOCK + tid; v < nvec; v += BLOCK)
        fold(v, bload_aux<kAuxStream1>(rs, (uint32_t)v * 16u), true, (v + 1) * EPV > V);
      wave_lse(R, s, c);
      if (lane == 0) {
        sh.f[wid] = R;
        sh.g[wid] = s;
      }
    }
    lds_barrier();
    if (wid == 0) {
      Student st{0.f, RestGrad{0.f, 0.f, 0.f}, true};
      if (valid) {
        R = lane < NW ? sh.f[lane] : -FLT_MAX;
        s = lane < NW ? sh.g[lane] : 0.f;
        wave_lse(R, s, c);
        st = student_list<E, true>(a, weight, sh.list, lane, sh.teacher, R, s);
      }
      if (lane == 0) {
        put_row(a, row, st.term, valid, on && bad, st.finite);
        sh.rest = st.rest;
      }
    }
    lds_barrier();
    // sweep 2
    const RestGrad g = sh.rest;
    const bool others = valid && g.g != 0.f;   // (else 0, whatever the logits are)
    opaque(r);
    fetch(next, tid);
    void* grow = (char*)a.dlogits + row * a.grow_bytes;
    const bool ragged = V % EPV != 0;
    const __amdgpu_buffer_rsrc_t ws = make_rsrc(grow, (uint32_t)(nvec - (ragged ? 1 : 0)) * 16u);
    auto put = [&](int v, u32x4 x, bool listed, bool last) {
      u32x4 out{0u, 0u, 0u, 0u};
      if (others) out = rest_vec<E>(x, c, g);
      if (valid && listed)
        each_listed(v, [&](uint32_t k, int e) { out = E::set(out, e, sh.list.grad[k]); });
      bstore(out, ws, (uint32_t)v * 16u, 0u);
      if (last && ragged && v == nvec - 1)
        for (int e = 0; e < V - v * EPV; ++e) E::store_elem(grow, v * EPV + e, E::elem_bits(out, e));
    };
    static_for<NV>([&](auto I) {
      if (I * BLOCK < nvec) put(I * BLOCK + tid, r[I], mine >> I & 1, (I + 1) * BLOCK >= nvec);
      slot_fence();
    });
    for (int v = NV * BLOCK + tid; v < nvec; v += BLOCK)
      put(v, bload_aux<kAuxStream2>(rs, (uint32_t)v * 16u), true, true);
    sh.mine[tid] = 0;
  }
}

// ------------------------------------------------------------------------------------------
// In parts, 2: NW waves per row (4 for few rows). The scan has left the chunks' sums over all tokens; the vectors that
// hold listed ones are read again, and taken out of the sums but for what else they hold (the sums
// are in double, and a vector's sum is the same bits wherever it is formed). Where less than 2^-28
// of the row remains, the row is summed again without the listed tokens. The vectors are found
// in a table in LDS: open addressing, a key and the listed tokens of the vector as bits. Bound by the
// latency of a row's steps: 8192 rows, K = 64, in 15 us.
// ------------------------------------------------------------------------------------------
template <int KMAX>
struct RowShared {
  static constexpr int kTable = 4 * KMAX;
  uint32_t key[kTable];
  uint32_t bits[kTable];
  uint16_t slot[KMAX];
  ListShared<KMAX> list;
  Teacher teacher;
  uint32_t u[4];
  double d[4];
};

template <class E, bool BWD, int KMAX, int NW>
__global__ __launch_bounds__(64 * NW) void cis_distill_row_kernel(const DistillArgs a) {
  constexpr int EPV = E::kPerVec, BLOCK = 64 * NW;
  typedef RowShared<KMAX> Shared;
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid) >> 6;
  const int V = a.r.V, nvec = a.r.nvec, K = a.K, nch = a.s.nch;
  const float c = a.c;
  const int64_t row = a.row0 + blockIdx.x;
  const bool on = tok_on(a.r, row);
  const float* cmax = a.s.cmax + row * nch;
  const double* csum = a.s.csum + row * nch;
  uint32_t seen = 0, wrong = 0;
  for (int i = tid; i < Shared::kTable; i += BLOCK) sh.key[i] = kNone;
  for (int i = tid; i < Shared::kTable; i += BLOCK) sh.bits[i] = 0;
  __syncthreads();
  if (on)
    for (int k = tid; k < K; k += BLOCK) {
      const int32_t id = a.ids[row * a.ld_top + k];
      sh.list.lq[k] = a.values[row * a.ld_top + k];
      const bool in = id >= 0 && id < V;
      sh.list.id[k] = in ? id : -1;
      if (in) {
        const uint32_t v = (uint32_t)(id / EPV);
        uint32_t at = (v * 0x9E3779B1u >> 16) & (Shared::kTable - 1);
        for (;; at = (at + 1) & (Shared::kTable - 1)) {   // (a quarter full at most)
          const uint32_t was = atomicCAS(&sh.key[at], kNone, v);
          if (was == kNone || was == v) break;
        }
        const uint32_t bit = 1u << (id % EPV);
        wrong += atomicOr(&sh.bits[at], bit) & bit ? 1 : 0;
        sh.slot[k] = (uint16_t)at;
        ++seen;
      } else {
        wrong += id != -1 ? 1 : 0;
      }
    }
  seen = block_sum<NW>(seen | wrong << 16, sh.u);   // (K entries at most, in each)
  const bool bad = seen >> 16 != 0, valid = on && !bad && seen != 0;
  Student st{0.f, RestGrad{0.f, 0.f, 0.f}, true};
  if (valid) {
    const __amdgpu_buffer_rsrc_t rs = tok_rsrc(a.r, row);
    float M = -INFINITY;
    for (int i = lane; i < nch; i += 64) M = fmaxf(M, cmax[i]);
    M = sum_ref(wave_max(M));
    double whole = 0.0, less = 0.0;
    for (int i = lane; i < nch; i += 64)
      if (!(cmax[i] == -INFINITY && csum[i] == 0.0))
        whole += csum[i] * (double)fast_exp2((cmax[i] - M) * c);
    if (wid == NW - 1) {
      const Teacher t = teacher_list(a, row_tail(a, row), sh.list, lane);
      if (lane == 0) sh.teacher = t;
    }
    for (int k = tid; k < K; k += BLOCK) {
      const int id = sh.list.id[k];
      if (id < 0) continue;
      const int v = id / EPV;
      const uint32_t bits = sh.bits[sh.slot[k]];
      float f[EPV];
      tok_vec<E>(rs, v, V, f);
      const float m = sum_ref(cmax[v / kScanVecs]);
      const float all = vec_sum<E>(f, c, m);
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        if (id % EPV == e) sh.list.z[k] = f[e];
        if (bits >> e & 1) f[e] = -INFINITY;
      }
      if (id % EPV == __ffs(bits) - 1)   // once for every vector
        less += ((double)all - (double)vec_sum<E>(f, c, m)) * (double)fast_exp2((m - M) * c);
    }
    whole = wave_sum(whole);
    double rest = whole - block_sum<NW>(less, sh.d);
    if (wid != 0) return;   // (no barrier follows)
    float R = M, s = (float)rest;
    if (!(rest > whole * 0x1p-28)) {
      R = -FLT_MAX;
      s = 0.f;
      for (int v = lane; v < nvec; v += 64) {
        float f[EPV];
        tok_vec<E>(rs, v, V, f);
        uint32_t at = ((uint32_t)v * 0x9E3779B1u >> 16) & (Shared::kTable - 1), bits = 0;
        for (; sh.key[at] != kNone; at = (at + 1) & (Shared::kTable - 1))
          if (sh.key[at] == (uint32_t)v) {
            bits = sh.bits[at];
            break;
          }
        float m = -INFINITY, part = 0.f;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
          if (bits >> e & 1) f[e] = -INFINITY;
          m = fmaxf(m, f[e]);
        }
        const float Rn = fmaxf(R, m);
#pragma unroll
        for (int e = 0; e < EPV; ++e) part += fast_exp2((f[e] - Rn) * c);
        s = s * fast_exp2((R - Rn) * c) + part;
        R = Rn;
      }
      wave_lse(R, s, c);
    }
    st = student_list<E, BWD>(a, row_weight(a, row), sh.list, lane, sh.teacher, R, s);
  }
  if (wid != 0) return;
  if (lane == 0) put_row(a, row, st.term, valid, on && bad, st.finite);
  if (BWD) {
    if (lane == 0) {
      a.rest[row] = st.rest;
      a.valid[row] = valid ? 1 : 0;
    }
    for (int k = lane; k < K; k += 64)
      a.grads[row * K + k] = valid && sh.list.id[k] >= 0 ? sh.list.grad[k] : 0u;
  }
}

// ------------------------------------------------------------------------------------------
// In parts, 3: the gradient by segments of kGradVecs vectors; listed tokens are put in by the segment
// that they lie in, once its own stores are done. The first workgroup sums up the call's statistics
// too: there are few rows, and they were done before the launch. 96 rows of V = 151936 in 14 us (4.3 TB/s).
// ------------------------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(kDistillGradBlock) void cis_distill_grad_kernel(const DistillArgs a) {
  constexpr int EPV = E::kPerVec, BLOCK = kDistillGradBlock, K = kDistillGradVecs / BLOCK;
  const int tid = threadIdx.x;
  const int64_t b = a.row0 + blockIdx.x, row = b / a.nseg;
  const int seg = (int)(b - row * a.nseg);
  const bool valid = a.valid[row] != 0;
  const RestGrad g = a.rest[row];
  const bool others = valid && g.g != 0.f;   // (else 0, whatever the logits are)
  const bool ragged = a.r.V % EPV != 0;
  const __amdgpu_buffer_rsrc_t rs =
      make_rsrc((const char*)a.r.logits + row * a.r.row_bytes, others ? (uint32_t)a.r.nvec * 16u : 0u);
  void* grow = (char*)a.dlogits + row * a.grow_bytes;
  const __amdgpu_buffer_rsrc_t ws =
      make_rsrc(grow, (uint32_t)(a.r.nvec - (ragged ? 1 : 0)) * 16u);
  const int v0 = seg * kDistillGradVecs + tid;
  u32x4 r[K];
  static_for<K>([&](auto I) { r[I] = bload(rs, (uint32_t)(v0 + I * BLOCK) * 16u, 0u); });
  static_for<K>([&](auto I) {
    const int v = v0 + I * BLOCK;
    const u32x4 out = others ? rest_vec<E>(r[I], a.c, g) : u32x4{0u, 0u, 0u, 0u};
    bstore(out, ws, (uint32_t)v * 16u, 0u);
    if (ragged && v == a.r.nvec - 1)
      for (int e = 0; e < a.r.V - v * EPV; ++e)
        E::store_elem(grow, v * EPV + e, E::elem_bits(out, e));
  });
  if (valid) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int k = tid; k < a.K; k += BLOCK) {
      const int id = a.ids[row * a.ld_top + k];
      if (id >= 0 && id / EPV / kDistillGradVecs == seg)
        E::store_elem(grow, id, a.grads[row * a.K + k]);
    }
  }
  if (b != 0) return;
  RowStats st{};
  for (int64_t t = tid; t < a.r.T; t += BLOCK)
    take_row(st, a.terms_ws[t], a.flags_ws[t], a.logk_ws[t], a.excess_ws[t]);
  st = block_stats<BLOCK>(st);
  if (tid == 0) write_stats(a.fin, st);
}

// Variants of the fused pass: the first that holds a row. 1024 x 19 vectors take 76 of a thread's
// 128 registers (10 others lie in scratch in bf16 and 6 in float32; no other variant has any); longer rows
// read the rest twice.
struct FusedVariant {
  int block, nv;
  const void *few, *many;   // lists of up to 256 and 1024 entries
};
#define CIS_FUSED(E, B, N)                                         \
  FusedVariant {                                                   \
    B, N, (const void*)&cis_distill_kernel<E, B, N, 256>,          \
        (const void*)&cis_distill_kernel<E, B, N, CIS_TOP_MAX_K>   \
  }
#define CIS_FUSED_TABLE(E)                                                                   \
  {CIS_FUSED(E, 64, 5),    CIS_FUSED(E, 64, 10),   CIS_FUSED(E, 64, 18),  CIS_FUSED(E, 256, 8),  \
   CIS_FUSED(E, 256, 12),  CIS_FUSED(E, 256, 16),  CIS_FUSED(E, 512, 10), CIS_FUSED(E, 512, 13), \
   CIS_FUSED(E, 512, 17),  CIS_FUSED(E, 1024, 12), CIS_FUSED(E, 1024, 15), CIS_FUSED(E, 1024, 19)}
static const FusedVariant kFusedBf16[] = CIS_FUSED_TABLE(Bf16);
static const FusedVariant kFusedF32[] = CIS_FUSED_TABLE(F32);

DistillVariant distill_fused(int dtype, int32_t nvec, int64_t K) {
  const FusedVariant* t = dtype == CIS_BF16 ? kFusedBf16 : kFusedF32;
  constexpr int n = sizeof(kFusedBf16) / sizeof(kFusedBf16[0]);
  int i = 0;
  while (i < n - 1 && (int64_t)t[i].block * t[i].nv < nvec) ++i;
  return DistillVariant{t[i].block, K <= 256 ? t[i].few : t[i].many};
}

// (A forward call of 96 rows of V = 151936, K = 256: 17.7 us by 4 waves a row, 22.0 by one. With the
// gradient, rows that go in parts are always few.)
const void* distill_row_kernel(int dtype, bool bwd, int64_t K, bool few) {
#define CIS_ROW_N(E, B, N)                                               \
  (K <= 64 ? (const void*)&cis_distill_row_kernel<E, B, 64, N>           \
   : K <= 256 ? (const void*)&cis_distill_row_kernel<E, B, 256, N>       \
              : (const void*)&cis_distill_row_kernel<E, B, CIS_TOP_MAX_K, N>)
#define CIS_ROW(E) \
  (bwd ? CIS_ROW_N(E, true, 4) : few ? CIS_ROW_N(E, false, 4) : CIS_ROW_N(E, false, 1))
  return dtype == CIS_BF16 ? CIS_ROW(Bf16) : CIS_ROW(F32);
#undef CIS_ROW
#undef CIS_ROW_N
}
const void* distill_grad_kernel(int dtype) {
  return dtype == CIS_BF16 ? (const void*)&cis_distill_grad_kernel<Bf16>
                           : (const void*)&cis_distill_grad_kernel<F32>;
}

}  // namespace cis
