// C-ABI entry points of the token operators (cis_tokens.h): argument checks, launch configuration and
// launches on the caller's stream. No device memory is allocated and nothing synchronises.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <mutex>

#include "cis_tok.h"

namespace {

constexpr int64_t kMaxV = int64_t(1) << 28;
constexpr int kMaxDevices = 64;

// Compute units of the current device, or CIS_ERR_DEVICE.
int device_cus() {
  static std::mutex mu;
  static int cus[kMaxDevices] = {};   // 0: not looked at yet
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return CIS_ERR_DEVICE;
  std::lock_guard<std::mutex> lk(mu);
  if (cus[dev] == 0) {
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return CIS_ERR_DEVICE;
    cus[dev] = strncmp(prop.gcnArchName, "gfx950", 6) == 0 ? prop.multiProcessorCount
                                                           : CIS_ERR_DEVICE;
  }
  return cus[dev];
}

// Workgroups of a kernel that a compute unit holds at once. (The devices are all gfx950.)
int blocks_per_cu(const void* fn, int block) {
  static std::mutex mu;
  static struct {
    const void* fn;
    int n;
  } seen[64];
  static int count = 0;
  std::lock_guard<std::mutex> lk(mu);
  for (int i = 0; i < count; ++i)
    if (seen[i].fn == fn) return seen[i].n;
  int n = 0;
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, fn, block, 0) != hipSuccess || n < 1) n = 1;
  if (count < 64) seen[count++] = {fn, n};
  return n;
}

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool known(int dtype) { return dtype == CIS_BF16 || dtype == CIS_F32; }
int elem_bytes(int dtype) { return dtype == CIS_BF16 ? 2 : 4; }

int launch(const void* fn, int64_t grid, int block, void* arg, hipStream_t stream) {
  void* args[] = {arg};
  return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(block), args, 0, stream) == hipSuccess
             ? CIS_OK
             : CIS_ERR_LAUNCH;
}

// The rows' shape; pointers and alignment follow once every size has been found right.
int check_shape(int dtype, int64_t T, int64_t V, int64_t ld) {
  if (!known(dtype)) return CIS_ERR_DTYPE;
  if (T < 0 || V < 1 || V > kMaxV || ld < V || ld > INT64_MAX / elem_bytes(dtype))
    return CIS_ERR_SHAPE;
  return CIS_OK;
}
bool aligned_rows(const void* p, int dtype, int64_t ld) {
  return aligned(p, 16) && (ld * elem_bytes(dtype)) % 16 == 0;
}
int check_workspace(const void* workspace, size_t have, size_t need) {
  if (!aligned(workspace, 256)) return CIS_ERR_ALIGN;
  return have < need ? CIS_ERR_WORKSPACE : CIS_OK;
}

int32_t row_vecs(int64_t V, int dtype) {
  const int epv = 16 / elem_bytes(dtype);
  return (int32_t)((V + epv - 1) / epv);
}
cis::TokRows tok_rows(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                      const uint8_t* mask) {
  return cis::TokRows{logits, ld * elem_bytes(dtype), mask, T, (int32_t)V, row_vecs(V, dtype)};
}

cis::ScanLayout top_layout(int64_t T, int64_t V, int64_t K, int dtype) {
  const int32_t nvec = row_vecs(V, dtype);
  return cis::scan_layout(T, nvec, elem_bytes(dtype), cis::scan_group(nvec, K));
}
// Workgroups of 256 threads per launch of kernels that loop beyond (HIP refuses 2^32 work items).
constexpr int64_t kMaxBlocks = int64_t(1) << 23;
// Rows of a distillation call that may go in parts with the gradient.
constexpr int64_t kFewRows = 448;
// Rows up to which cis_distill_row_kernel gives a row 4 waves: two such workgroups per compute unit. The
// loss alone, us by one wave and by four, 4096 rows of 8192 bytes, bf16 (float32 within 10% of it):
//   K = 8 21.6, 25.7; K = 64 23.7, 26.9; K = 200 40.9, 34.3; K = 500 179, 108; K = 1000 290, 169
// The bound suits lists of up to 64. Beyond them four waves are the faster at every count of rows, since a
// workgroup's table and list (14 KB up to K = 256, then 55 KB of LDS) leave room for few: it does not look at K.
constexpr int64_t kWaveRows = 512;
static_assert(kFewRows <= kWaveRows, "with the gradient, a row has 4 waves");
// Logits that a draw may have to look at where its parameters do not say.
constexpr int64_t kManyLogits = 256;

// Rows whose steps of a cut are listed at once, and workgroups that the histograms of few rows take.
constexpr int64_t kStepRows = 2048;
constexpr int64_t kHistBlocks = 256;
// Workgroups of cis_weigh_kernel beyond which a wave takes several chunks.
constexpr int64_t kWeighBlocks = 2048;

struct SampleLayout {
  cis::ScanLayout scan;
  size_t draw, ties, steps, step_ids, hist, total;
  int32_t step_ld, parts;
};
SampleLayout sample_layout(int64_t T, int64_t V, int32_t nvec, int es, int32_t gv) {
  SampleLayout L{};
  L.scan = cis::scan_layout(T, nvec, es, gv);
  L.draw = L.scan.total;
  L.ties = L.draw + cis::align_up((size_t)T * L.scan.nch * 8, 256);
  L.steps = L.ties + cis::align_up((size_t)T * L.scan.nch * 4, 256);
  const int64_t rows = T < kStepRows ? T : kStepRows;
  L.step_ld = (int32_t)(V < cis::kStepTokens ? V : cis::kStepTokens);
  L.step_ids = L.steps + cis::align_up((size_t)rows * sizeof(cis::DrawStep), 256);
  L.hist = L.step_ids + cis::align_up((size_t)rows * L.step_ld * 4, 256);
  // a row's histogram by one workgroup, or in parts where there are few rows: of a chunk per wave
  const int64_t most = (L.scan.nch + cis::kHistBlock / 64 - 1) / (cis::kHistBlock / 64),
                fill = T > 0 ? kHistBlocks / T : 1;
  L.parts = (int32_t)(fill < 1 ? 1 : fill < most ? fill : most);
  L.total = L.hist + (L.parts > 1 ? (size_t)T * L.parts * cis::kFineSteps * 8 : 0);
  return L;
}
cis::TokScan scan_at(char* base, const cis::ScanLayout& L) {
  return cis::TokScan{base + L.gmax, reinterpret_cast<float*>(base + L.cmax),
                      reinterpret_cast<double*>(base + L.csum), L.nch, L.ngrp, L.gv};
}
int launch_scan(const cis::TokRows& r, const cis::TokScan& s, int dtype, float c,
                hipStream_t stream) {
  cis::ScanArgs a{r, s, c};
  const int64_t per = cis::kScanBlock / 64, need = (r.T * s.nch + per - 1) / per;
  // What fits the memory-side cache (256 MiB) is read from it later on.
  const bool keep = r.T * r.row_bytes <= int64_t(192) << 20;
  return launch(cis::scan_kernel(dtype, s.gv, keep), need < kMaxBlocks ? need : kMaxBlocks,
                cis::kScanBlock, &a, stream);
}

// Rows per launch of kernels of one workgroup per row (HIP refuses 2^32 work items).
constexpr int64_t kMaxRows = int64_t(1) << 20;
// Temperatures of a softmax: log2(e) / temperature and a logit's exponent stay within float32.
bool softmax_temperature(float t) { return t >= 0x1p-64f && t <= 0x1p64f; }

cis::FinalizeArgs finalize_args(char* base, const cis::WsLayout& L, int64_t T, float* loss_out) {
  auto f = [&](size_t off) { return reinterpret_cast<float*>(base + off); };
  return cis::FinalizeArgs{f(L.terms), reinterpret_cast<uint8_t*>(base + L.flags), f(L.logk),
                           f(L.excess), T, reinterpret_cast<cis_stats_t*>(base), loss_out, nullptr,
                           reinterpret_cast<cis::RowStats*>(base + L.wpre), 0, 0};
}

// The call's statistics and loss, as in the loss entry points: few rows by one workgroup, more
// by one per part and another over the parts (at wpre, which nothing else uses here).
int launch_finalize(char* base, const cis::WsLayout& L, int64_t T, float* loss_out,
                    hipStream_t stream) {
  cis::FinalizeArgs fa = finalize_args(base, L, T, loss_out);
  if (T <= cis::kFinalizeOne) {
    const int block = T <= cis::kFinalizeSmall ? 256 : cis::kFinalizeBlock;
    return launch(cis::finalize_kernel(block, false), 1, block, &fa, stream);
  }
  const int64_t even = (T + cis::kFinalizeParts - 1) / cis::kFinalizeParts;
  fa.rows = even <= cis::kFinalizeRows ? cis::kFinalizeRows : (even + 3) / 4 * 4;
  fa.nparts = (int32_t)((T + fa.rows - 1) / fa.rows);
  if (int rc = launch(cis::finalize_kernel(256, true), fa.nparts, 256, &fa, stream)) return rc;
  return launch(cis::finalize_parts_kernel(), 1, cis::kFinalizeParts, &fa, stream);
}

struct DistillCall {
  const void* logits;
  int dtype;
  int64_t T, V, ld;
  const int32_t* ids;
  const float* values;
  int64_t K, ld_top;
  const float *tail, *weight;
  const uint8_t* mask;
  const cis_distill_params_t* prm;
  bool bwd;
  void* dlogits;
  int64_t ld_g;
  float *terms, *loss;
  void* workspace;
  size_t workspace_bytes;
};

struct DistillLayout {
  cis::WsLayout loss;
  cis::ScanLayout scan;
  size_t scan_off, rest, valid, grads, total;
};
DistillLayout distill_layout(int64_t T, int64_t V, int64_t K, int dtype) {
  DistillLayout D{};
  D.loss = cis::ws_layout(T, 0);
  D.scan = cis::scan_layout(T, row_vecs(V, dtype), elem_bytes(dtype), 0);
  D.scan_off = D.loss.total;
  D.rest = D.scan_off + D.scan.total;
  D.valid = D.rest + cis::align_up((size_t)T * sizeof(cis::RestGrad), 256);
  D.grads = D.valid + cis::align_up((size_t)T, 256);
  // (the fused pass over many rows does not come here)
  const int64_t few = T < kFewRows ? T : kFewRows;
  D.total = D.grads + cis::align_up((size_t)few * (size_t)K * 4, 256);
  return D;
}

// With the gradient, one workgroup per row, unless the rows are too few for that: then, and without
// the gradient, in parts. The bounds follow the fused pass's ladder (distill_fused): rows that a wave
// holds 10 or 18 vectors a thread of, those of 256 threads from 12 vectors and 512 threads of 10, and
// longer ones, which take half of a compute unit and all of it. K = 64, bf16, us in parts and fused:
//   V = 1024   64 rows 15, 13       V = 4096   448 rows 17, 21     V = 12800  320 rows 18, 18
//   V = 20000  320 rows 19, 23; 448 rows 22, 22
//   V = 50400  112 rows 18, 20; 144 rows 19, 21; 240 rows 25, 21
//   V = 151936 64 rows 21, 29; 112 rows 30, 30; 144 rows 35, 30
// K = 8 and 500 and float32 take the same bounds. Over 594 points (both types, K = 8, 64, 500, rows of
// 128 to 30000 vectors, 64 to 448 rows) the side that the rule takes is 12% the faster one on average, and at
// 101 of them the slower one by more than 3%. The largest of those, us in parts and fused:
//   4500 vectors, 320 rows: K = 500 float32 37, 28; K = 64 float32 22, 18, bf16 25, 22; K = 8 bf16 24, 19
//   18992 vectors, 112 rows, float32: K = 500 40, 31; K = 8 26, 22
//   128 vectors, 112 rows, K = 500, bf16 25, 29; 30000 vectors, 320 rows, K = 64, bf16 82, 94
bool distill_in_parts(int64_t T, int32_t nvec) {
  const int64_t most = nvec <= 320    ? 0
                       : nvec <= 1152 ? 448
                       : nvec <= 2048 ? 0
                       : nvec <= 5120 ? 320
                       : nvec <= 8704 ? 144
                                      : 112;
  return T <= most;
}

int launch_distill(const DistillCall& c, const DistillLayout& D, char* base, cis::DistillArgs& a,
                   int cus, hipStream_t stream) {
  auto by_rows = [&](const void* fn, int block, int64_t n) {
    for (a.row0 = 0; a.row0 < n; a.row0 += kMaxRows)
      if (int rc = launch(fn, n - a.row0 < kMaxRows ? n - a.row0 : kMaxRows, block, &a, stream))
        return rc;
    return (int)CIS_OK;
  };
  if (c.bwd && !distill_in_parts(c.T, a.r.nvec)) {
    const cis::DistillVariant v = cis::distill_fused(c.dtype, a.r.nvec, c.K);
    const int64_t resident = (int64_t)blocks_per_cu(v.fn, v.block) * cus;
    return launch(v.fn, c.T < resident ? c.T : resident, v.block, &a, stream);
  }
  a.s = scan_at(base + D.scan_off, D.scan);
  a.rest = reinterpret_cast<cis::RestGrad*>(base + D.rest);
  a.valid = reinterpret_cast<uint8_t*>(base + D.valid);
  a.grads = reinterpret_cast<uint32_t*>(base + D.grads);
  a.nseg = (a.r.nvec + cis::kDistillGradVecs - 1) / cis::kDistillGradVecs;
  if (int rc = launch_scan(a.r, a.s, c.dtype, a.c, stream)) return rc;
  const bool few = c.T <= kWaveRows;
  if (int rc = by_rows(cis::distill_row_kernel(c.dtype, c.bwd, c.K, few), few ? 256 : 64, c.T))
    return rc;
  if (!c.bwd) return CIS_OK;
  return by_rows(cis::distill_grad_kernel(c.dtype), cis::kDistillGradBlock, c.T * a.nseg);
}

int run_distill(const DistillCall& c, hipStream_t stream) {
  if (!c.prm) return CIS_ERR_NULL;
  if (int rc = check_shape(c.dtype, c.T, c.V, c.ld)) return rc;
  const int es = elem_bytes(c.dtype);
  if (c.K < 1 || c.K > CIS_TOP_MAX_K || c.ld_top < c.K || c.ld_top > INT64_MAX / 4)
    return CIS_ERR_SHAPE;
  if (c.bwd && (c.ld_g < c.V || c.ld_g > INT64_MAX / es)) return CIS_ERR_SHAPE;
  const cis_distill_params_t& p = *c.prm;
  if (p.kind != CIS_KL_FORWARD && p.kind != CIS_KL_REVERSE) return CIS_ERR_PARAM;
  if (!softmax_temperature(p.temperature) || !isfinite(p.scale)) return CIS_ERR_PARAM;
  if (p.kind == CIS_KL_REVERSE && c.T > 0 && !c.tail) return CIS_ERR_PARAM;
  if (!c.workspace) return CIS_ERR_NULL;
  if (c.T > 0 && (!c.logits || !c.ids || !c.values || (c.bwd && !c.dlogits))) return CIS_ERR_NULL;
  if (int rc = check_workspace(c.workspace, c.workspace_bytes,
                               cis_distill_workspace_bytes(c.T, c.V, c.K, c.dtype)))
    return rc;
  if (c.T > 0) {
    if (!aligned_rows(c.logits, c.dtype, c.ld)) return CIS_ERR_ALIGN;
    if (c.bwd) {
      if (!aligned_rows(c.dlogits, c.dtype, c.ld_g)) return CIS_ERR_ALIGN;
      const uintptr_t a0 = (uintptr_t)c.logits, a1 = a0 + (uintptr_t)(c.T * c.ld * es);
      const uintptr_t b0 = (uintptr_t)c.dlogits, b1 = b0 + (uintptr_t)(c.T * c.ld_g * es);
      if (a0 == b0 ? c.ld_g != c.ld : a0 < b1 && b0 < a1) return CIS_ERR_ALIAS;
    }
  }
  const int cus = device_cus();
  if (cus < 0) return cus;

  char* base = static_cast<char*>(c.workspace);
  const DistillLayout D = distill_layout(c.T, c.V, c.K, c.dtype);
  const cis::WsLayout& L = D.loss;
  if (c.T > 0) {
    cis::DistillArgs a{};
    a.r = tok_rows(c.logits, c.dtype, c.T, c.V, c.ld, c.mask);
    a.dlogits = c.dlogits;
    a.grow_bytes = c.bwd ? c.ld_g * es : 0;
    a.ids = c.ids;
    a.values = c.values;
    a.ld_top = c.ld_top;
    a.K = (int32_t)c.K;
    a.tail = c.tail;
    a.weight = c.weight;
    a.reverse = p.kind == CIS_KL_REVERSE;
    a.temperature = p.temperature;
    a.scale = p.scale;
    a.terms_user = c.terms;
    a.terms_ws = reinterpret_cast<float*>(base + L.terms);
    a.flags_ws = reinterpret_cast<uint8_t*>(base + L.flags);
    a.logk_ws = reinterpret_cast<float*>(base + L.logk);
    a.excess_ws = reinterpret_cast<float*>(base + L.excess);
    a.c = cis::scan_c(p.temperature);
    a.inv_t = 1.f / p.temperature;
    a.inv_t64 = 1.0 / (double)p.temperature;
    a.fin = finalize_args(base, L, c.T, c.loss);
    if (int rc = launch_distill(c, D, base, a, cus, stream)) return rc;
    if (c.bwd && distill_in_parts(c.T, a.r.nvec)) return CIS_OK;   // (the last kernel sums up)
  }
  return launch_finalize(base, L, c.T, c.loss, stream);
}

}  // namespace

extern "C" {

size_t cis_sample_workspace_bytes(int64_t T, int64_t V, int dtype) {
  if (T < 0 || V < 1 || V > kMaxV || !known(dtype)) return 0;
  // (the shape of the scan goes by the call's parameters: the larger of its two)
  const int32_t nvec = row_vecs(V, dtype);
  const SampleLayout a = sample_layout(T, V, nvec, elem_bytes(dtype), 1),
                     b = sample_layout(T, V, nvec, elem_bytes(dtype), 8);
  const size_t n = a.total > b.total ? a.total : b.total;
  return n < 256 ? 256 : n;
}

size_t cis_top_logits_workspace_bytes(int64_t T, int64_t V, int64_t K, int dtype) {
  if (T < 0 || V < 1 || V > kMaxV || K < 1 || K > CIS_TOP_MAX_K || !known(dtype)) return 0;
  const size_t n = top_layout(T, V, K, dtype).total;
  return n < 256 ? 256 : n;
}

size_t cis_distill_workspace_bytes(int64_t T, int64_t V, int64_t K, int dtype) {
  if (T < 0 || V < 1 || V > kMaxV || K < 1 || K > CIS_TOP_MAX_K || !known(dtype)) return 0;
  return distill_layout(T, V, K, dtype).total;
}

int cis_sample(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const float* u,
               const uint8_t* mask, const cis_sample_params_t* params, const float* temperature,
               const int32_t* top_k, const float* top_p, const float* min_p, int64_t* ids_out,
               float* logp_out, float* logp_kept_out, void* workspace, size_t workspace_bytes,
               hipStream_t stream) {
  if (!params) return CIS_ERR_NULL;
  if (int rc = check_shape(dtype, T, V, ld)) return rc;
  const cis_sample_params_t& p = *params;
  if (!temperature && !(p.temperature >= 0.f && isfinite(p.temperature))) return CIS_ERR_PARAM;
  if (!top_k && p.top_k < 0) return CIS_ERR_PARAM;
  if (!top_p && !(p.top_p > 0.f && p.top_p <= 1.f)) return CIS_ERR_PARAM;
  if (!min_p && !(p.min_p >= 0.f && p.min_p <= 1.f)) return CIS_ERR_PARAM;
  if (!workspace) return CIS_ERR_NULL;
  if (T > 0 && (!logits || !u || !ids_out)) return CIS_ERR_NULL;
  if (int rc = check_workspace(workspace, workspace_bytes, cis_sample_workspace_bytes(T, V, dtype)))
    return rc;
  if (T > 0 && !aligned_rows(logits, dtype, ld)) return CIS_ERR_ALIGN;
  if (const int cus = device_cus(); cus < 0) return cus;
  if (T == 0) return CIS_OK;
  // What the call's rows can ask for. A row whose list is short takes a small workgroup; rows that no
  // count cuts need their weights summed up.
  const bool greedy = !temperature && !(cis::scan_c(p.temperature) < INFINITY);
  const int64_t k = greedy ? 1 : p.top_k == 0 || p.top_k >= V ? V : p.top_k;
  const bool counted = greedy || (!top_k && k <= cis::kDrawListK && k < V);   // every row
  const bool uncut = !counted && !top_k && k == V && !top_p && p.top_p == 1.f;
  const bool wide = !counted && !uncut;
  const bool weighed = !counted && (top_k || k == V);
  const bool stepped = weighed && (top_p || p.top_p < 1.f);
  // lists start from the groups; nothing else does (512 uncut rows: the scan 28 us, 24 without)
  const bool lists = counted || top_k || temperature || k <= cis::kDrawK;
  const cis::TokRows r = tok_rows(logits, dtype, T, V, ld, mask);
  char* base = static_cast<char*>(workspace);
  const SampleLayout L = sample_layout(T, V, r.nvec, elem_bytes(dtype),
                                       lists ? cis::scan_group(r.nvec, counted ? k : kManyLogits)
                                             : 0);
  const cis::TokScan s = scan_at(base, L.scan);
  if (int rc = launch_scan(r, s, dtype, cis::scan_c(1.f), stream)) return rc;
  cis::SampleArgs a{};
  a.r = r;
  a.s = s;
  a.draw = reinterpret_cast<unsigned long long*>(base + L.draw);
  a.ties = reinterpret_cast<uint32_t*>(base + L.ties);
  a.steps = reinterpret_cast<cis::DrawStep*>(base + L.steps);
  a.step_ids = reinterpret_cast<uint32_t*>(base + L.step_ids);
  a.hist = reinterpret_cast<unsigned long long*>(base + L.hist);
  a.step_ld = L.step_ld;
  a.parts = L.parts;
  a.u = u;
  a.prm = p;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.ids = ids_out;
  a.logp = logp_out;
  a.logp_kept = logp_kept_out;
  const int block = wide ? cis::kTokBlock : cis::kTopBlock;
  const int64_t most = stepped ? kStepRows : kMaxRows;
  for (; a.row0 < T; a.row0 += most) {
    a.rows = T - a.row0 < most ? T - a.row0 : most;
    if (stepped) {
      if (int rc = launch(cis::hist_kernel(dtype), a.rows * L.parts, cis::kHistBlock, &a, stream))
        return rc;
      if (L.parts > 1)
        if (int rc = launch(cis::step_kernel(), a.rows, cis::kHistBlock, &a, stream)) return rc;
    }
    if (weighed) {
      // a chunk per wave, or more of them where the chip is filled all the same
      const int64_t per = cis::kWeighBlock / 64, most = (s.nch + per - 1) / per,
                    fill = (kWeighBlocks + a.rows - 1) / a.rows;
      a.weigh_parts = (int32_t)(fill < most ? fill : most);
      if (int rc = launch(cis::weigh_kernel(dtype, stepped), a.rows * a.weigh_parts, cis::kWeighBlock, &a,
                          stream))
        return rc;
    }
    if (int rc = launch(cis::sample_kernel(dtype, wide), a.rows, block, &a, stream)) return rc;
  }
  return CIS_OK;
}

int cis_top_logits(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                   const uint8_t* mask, int64_t K, float temperature, int32_t* ids_out,
                   float* values_out, float* tail_out, void* workspace, size_t workspace_bytes,
                   hipStream_t stream) {
  if (int rc = check_shape(dtype, T, V, ld)) return rc;
  if (K < 1 || K > CIS_TOP_MAX_K) return CIS_ERR_SHAPE;
  if (!softmax_temperature(temperature)) return CIS_ERR_PARAM;
  if (!workspace) return CIS_ERR_NULL;
  if (T > 0 && (!logits || !ids_out || !values_out)) return CIS_ERR_NULL;
  if (int rc = check_workspace(workspace, workspace_bytes,
                               cis_top_logits_workspace_bytes(T, V, K, dtype)))
    return rc;
  if (T > 0 && !aligned_rows(logits, dtype, ld)) return CIS_ERR_ALIGN;
  if (const int cus = device_cus(); cus < 0) return cus;
  if (T == 0) return CIS_OK;
  const cis::TokRows r = tok_rows(logits, dtype, T, V, ld, mask);
  const cis::ScanLayout L = top_layout(T, V, K, dtype);
  const cis::TokScan s = scan_at(static_cast<char*>(workspace), L);
  if (int rc = launch_scan(r, s, dtype, cis::scan_c(temperature), stream)) return rc;
  cis::TopArgs a{r, s, (int32_t)K, temperature, cis::scan_c(temperature), 0, ids_out, values_out,
                 tail_out};
  for (; a.row0 < T; a.row0 += kMaxRows)
    if (int rc = launch(cis::top_kernel(dtype, K), T - a.row0 < kMaxRows ? T - a.row0 : kMaxRows,
                        cis::top_block(K), &a, stream))
      return rc;
  return CIS_OK;
}

int cis_distill_fwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                    const int32_t* top_ids, const float* top_values, int64_t K, int64_t ld_top,
                    const float* top_tail, const float* row_weight, const uint8_t* mask,
                    const cis_distill_params_t* params, float* terms_out, float* loss_out,
                    void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return run_distill(DistillCall{logits, dtype, T, V, ld, top_ids, top_values, K, ld_top, top_tail,
                                 row_weight, mask, params, false, nullptr, 0, terms_out, loss_out,
                                 workspace, workspace_bytes},
                     stream);
}

int cis_distill_bwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                    const int32_t* top_ids, const float* top_values, int64_t K, int64_t ld_top,
                    const float* top_tail, const float* row_weight, const uint8_t* mask,
                    const cis_distill_params_t* params, void* dlogits, int64_t ld_g,
                    float* terms_out, float* loss_out, void* workspace, size_t workspace_bytes,
                    hipStream_t stream) {
  return run_distill(DistillCall{logits, dtype, T, V, ld, top_ids, top_values, K, ld_top, top_tail,
                                 row_weight, mask, params, true, dlogits, ld_g, terms_out, loss_out,
                                 workspace, workspace_bytes},
                     stream);
}

}  // extern "C"
