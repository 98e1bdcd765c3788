// C-ABI entry points of the RMS norm (cis_norm.h): argument checks and launches on the caller's stream.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cis_host.h"
#include "cis_norm.h"

namespace {

using namespace cis::host;

// Workgroups per launch (HIP refuses 2^32 work items).
constexpr int64_t kMaxBlocks = int64_t(1) << 21;
// Waves that take rows in turn in the backward pass: 20 to a compute unit, of the 24 that registers leave room for
// (20 of short float32 rows). us with 20 and 24:
//   dy in float32   16384 x 2048 62.9, 64.7; 8192 x 4096 53.4, 55.5; 6000 x 6144 69.0, 60.2
//   bf16            262144 x 128 42.1, 39.5; 16384 x 2048 48.8, 46.6; 8192 x 3000 41.8, 45.4; 1000 x 4096 18.7, 22.4;
//                   6000 x 5632 57.1, 50.2 (of 11 and 12 waves a row, 20 leave a compute unit one row); 8192 wide 49.5 both
constexpr int64_t kGradCus = 256, kGradWaves = 20;

int bytes_of(int dtype) { return dtype == CIS_E4M3 ? 1 : elem_bytes(dtype); }

struct Shape {
  int64_t T, N, H;
};
int check_shape(const Shape& s) {
  if (s.T < 0 || s.N < 1 || s.H < 1 || s.H > CIS_NORM_MAX_H || s.N > INT32_MAX ||
      s.T > INT32_MAX / s.N)
    return CIS_ERR_SHAPE;
  return CIS_OK;
}

// A tensor's type, strides and alignment, and the bytes from its first to its last row.
struct View {
  cis::NormRows m{};
  int dtype = 0;
  uintptr_t lo = 0, hi = 0;
  bool given() const { return m.p != nullptr; }
};
int check_strides(const cis_rows_t& r, const Shape& s) {
  const int64_t most = INT64_MAX / 16;   // an address's offset fits 64 bits
  if ((s.T > 1 && (r.stride_t < 0 || r.stride_t > most / s.T)) ||
      (s.N > 1 && (r.stride_n < 0 || r.stride_n > most / s.N)))
    return CIS_ERR_SHAPE;
  return CIS_OK;
}
int view(const cis_rows_t& r, const Shape& s, View& v) {
  const int es = bytes_of(r.dtype);
  v.dtype = r.dtype;
  v.m.p = (char*)r.data;
  v.m.st = s.T > 1 ? r.stride_t * es : 0;
  v.m.sn = s.N > 1 ? r.stride_n * es : 0;
  const int vec = r.dtype == CIS_E4M3 ? 8 : 16;
  if (!aligned(r.data, vec) || v.m.st % vec || v.m.sn % vec) return CIS_ERR_ALIGN;
  v.lo = (uintptr_t)r.data;
  v.hi = v.lo + (s.T > 0 ? (uintptr_t)((s.T - 1) * v.m.st + (s.N - 1) * v.m.sn + s.H * es) : 0);
  return CIS_OK;
}
bool overlap(const View& a, const View& b) { return a.lo < b.hi && b.lo < a.hi; }
bool same(const View& a, const View& b) {
  return a.m.p == b.m.p && a.dtype == b.dtype && a.m.st == b.m.st && a.m.sn == b.m.sn;
}
View range(const void* p, size_t bytes) {
  View v;
  v.m.p = (char*)p;
  v.lo = (uintptr_t)p;
  v.hi = v.lo + bytes;
  return v;
}
// Whether an output's rows are apart from each other.
bool rows_apart(const View& v, const Shape& s) {
  const int64_t row = s.H * bytes_of(v.dtype);
  auto nested = [&](int64_t outer, int64_t n_outer, int64_t inner, int64_t n_inner) {
    return (n_inner <= 1 || inner >= row) &&
           (n_outer <= 1 || outer >= (n_inner > 1 ? (n_inner - 1) * inner : 0) + row);
  };
  return nested(v.m.st, s.T, v.m.sn, s.N) || nested(v.m.sn, s.N, v.m.st, s.T);
}

int check_weight(const void* w, int dtype) {
  return w && !known(dtype) ? CIS_ERR_DTYPE : CIS_OK;
}

// Workgroups of cis_norm_part_kernel over the columns.
int64_t part_columns(int64_t H) { return (H + 8 * cis::kNormColumns - 1) / (8 * cis::kNormColumns); }
// Parts of dweight's sums: the workgroups of the pass, or where its registers do not hold them, shares of the
// rows that fill the chip together with the shares of the columns.
uint32_t grad_parts(int64_t rows, int32_t H) {
  const int lanes = cis::norm_grad_lanes(H);
  int64_t need = rows, most = kGradCus * (kGradWaves / (cis::kNormColumns / 64)) / part_columns(H);
  if (H <= cis::kNormGradResident) {
    const int64_t per = cis::norm_block_rows(lanes);
    need = (rows + per - 1) / per;
    most = kGradCus * (kGradWaves / (cis::norm_block(lanes) / 64));
  }
  if (most < 16) most = 16;
  return (uint32_t)(need < most ? need : most);
}
struct GradLayout {
  size_t rstd, part, total;
  uint32_t parts;
};
GradLayout grad_layout(const Shape& s) {
  GradLayout L{};
  const int64_t rows = s.T * s.N;
  L.parts = grad_parts(rows, (int32_t)s.H);
  L.rstd = 0;
  L.part = s.H <= cis::kNormGradResident ? 0 : cis::align_up((size_t)rows * 4, 256);
  L.total = L.part + cis::align_up((size_t)L.parts * s.H * 4, 256);
  return L;
}

}  // namespace

extern "C" {

int cis_rms_norm_fwd(int64_t T, int64_t N, int64_t H, const cis_rows_t* x,
                     const cis_rows_t* residual, const void* weight, int weight_dtype, float eps,
                     const cis_rows_t* residual_out, const cis_rows_t* y, float* scale_out,
                     int64_t group, hipStream_t stream) {
  if (!x || !y) return CIS_ERR_NULL;
  const Shape s{T, N, H};
  const bool e4m3 = y->dtype == CIS_E4M3;
  if (!known(x->dtype) || (!known(y->dtype) && !e4m3)) return CIS_ERR_DTYPE;
  if (residual && residual->dtype != x->dtype && residual->dtype != CIS_F32) return CIS_ERR_DTYPE;
  if (residual_out && (!residual || residual_out->dtype != residual->dtype)) return CIS_ERR_DTYPE;
  if (int rc = check_weight(weight, weight_dtype)) return rc;
  if (int rc = check_shape(s)) return rc;
  if (group != 0 && (!e4m3 || (group != 32 && group != 64 && group != 128))) return CIS_ERR_SHAPE;
  for (const cis_rows_t* r : {x, residual, residual_out, y})
    if (r)
      if (int rc = check_strides(*r, s)) return rc;
  if (!(eps >= 0.f && isfinite(eps))) return CIS_ERR_PARAM;
  if (T == 0) return device_cus() < 0 ? CIS_ERR_DEVICE : CIS_OK;
  if (!x->data || !y->data || (residual && !residual->data) || (residual_out && !residual_out->data) ||
      (e4m3 && !scale_out))
    return CIS_ERR_NULL;
  View vx, vr, vs, vy;
  if (int rc = view(*x, s, vx)) return rc;
  if (residual)
    if (int rc = view(*residual, s, vr)) return rc;
  if (residual_out)
    if (int rc = view(*residual_out, s, vs)) return rc;
  if (int rc = view(*y, s, vy)) return rc;
  if (weight && !aligned(weight, 16)) return CIS_ERR_ALIGN;
  if (scale_out && !aligned(scale_out, 4)) return CIS_ERR_ALIGN;
  const int64_t rows = T * N, blocks = group ? (H + group - 1) / group : 1;
  const View vw = range(weight, weight ? H * bytes_of(weight_dtype) : 0),
             vc = range(scale_out, e4m3 ? rows * blocks * 4 : 0);
  for (const View* out : {&vs, &vy}) {
    if (!out->given()) continue;
    if (!rows_apart(*out, s)) return CIS_ERR_ALIAS;
    for (const View* in : {&vx, &vr})
      if (in->given() && overlap(*out, *in) && !same(*out, *in)) return CIS_ERR_ALIAS;
    if (overlap(*out, vw) || overlap(*out, vc)) return CIS_ERR_ALIAS;
  }
  if (vs.given() && overlap(vs, vy)) return CIS_ERR_ALIAS;
  for (const View* in : {(const View*)&vx, (const View*)&vr, &vw})
    if (in->given() && overlap(*in, vc)) return CIS_ERR_ALIAS;
  if (const int cus = device_cus(); cus < 0) return cus;

  cis::NormArgs a{};
  a.x = vx.m;
  a.r = vr.m;
  a.s = vs.m;
  a.y = vy.m;
  a.rows = (uint32_t)rows;
  a.N = (uint32_t)N;
  a.H = (int32_t)H;
  a.w = weight;
  a.w_f32 = weight_dtype == CIS_F32;
  a.eps = eps;
  a.ydt = y->dtype;
  a.group = (int32_t)group;
  a.blocks = (int32_t)blocks;
  a.scale = e4m3 ? scale_out : nullptr;
  const cis::NormVariant v = cis::norm_kernel((int32_t)H, rows, x->dtype == CIS_F32,
                                              residual && residual->dtype == CIS_F32,
                                              residual != nullptr);
  const int64_t per = cis::norm_block_rows(v.lanes), most = kMaxBlocks * per;
  for (int64_t row0 = 0; row0 < rows; row0 += most) {
    a.row0 = (uint32_t)row0;
    const int64_t n = rows - row0 < most ? rows - row0 : most;
    if (int rc = launch(v.fn, (n + per - 1) / per, cis::norm_block(v.lanes), &a, stream)) return rc;
  }
  return CIS_OK;
}

size_t cis_rms_norm_workspace_bytes(int64_t T, int64_t N, int64_t H) {
  const Shape s{T, N, H};
  if (check_shape(s)) return 0;
  const size_t n = grad_layout(s).total;
  return n < 256 ? 256 : n;
}

int cis_rms_norm_bwd(int64_t T, int64_t N, int64_t H, const cis_rows_t* dy, const cis_rows_t* x,
                     const void* weight, int weight_dtype, float eps, const cis_rows_t* dresidual,
                     const cis_rows_t* dx, float* dweight, void* workspace, size_t workspace_bytes,
                     hipStream_t stream) {
  if (!dy || !x || !dx) return CIS_ERR_NULL;
  const Shape s{T, N, H};
  if (!known(dy->dtype) || !known(x->dtype) || !known(dx->dtype)) return CIS_ERR_DTYPE;
  if (dresidual && dresidual->dtype != dx->dtype) return CIS_ERR_DTYPE;
  if (int rc = check_weight(weight, weight_dtype)) return rc;
  if (int rc = check_shape(s)) return rc;
  for (const cis_rows_t* r : {dy, x, dresidual, dx})
    if (r)
      if (int rc = check_strides(*r, s)) return rc;
  if (!(eps >= 0.f && isfinite(eps))) return CIS_ERR_PARAM;
  const size_t need = cis_rms_norm_workspace_bytes(T, N, H);
  if (dweight) {
    if (!workspace) return CIS_ERR_NULL;
    if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
    if (!aligned(dweight, 16)) return CIS_ERR_ALIGN;
  }
  View vd, vx, vr, vg;
  if (T > 0) {
    if (!dy->data || !x->data || !dx->data || (dresidual && !dresidual->data)) return CIS_ERR_NULL;
    if (int rc = view(*dy, s, vd)) return rc;
    if (int rc = view(*x, s, vx)) return rc;
    if (dresidual)
      if (int rc = view(*dresidual, s, vr)) return rc;
    if (int rc = view(*dx, s, vg)) return rc;
    if (weight && !aligned(weight, 16)) return CIS_ERR_ALIGN;
    if (!rows_apart(vg, s)) return CIS_ERR_ALIAS;
  }
  const View vw = range(weight, weight ? H * bytes_of(weight_dtype) : 0),
             vdw = range(dweight, dweight ? H * 4 : 0),
             vws = range(workspace, dweight ? need : 0);
  for (const View* in : {&vd, &vx, &vr})
    if (in->given() && overlap(vg, *in) && !same(vg, *in)) return CIS_ERR_ALIAS;
  for (const View* in : {(const View*)&vd, (const View*)&vx, (const View*)&vr, (const View*)&vg, &vw})
    if (overlap(*in, vdw) || overlap(*in, vws)) return CIS_ERR_ALIAS;
  if (overlap(vg, vw) || overlap(vdw, vws)) return CIS_ERR_ALIAS;
  if (const int cus = device_cus(); cus < 0) return cus;

  cis::NormGradArgs a{};
  a.dy = vd.m;
  a.x = vx.m;
  a.dr = vr.m;
  a.dx = vg.m;
  a.rows = (uint32_t)(T * N);
  a.N = (uint32_t)N;
  a.H = (int32_t)H;
  a.w = weight;
  a.w_f32 = weight_dtype == CIS_F32;
  a.eps = eps;
  a.dx_f32 = dx->dtype == CIS_F32;
  a.dw = dweight;
  const bool df = dy->dtype == CIS_F32, xf = x->dtype == CIS_F32;
  const GradLayout L = grad_layout(s);
  if (dweight) {
    a.rstd = reinterpret_cast<float*>((char*)workspace + L.rstd);
    a.part = reinterpret_cast<float*>((char*)workspace + L.part);
  }
  auto sum_parts = [&] {
    const int64_t grid = (H + cis::kNormReduceCols - 1) / cis::kNormReduceCols;
    return launch(cis::norm_reduce_kernel(), grid, cis::kNormReduce, &a, stream);
  };
  if (a.rows == 0) return dweight ? sum_parts() : CIS_OK;
  a.parts = L.parts;
  const cis::NormVariant v = cis::norm_grad_kernel((int32_t)H, df, xf);
  if (H <= cis::kNormGradResident) {
    if (int rc = launch(v.fn, a.parts, cis::norm_block(v.lanes), &a, stream)) return rc;
    return dweight ? sum_parts() : CIS_OK;
  }
  auto by_rows = [&](const void* fn) {
    for (int64_t row0 = 0; row0 < (int64_t)a.rows; row0 += kMaxBlocks) {
      a.row0 = (uint32_t)row0;
      const int64_t n = a.rows - row0 < kMaxBlocks ? a.rows - row0 : kMaxBlocks;
      if (int rc = launch(fn, n, cis::kNormBlock, &a, stream)) return rc;
    }
    return (int)CIS_OK;
  };
  if (!dweight) return by_rows(v.fn);
  // dx, then the sums with the rstd that it leaves; ahead of a dx that replaces what they are made from,
  // with a pass for rstd
  const bool replaces = overlap(vg, vd) || overlap(vg, vx);
  if (int rc = by_rows(replaces ? cis::norm_rstd_kernel(xf) : v.fn)) return rc;
  if (int rc = launch(cis::norm_part_kernel(df, xf), part_columns(H) * a.parts, cis::kNormColumns, &a,
                      stream))
    return rc;
  if (int rc = sum_parts()) return rc;
  return replaces ? by_rows(v.fn) : CIS_OK;
}

}  // extern "C"
