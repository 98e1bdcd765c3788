// RMS norm kernels (gfx950): forward with the residual's addition, in 16, 32 or 8 bits, and backward.
//
// A row is taken in groups of 8 elements. Sums of squares and of products are in double: squares of
// float32 values neither overflow nor vanish there, and the extra cost, a conversion an element, is
// hidden behind the memory.
#include <type_traits>

#include "cis_norm.h"
#include "cis_tok_row.h"

namespace cis {

template <class E>
constexpr int kVecs = 8 / E::kPerVec;   // 16-byte vectors per group
template <class E>
struct Raw {
  u32x4 v[kVecs<E>];
};

__device__ __forceinline__ char* row_at(const NormRows& m, uint32_t row, uint32_t N) {
  if (N == 1) return m.p + (int64_t)row * m.st;
  const uint32_t t = row / N;
  return m.p + (int64_t)t * m.st + (int64_t)(row - t * N) * m.sn;
}

// Group g of a row of nvec vectors; beyond the row its last vector again.
template <class E>
__device__ __forceinline__ Raw<E> load_raw(const char* row, int g, int nvec) {
  Raw<E> x;
#pragma unroll
  for (int k = 0; k < kVecs<E>; ++k) {
    const int v = g * kVecs<E> + k;
    x.v[k] = *(const u32x4*)(row + 16 * (int64_t)(v < nvec ? v : nvec - 1));
  }
  return x;
}
// Its elements; 0 past the row's end.
template <class E>
__device__ __forceinline__ void unpack8(const Raw<E>& x, int g, int H, float (&f)[8]) {
#pragma unroll
  for (int k = 0; k < kVecs<E>; ++k) {
    float t[E::kPerVec];
    E::unpack(x.v[k], t);
#pragma unroll
    for (int e = 0; e < E::kPerVec; ++e) f[k * E::kPerVec + e] = t[e];
  }
  if ((g + 1) * 8 > H) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = g * 8 + e < H ? f[e] : 0.f;
  }
}
template <class E>
__device__ __forceinline__ void round_to(float (&f)[8]) {
  if constexpr (E::kPerVec == 8) {
    const u32x4 b = E::pack(f);
    E::unpack(b, f);
  }
}
template <class E>
__device__ __forceinline__ void store8(char* row, int g, int H, const float (&f)[8]) {
  if ((g + 1) * 8 <= H) {
#pragma unroll
    for (int k = 0; k < kVecs<E>; ++k) {
      float t[E::kPerVec];
#pragma unroll
      for (int e = 0; e < E::kPerVec; ++e) t[e] = f[k * E::kPerVec + e];
      *(u32x4*)(row + 16 * (int64_t)(g * kVecs<E> + k)) = E::pack(t);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (g * 8 + e < H) E::store_elem(row, g * 8 + e, E::bits_of(f[e]));
  }
}
// The weight's group, which is not read past its end.
__device__ __forceinline__ void load_weight(const void* w, bool f32, int g, int H, float (&f)[8]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.f;
  } else if ((g + 1) * 8 <= H) {
    if (f32)
      unpack8<F32>(load_raw<F32>((const char*)w, g, INT32_MAX), g, H, f);
    else
      unpack8<Bf16>(load_raw<Bf16>((const char*)w, g, INT32_MAX), g, H, f);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = 0.f;
      if (g * 8 + e < H)
        f[e] = f32 ? ((const float*)w)[g * 8 + e]
                   : __uint_as_float((uint32_t)((const uint16_t*)w)[g * 8 + e] << 16);
    }
  }
}

// The largest |f| as whole numbers: the order of positive floats, with a NaN above all of them.
__device__ __forceinline__ uint32_t size_of8(const float (&f)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t b = __float_as_uint(f[e]) & 0x7FFFFFFFu;
    m = b > m ? b : m;
  }
  return m;
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_step(uint32_t x) {
  const uint32_t y = dpp_word<CTRL>(x);
  return y > x ? y : x;
}
// The largest over 4, 8 or 16 lanes that follow each other.
__device__ __forceinline__ uint32_t lanes_max(uint32_t x, int lanes) {
  x = max_step<kDppXor1>(x);
  x = max_step<kDppXor2>(x);
  if (lanes > 4) x = max_step<kDppHalfMirror>(x);
  if (lanes > 8) x = max_step<kDppRowMirror>(x);
  return x;
}
// A block's scale from its largest |y|. (The least one keeps 1 / scale finite.)
__device__ __forceinline__ float e4m3_scale(uint32_t size) {
  const float s = __uint_as_float(size) / 448.f;
  return s < 0x1p-126f ? 0x1p-126f : s;
}
__device__ __forceinline__ void store_e4m3(char* row, int g, int H, const float (&f)[8], float inv) {
  uint32_t b[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    b[k] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k] * inv, f[4 * k + 1] * inv, 0, false);
    b[k] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k + 2] * inv, f[4 * k + 3] * inv, b[k], true);
  }
  if ((g + 1) * 8 <= H) {
    *(u32x2*)(row + 8 * (int64_t)g) = u32x2{b[0], b[1]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (g * 8 + e < H) row[g * 8 + e] = (char)(b[e / 4] >> (8 * (e % 4)));
  }
}
__device__ __forceinline__ float rstd_of(double ss, int H, float eps) {
  return (float)(1.0 / sqrt(ss / (double)H + (double)eps));
}

// ------------------------------------------------------------------------------------------
// One workgroup per row, in passes over it.
// ------------------------------------------------------------------------------------------
template <class X, class S, bool RES>
__global__ __launch_bounds__(kNormBlock) void cis_norm_kernel(const NormArgs a) {
  constexpr int NW = kNormBlock / 64;
  __shared__ double sh[NW];
  __shared__ uint32_t shm[NW];
  const int H = a.H, n8 = (H + 7) / 8;
  const int xv = (H + X::kPerVec - 1) / X::kPerVec, sv = (H + S::kPerVec - 1) / S::kPerVec;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const uint32_t row = a.row0 + blockIdx.x;
  const char* x = row_at(a.x, row, a.N);
  const char* r = RES ? row_at(a.r, row, a.N) : nullptr;
  char* s = RES && a.s.p ? row_at(a.s, row, a.N) : nullptr;
  char* y = row_at(a.y, row, a.N);
  auto sum8 = [&](int g, float (&f)[8]) {
    unpack8<X>(load_raw<X>(x, g, xv), g, H, f);
    if constexpr (RES) {
      float t[8];
      unpack8<S>(load_raw<S>(r, g, sv), g, H, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] += t[e];
      round_to<S>(f);
    }
  };
  double ss = 0.0;
  for (int g = tid; g < n8; g += kNormBlock) {
    float f[8];
    sum8(g, f);
    if (s) store8<S>(s, g, H, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[e], (double)f[e], ss);
  }
  const float rstd = rstd_of(block_sum<NW>(ss, sh), H, a.eps);
  // y's group; of lanes past the row zeros. (The sum is read again as it was stored, by the thread that
  // stored it: it may have replaced what it was made from.)
  auto out8 = [&](int g, float (&f)[8]) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 0.f;
    if (g >= n8) return;
    if (s)
      unpack8<S>(load_raw<S>(s, g, sv), g, H, f);
    else
      sum8(g, f);
    load_weight(a.w, a.w_f32, g, H, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] * rstd * w[e];
  };
  float inv = 0.f;
  if (a.ydt == CIS_E4M3 && a.group == 0) {
    uint32_t m = 0;
    for (int g = tid; g < n8; g += kNormBlock) {
      float f[8];
      out8(g, f);
      const uint32_t b = size_of8(f);
      m = b > m ? b : m;
    }
    m = lanes_max(m, 16);
#pragma unroll
    for (int l = 16; l < 64; l += 16) {
      const uint32_t o = __shfl_xor(m, l, 64);
      m = o > m ? o : m;
    }
    if (lane == 0) shm[wid] = m;
    __syncthreads();
    for (int w = 0; w < NW; ++w) m = shm[w] > m ? shm[w] : m;
    const float scale = e4m3_scale(m);
    if (tid == 0) a.scale[row] = scale;
    inv = 1.f / scale;
  }
  for (int g0 = 0; g0 < n8; g0 += kNormBlock) {   // (whole waves together)
    const int g = g0 + tid;
    float f[8];
    out8(g, f);
    if (a.ydt == CIS_E4M3) {
      if (a.group) {
        const int lanes = a.group / 8;
        const float scale = e4m3_scale(lanes_max(size_of8(f), lanes));
        if (g < n8 && g % lanes == 0) a.scale[(int64_t)row * a.blocks + g / lanes] = scale;
        inv = 1.f / scale;
      }
      if (g < n8) store_e4m3(y, g, H, f, inv);
    } else if (g < n8) {
      if (a.ydt == CIS_F32)
        store8<F32>(y, g, H, f);
      else
        store8<Bf16>(y, g, H, f);
    }
  }
}

// The gradient of the sum, by one workgroup per row.
template <class D, class X>
__global__ __launch_bounds__(kNormBlock) void cis_norm_grad_kernel(const NormGradArgs a) {
  constexpr int NW = kNormBlock / 64;
  __shared__ double sh[2][NW];
  const int H = a.H, n8 = (H + 7) / 8;
  const int dv = (H + D::kPerVec - 1) / D::kPerVec, xv = (H + X::kPerVec - 1) / X::kPerVec;
  const uint32_t row = a.row0 + blockIdx.x;
  const char* dy = row_at(a.dy, row, a.N);
  const char* x = row_at(a.x, row, a.N);
  const char* dr = a.dr.p ? row_at(a.dr, row, a.N) : nullptr;
  char* dx = row_at(a.dx, row, a.N);
  auto load = [&](int g, float (&f)[8], float (&d)[8]) {
    float w[8];
    unpack8<X>(load_raw<X>(x, g, xv), g, H, f);
    unpack8<D>(load_raw<D>(dy, g, dv), g, H, d);
    load_weight(a.w, a.w_f32, g, H, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] *= w[e];
  };
  double ss = 0.0, dot = 0.0;
  for (int g = threadIdx.x; g < n8; g += kNormBlock) {
    float f[8], d[8];
    load(g, f, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ss = fma((double)f[e], (double)f[e], ss);
      dot = fma((double)f[e], (double)d[e], dot);
    }
  }
  ss = block_sum<NW>(ss, sh[0]);
  dot = block_sum<NW>(dot, sh[1]);
  const float rstd = rstd_of(ss, H, a.eps), mean = (float)(dot * (double)rstd / (double)H);
  for (int g = threadIdx.x; g < n8; g += kNormBlock) {
    float f[8], d[8];
    load(g, f, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = rstd * (d[e] - f[e] * rstd * mean);
    if (dr) {
      float t[8];
      if (a.dx_f32)
        unpack8<F32>(load_raw<F32>(dr, g, (H + 3) / 4), g, H, t);
      else
        unpack8<Bf16>(load_raw<Bf16>(dr, g, n8), g, H, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] += t[e];
    }
    if (a.dx_f32)
      store8<F32>(dx, g, H, d);
    else
      store8<Bf16>(dx, g, H, d);
  }
}

template <class X>
__global__ __launch_bounds__(kNormBlock) void cis_norm_rstd_kernel(const NormGradArgs a) {
  constexpr int NW = kNormBlock / 64;
  __shared__ double sh[NW];
  const int H = a.H, n8 = (H + 7) / 8, xv = (H + X::kPerVec - 1) / X::kPerVec;
  const uint32_t row = a.row0 + blockIdx.x;
  const char* x = row_at(a.x, row, a.N);
  double ss = 0.0;
  for (int g = threadIdx.x; g < n8; g += kNormBlock) {
    float f[8];
    unpack8<X>(load_raw<X>(x, g, xv), g, H, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[e], (double)f[e], ss);
  }
  ss = block_sum<NW>(ss, sh);
  if (threadIdx.x == 0) a.rstd[row] = rstd_of(ss, H, a.eps);
}

// dweight's sums over the rows p, p + parts, ... of part p, 8 columns to a thread.
template <class D, class X>
__global__ __launch_bounds__(kNormColumns) void cis_norm_part_kernel(const NormGradArgs a) {
  const int H = a.H, n8 = (H + 7) / 8;
  const int dv = (H + D::kPerVec - 1) / D::kPerVec, xv = (H + X::kPerVec - 1) / X::kPerVec;
  const uint32_t part = blockIdx.x % a.parts;
  const int g = (int)(blockIdx.x / a.parts) * kNormColumns + threadIdx.x;
  if (g >= n8) return;
  float acc[8] = {};
  for (uint64_t row = part; row < a.rows; row += a.parts) {
    float f[8], d[8];
    unpack8<X>(load_raw<X>(row_at(a.x, (uint32_t)row, a.N), g, xv), g, H, f);
    unpack8<D>(load_raw<D>(row_at(a.dy, (uint32_t)row, a.N), g, dv), g, H, d);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(d[e], f[e] * rstd, acc[e]);
  }
  float* out = a.part + (int64_t)part * H;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (g * 8 + e < H) out[g * 8 + e] = acc[e];
}

// dweight from the parts, in double: a column per lane, the parts in turn over the waves.
__global__ __launch_bounds__(kNormReduce) void cis_norm_reduce_kernel(const NormGradArgs a) {
  constexpr int NW = kNormReduce / kNormReduceCols;
  __shared__ double sh[NW][kNormReduceCols];
  const int lane = threadIdx.x % kNormReduceCols, wid = threadIdx.x / kNormReduceCols;
  const int h = blockIdx.x * kNormReduceCols + lane;
  double s = 0.0;
  if (h < a.H)
    for (uint32_t p = wid; p < a.parts; p += NW) s += (double)a.part[(int64_t)p * a.H + h];
  sh[wid][lane] = s;
  __syncthreads();
  if (wid == 0 && h < a.H) {
    for (int w = 1; w < NW; ++w) s += sh[w][lane];
    a.dw[h] = (float)s;
  }
}

const void* norm_kernel(bool x_f32, bool stream_f32, bool res) {
  if (!res)
    return x_f32 ? (const void*)&cis_norm_kernel<F32, F32, false>
                 : (const void*)&cis_norm_kernel<Bf16, Bf16, false>;
  if (x_f32) return (const void*)&cis_norm_kernel<F32, F32, true>;
  return stream_f32 ? (const void*)&cis_norm_kernel<Bf16, F32, true>
                    : (const void*)&cis_norm_kernel<Bf16, Bf16, true>;
}
const void* norm_grad_kernel(bool dy_f32, bool x_f32) {
  if (dy_f32)
    return x_f32 ? (const void*)&cis_norm_grad_kernel<F32, F32>
                 : (const void*)&cis_norm_grad_kernel<F32, Bf16>;
  return x_f32 ? (const void*)&cis_norm_grad_kernel<Bf16, F32>
               : (const void*)&cis_norm_grad_kernel<Bf16, Bf16>;
}
const void* norm_rstd_kernel(bool x_f32) {
  return x_f32 ? (const void*)&cis_norm_rstd_kernel<F32> : (const void*)&cis_norm_rstd_kernel<Bf16>;
}
const void* norm_part_kernel(bool dy_f32, bool x_f32) {
  if (dy_f32)
    return x_f32 ? (const void*)&cis_norm_part_kernel<F32, F32>
                 : (const void*)&cis_norm_part_kernel<F32, Bf16>;
  return x_f32 ? (const void*)&cis_norm_part_kernel<Bf16, F32>
               : (const void*)&cis_norm_part_kernel<Bf16, Bf16>;
}
const void* norm_reduce_kernel() { return (const void*)&cis_norm_reduce_kernel; }

}  // namespace cis
