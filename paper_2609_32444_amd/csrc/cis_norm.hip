// RMS norm kernels (gfx950): forward with the residual's addition, in 16, 32 or 8 bits, and backward.
//
// A row is taken in groups of 8 elements, which LANES lanes hold in registers (a part of a wave, a wave
// or a workgroup to a row); rows beyond that go in passes. Sums of squares and of products are in
// double: squares of float32 values neither overflow nor vanish there, and the extra cost, a conversion
// an element, is hidden behind the memory.
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

// Unpacked again from here on, rather than kept unpacked (see opaque()).
template <class E, int NV>
__device__ __forceinline__ void hold(Raw<E> (&x)[NV]) {
  static_for<NV>([&](auto I) __attribute__((always_inline)) { opaque(x[I].v); });
}

__device__ __forceinline__ char* row_at(const NormRows& m, uint32_t row, uint32_t N) {
  if (N == 1) return m.p + (int64_t)row * m.st;
  const uint32_t t = row / N;
  return m.p + (int64_t)t * m.st + (int64_t)(row - t * N) * m.sn;
}

// A row: an address, or where it is the whole wave's a descriptor of its vectors, beyond which loads give
// zeros and stores are dropped.
struct RowPtr {
  char* p;
  int nvec;
  __device__ __forceinline__ u32x4 load(int v) const {   // beyond the row its last vector again
    return *(const u32x4*)(p + 16 * (int64_t)(v < nvec ? v : nvec - 1));
  }
  __device__ __forceinline__ void store(int v, u32x4 x) const { *(u32x4*)(p + 16 * (int64_t)v) = x; }
  __device__ __forceinline__ void store2(int v, u32x2 x) const { *(u32x2*)(p + 8 * (int64_t)v) = x; }
};
struct RowBuf {
  char* p;
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ u32x4 load(int v) const { return bload_aux<0>(r, (uint32_t)v * 16u); }
  __device__ __forceinline__ void store(int v, u32x4 x) const {
    __builtin_amdgcn_raw_buffer_store_b128(x, r, (uint32_t)v * 16u, 0, 0);
  }
  __device__ __forceinline__ void store2(int v, u32x2 x) const {
    __builtin_amdgcn_raw_buffer_store_b64(x, r, (uint32_t)v * 8u, 0, 0);
  }
};
template <bool WAVE>
__device__ __forceinline__ auto row_of(const NormRows& m, uint32_t row, uint32_t N, int nvec) {
  char* p = row_at(m, row, N);
  if constexpr (WAVE)
    return RowBuf{p, make_rsrc(p, (uint32_t)nvec * 16u)};
  else
    return RowPtr{p, nvec};
}

// Group g of a row.
template <class E, class R>
__device__ __forceinline__ Raw<E> load_raw(const R& row, int g) {
  Raw<E> x;
#pragma unroll
  for (int k = 0; k < kVecs<E>; ++k) x.v[k] = row.load(g * kVecs<E> + k);
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
// The first n elements of 1 << LOG bytes of four words (fewer than fill them), in as few stores as there
// are bits in n.
template <int LOG>
__device__ __forceinline__ void store_tail(char* p, u32x4 w, int n) {
  uint32_t x = w[0], y = w[1];
  const int bytes = n << LOG;
  if (bytes & 8) {
    *(u32x2*)p = u32x2{x, y};
    x = w[2];
    y = w[3];
    p += 8;
  }
  if (bytes & 4) {
    *(uint32_t*)p = x;
    x = y;
    p += 4;
  }
  if (LOG <= 1 && (bytes & 2)) {
    *(uint16_t*)p = (uint16_t)x;
    x >>= 16;
    p += 2;
  }
  if (LOG == 0 && (bytes & 1)) *p = (char)x;
}
template <class E, class R>
__device__ __forceinline__ void store8(const R& row, int g, int H, const float (&f)[8]) {
#pragma unroll
  for (int k = 0; k < kVecs<E>; ++k) {
    float t[E::kPerVec];
#pragma unroll
    for (int e = 0; e < E::kPerVec; ++e) t[e] = f[k * E::kPerVec + e];
    const int v = g * kVecs<E> + k, n = H - v * E::kPerVec;
    const u32x4 x = E::pack(t);
    if (n >= E::kPerVec) {
      row.store(v, x);
    } else if (n > 0) {
      store_tail<E::kPerVec == 8 ? 1 : 2>(row.p + 16 * (int64_t)v, x, n);
    }
  }
}
// The weight's group, which is not read past its end.
__device__ __forceinline__ void load_weight(const void* w, bool f32, int g, int H, float (&f)[8]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.f;
  } else if ((g + 1) * 8 <= H) {
    if (f32)
      unpack8<F32>(load_raw<F32>(RowPtr{(char*)w, INT32_MAX}, g), g, H, f);
    else
      unpack8<Bf16>(load_raw<Bf16>(RowPtr{(char*)w, INT32_MAX}, g), g, H, f);
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
// 1 / scale in double, within 2^-52: the reciprocal in float32 is off by e (2^-22 at most), and e + e^2 of it is
// added. The product of y with it, rounded to float32, is the quotient y / scale as float32 rounds it: of two
// numbers of 24 bits the quotient is never a border between two float32 numbers, nor nearer to one than 2^-49 of
// itself. (Quotients below float32's normal numbers are zeros of e4m3 either way.) In float32, y * (1 / scale)
// gave 61 of the 1536000 values of 300 rows of 5120 the e4m3 number beside theirs; it took 5.5 us for 5.8, 132 for 133 of
// 8192 rows of 8192. A division takes 6.2 and 133, and of 16384 rows of 2048 from the caches 24 us where this takes 20.4.
__device__ __forceinline__ double e4m3_inverse(float scale) {
  const double s = scale, x = __builtin_amdgcn_rcpf(scale), e = fma(-s, x, 1.0);
  return scale == INFINITY ? 0.0 : fma(x, fma(e, e, e), x);
}
template <class R>
__device__ __forceinline__ void store_e4m3(const R& row, int g, int H, const float (&f)[8],
                                           double inv) {
  auto over = [&](float y) __attribute__((always_inline)) { return (float)((double)y * inv); };
  uint32_t b[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    b[k] = __builtin_amdgcn_cvt_pk_fp8_f32(over(f[4 * k]), over(f[4 * k + 1]), 0, false);
    b[k] = __builtin_amdgcn_cvt_pk_fp8_f32(over(f[4 * k + 2]), over(f[4 * k + 3]), b[k], true);
  }
  if ((g + 1) * 8 <= H) {
    row.store2(g, u32x2{b[0], b[1]});
  } else {
    store_tail<0>(row.p + 8 * (int64_t)g, u32x4{b[0], b[1], 0, 0}, H - g * 8);
  }
}
__device__ __forceinline__ int vecs_of(int dtype, int H) {
  return dtype == CIS_E4M3 ? (H + 15) / 16 : dtype == CIS_F32 ? (H + 3) / 4 : (H + 7) / 8;
}
__device__ __forceinline__ float rstd_of(double ss, double inv_h, float eps) {
  return (float)rsqrt(ss * inv_h + (double)eps);
}

// The weight's groups as they are stored, asked for without waiting: ones where there is no weight, zeros
// past its end, beyond which it is not read.
// (Values are chosen, not stores: else the arrays end up in scratch memory.)
template <int NV>
struct WeightRow {
  u32x4 lo[NV], hi[NV];
  __device__ __forceinline__ void load(const void* w, bool f32, int l, int lanes, int H) {
    const int nvec = f32 ? H / 4 : H / 8;   // whole ones
    const uint32_t one = w ? 0u : f32 ? 0x3F800000u : 0x3F803F80u;
    const u32x4 none{one, one, one, one};
    const bool any = w && nvec > 0;
    auto at = [&](int i) {
      u32x4 x = none;
      if (any) x = *(const u32x4*)((const char*)w + 16 * (int64_t)(i < nvec ? i : nvec - 1));
      return i < nvec ? x : none;
    };
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      const int g = l + I * lanes;
      lo[I] = at(f32 ? 2 * g : g);
      hi[I] = none;
      if (f32) hi[I] = at(2 * g + 1);
    });
    const int h0 = nvec * (f32 ? 4 : 8);
    if (w && h0 < H) {   // the vector that it ends in
      uint32_t x[4] = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (f32) {
          if (h0 + e < H) x[e] = ((const uint32_t*)w)[h0 + e];
        } else {
          if (h0 + 2 * e < H) x[e] = ((const uint16_t*)w)[h0 + 2 * e];
          if (h0 + 2 * e + 1 < H) x[e] |= (uint32_t)((const uint16_t*)w)[h0 + 2 * e + 1] << 16;
        }
      const u32x4 last{x[0], x[1], x[2], x[3]};
      static_for<NV>([&](auto I) __attribute__((always_inline)) {
        const int g = l + I * lanes;
        lo[I] = (f32 ? 2 * g : g) == nvec ? last : lo[I];
        hi[I] = f32 && 2 * g + 1 == nvec ? last : hi[I];
      });
    }
  }
  template <int I>
  __device__ __forceinline__ void get(bool f32, float (&f)[8]) const {
    if (f32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = __uint_as_float(lo[I][e]);
        f[e + 4] = __uint_as_float(hi[I][e]);
      }
    } else {
      Bf16::unpack(lo[I], f);
    }
  }
};

// Sums and maxima over the LANES lanes of a row, in each of them. `sh` may be used again after the next
// barrier.
template <int LANES>
__device__ __forceinline__ double lanes_sum(double x, double* sh) {
  if constexpr (LANES > 64) {
    return block_sum<LANES / 64>(x, sh);
  } else if constexpr (LANES == 64) {
    return wave_sum(x);
  } else {
    auto step = [](double y, auto ctrl) {
      constexpr int C = ctrl;
      const u64 b = __builtin_bit_cast(u64, y);
      return __builtin_bit_cast(double, ((u64)dpp_word<C>((uint32_t)(b >> 32)) << 32) |
                                            dpp_word<C>((uint32_t)b));
    };
    x += step(x, std::integral_constant<int, kDppXor1>{});
    x += step(x, std::integral_constant<int, kDppXor2>{});
    if constexpr (LANES >= 8) x += step(x, std::integral_constant<int, kDppHalfMirror>{});
    if constexpr (LANES >= 16) x += step(x, std::integral_constant<int, kDppRowMirror>{});
    if constexpr (LANES >= 32) x += __shfl_xor(x, 16, 64);
    return x;
  }
}
// The same over a workgroup of any number of waves.
__device__ __forceinline__ double waves_sum(double x, double* sh, int waves) {
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  const int w = threadIdx.x & 15;
  return lanes_sum<16>(w < waves ? sh[w] : 0.0, nullptr);
}
// LANES = 0: over a workgroup.
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* sh) {
  m = lanes_max(m, LANES == 0 || LANES > 16 ? 16 : LANES);
#pragma unroll
  for (int l = 16; l < 64 && (LANES == 0 || l < LANES); l += l) {
    const uint32_t o = __shfl_xor(m, l, 64);
    m = o > m ? o : m;
  }
  if constexpr (LANES == 0 || LANES > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
    __syncthreads();
    const int w = threadIdx.x & 15;
    m = lanes_max(w < (int)(blockDim.x >> 6) ? sh[w] : 0, 16);
  }
  return m;
}

// ------------------------------------------------------------------------------------------
// LANES lanes to a row, which holds at most 8 * NV * LANES elements; LANES = 0: a workgroup, of as many waves
// as the row fills. Bound by the memory: 16384 rows of 2048 in 48 us (5.6 TB/s; a copy reaches 6.2), 8192 of
// 8192 to e4m3 in 133 (5.6). Few rows are bound by the steps' latency, 2.3 us for one.
// ------------------------------------------------------------------------------------------
template <int LANES>
constexpr int kRowBlock = LANES == 0 ? 1024 : LANES > 256 ? LANES : 256;   // threads of a workgroup (at most)
template <class X, class S, bool RES, int LANES, int NV>
__global__ __launch_bounds__(kRowBlock<LANES>) void cis_norm_row_kernel(const NormArgs a) {
  constexpr bool WAVES = LANES == 0;
  constexpr int R = WAVES ? 1 : kRowBlock<LANES> / (LANES + WAVES);
  __shared__ double sh[16];
  __shared__ uint32_t shm[16];
  const int H = a.H, n8 = (H + 7) / 8, lanes = WAVES ? (int)blockDim.x : LANES;
  const int xv = (H + X::kPerVec - 1) / X::kPerVec, sv = (H + S::kPerVec - 1) / S::kPerVec;
  const int l = WAVES ? threadIdx.x : threadIdx.x % (LANES + WAVES);
  uint32_t at = WAVES ? 0 : threadIdx.x / (LANES + WAVES);
  if (LANES >= 64) at = __builtin_amdgcn_readfirstlane(at);
  uint32_t row = a.row0 + blockIdx.x * R + at;
  const bool on = row < a.rows;
  if (!on) row = a.rows - 1;
  constexpr bool WAVE = WAVES || LANES >= 64;
  const auto x = row_of<WAVE>(a.x, row, a.N, xv), r = row_of<WAVE>(RES ? a.r : a.x, row, a.N, sv);
  const auto y = row_of<WAVE>(a.y, row, a.N, vecs_of(a.ydt, H));
  Raw<X> rx[NV];
  Raw<S> rr[RES ? NV : 1];
  static_for<NV>([&](auto I) __attribute__((always_inline)) {
    rx[I] = load_raw<X>(x, l + I * lanes);
    if constexpr (RES) rr[I] = load_raw<S>(r, l + I * lanes);
  });
  WeightRow<NV> w;
  w.load(a.w, a.w_f32, l, lanes, H);
  float f[NV][8];
  double ss = 0.0;
  static_for<NV>([&](auto I) __attribute__((always_inline)) {
    const int g = l + I * lanes;
    unpack8<X>(rx[I], g, H, f[I]);
    if constexpr (RES) {
      float t[8];
      unpack8<S>(rr[I], g, H, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[I][e] += t[e];
      round_to<S>(f[I]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[I][e], (double)f[I][e], ss);
  });
  if constexpr (WAVES)
    ss = waves_sum(ss, sh, lanes / 64);
  else
    ss = lanes_sum<LANES + WAVES>(ss, sh);
  const float rstd = rstd_of(ss, 1.0 / (double)H, a.eps);
  if (RES && a.s.p && on) {   // (all of the row has been read)
    const auto s = row_of<WAVE>(a.s, row, a.N, sv);
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      if (l + I * lanes < n8) store8<S>(s, l + I * lanes, H, f[I]);
    });
  }
  static_for<NV>([&](auto I) __attribute__((always_inline)) {
    float t[8];
    w.template get<I>(a.w_f32, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[I][e] = f[I][e] * rstd * t[e];
  });
  if (a.ydt == CIS_E4M3) {
    double inv = 0.0;
    if (a.group == 0) {
      uint32_t m = 0;
      static_for<NV>([&](auto I) __attribute__((always_inline)) {
        const uint32_t b = l + I * lanes < n8 ? size_of8(f[I]) : 0;
        m = b > m ? b : m;
      });
      const float scale = e4m3_scale(row_max<LANES>(m, shm));
      if (l == 0 && on) a.scale[row] = scale;
      inv = e4m3_inverse(scale);
    }
    // lanes of a block (or of a row that is shorter)
    const int per = lanes < a.group / 8 ? lanes : a.group / 8;
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      const int g = l + I * lanes;
      if (a.group) {
        const float scale = e4m3_scale(lanes_max(g < n8 ? size_of8(f[I]) : 0, per));
        if (g < n8 && (g & (per - 1)) == 0 && on) a.scale[(int64_t)row * a.blocks + g / (a.group / 8)] = scale;
        inv = e4m3_inverse(scale);
      }
      if (g < n8 && on) store_e4m3(y, g, H, f[I], inv);
    });
  } else if (on) {
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      const int g = l + I * lanes;
      if (g < n8) {
        if (a.ydt == CIS_F32)
          store8<F32>(y, g, H, f[I]);
        else
          store8<Bf16>(y, g, H, f[I]);
      }
    });
  }
}

// The gradients, with rows that a workgroup's lanes take in turn and dweight's sums in registers; a
// workgroup's are a part. 16384 rows of 2048 with a float32 dy in 57 us (4.7 TB/s; 3001 of 4100 in 30, 3.3 TB/s):
// bound by a row's chain of loads, sums and a barrier, and by how few rows the registers leave a compute
// unit: 6 waves of a group of 8 elements to a lane fit a SIMD (with 84 registers 5, which leaves a compute unit one
// row of 9 waves for two: 38 us for 30; two groups to a lane 39), so that a row takes as many waves as it fills,
// not a power of two of them (49). The next row asked for ahead costs a wave a SIMD and gains nothing (61, 39).
// Of short rows in float32 throughout 5 waves fit: in the registers of 6 they would keep 3 to 5 words a lane in scratch
// memory (us, 131072 rows of 256 83.5 for 86.0, 1048576 of 32 85.4 for 87.9; 262144 of 128 83 and 524288 of 64 83 both ways).
template <class D, class X, int LANES>
constexpr int kGradEu = D::kPerVec == 4 && X::kPerVec == 4 && LANES > 0 && LANES < 64 ? 5 : 6;
template <class D, class X, int LANES>
__global__ __launch_bounds__(LANES ? 256 : 1024) __attribute__((amdgpu_waves_per_eu(kGradEu<D, X, LANES>)))
void cis_norm_grad_row_kernel(const NormGradArgs a) {
  constexpr bool WAVES = LANES == 0;   // a workgroup of any number of waves to a row
  constexpr int NV = 1;                // groups to a lane
  constexpr int R = WAVES ? 1 : 256 / LANES;
  const int lanes = WAVES ? (int)blockDim.x : LANES;
  __shared__ double sh[2][2][16];
  __shared__ float sum[R > 1 ? 256 : 1][9];
  const int H = a.H, n8 = (H + 7) / 8;
  const int dv = (H + D::kPerVec - 1) / D::kPerVec, xv = (H + X::kPerVec - 1) / X::kPerVec;
  const int rv = a.dx_f32 ? (H + 3) / 4 : n8;
  constexpr bool WAVE = WAVES || LANES == 64;
  const int l0 = WAVES ? threadIdx.x : threadIdx.x % (LANES + WAVES);
  uint32_t at = WAVES ? 0 : threadIdx.x / (LANES + WAVES);
  if (WAVE) at = __builtin_amdgcn_readfirstlane(at);
  WeightRow<NV> w;
  w.load(a.w, a.w_f32, l0, lanes, H);
  // (waited for here: else every row would wait for all that the row before it stored)
  opaque(w.lo);
  opaque(w.hi);
  const double inv_h = 1.0 / (double)H;
  float acc[NV][8] = {};
  int turn = 0;
  for (uint64_t row0 = (uint64_t)blockIdx.x * R; row0 < a.rows; row0 += (uint64_t)gridDim.x * R) {
    int l = l0;
    asm volatile("" : "+v"(l));   // (else what follows from it, and the weight unpacked, is kept for all rows)
    opaque(w.lo);
    opaque(w.hi);
    const bool on = row0 + at < a.rows;
    const uint32_t row = on ? (uint32_t)row0 + at : a.rows - 1;
    const auto x = row_of<WAVE>(a.x, row, a.N, xv), dy = row_of<WAVE>(a.dy, row, a.N, dv);
    Raw<X> rx[NV];
    Raw<D> rd[NV];
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      rx[I] = load_raw<X>(x, l + I * lanes);
      rd[I] = load_raw<D>(dy, l + I * lanes);
    });
    u32x4 lo[NV], hi[NV];   // dr
    static_for<NV>([&](auto I) __attribute__((always_inline)) { lo[I] = hi[I] = u32x4{0, 0, 0, 0}; });
    if (a.dr.p) {
      const auto dr = row_of<WAVE>(a.dr, row, a.N, rv);
      static_for<NV>([&](auto I) __attribute__((always_inline)) {
        const int g = l + I * lanes;
        lo[I] = dr.load(a.dx_f32 ? 2 * g : g);
        if (a.dx_f32) hi[I] = dr.load(2 * g + 1);
      });
    }
    double ss = 0.0, dot = 0.0;
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      const int g = l + I * lanes;
      float f[8], d[8], t[8];
      unpack8<X>(rx[I], g, H, f);
      unpack8<D>(rd[I], g, H, d);
      w.template get<I>(a.w_f32, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss = fma((double)f[e], (double)f[e], ss);
        dot = fma((double)f[e], (double)(d[e] * t[e]), dot);
      }
      slot_fence();
    });
    hold(rx);
    hold(rd);
    if constexpr (WAVES) {
      ss = wave_sum(ss);
      dot = wave_sum(dot);
      if ((threadIdx.x & 63) == 0) {
        sh[turn][0][threadIdx.x >> 6] = ss;
        sh[turn][1][threadIdx.x >> 6] = dot;
      }
      __syncthreads();
      const int v = threadIdx.x & 15;
      ss = lanes_sum<16>(v < lanes / 64 ? sh[turn][0][v] : 0.0, nullptr);
      dot = lanes_sum<16>(v < lanes / 64 ? sh[turn][1][v] : 0.0, nullptr);
      turn ^= 1;   // (a wave may be a row ahead of another's reading)
    } else {
      ss = lanes_sum<LANES + WAVES>(ss, nullptr);
      dot = lanes_sum<LANES + WAVES>(dot, nullptr);
    }
    const float rstd = rstd_of(ss, inv_h, a.eps), mean = (float)(dot * (double)rstd * inv_h);
    if (!on) continue;
    const auto dx = row_of<WAVE>(a.dx, row, a.N, rv);
    static_for<NV>([&](auto I) __attribute__((always_inline)) {
      const int g = l + I * lanes;
      if (g < n8) {
        float f[8], d[8], t[8];
        unpack8<X>(rx[I], g, H, f);
        unpack8<D>(rd[I], g, H, d);
        w.template get<I>(a.w_f32, t);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float xh = f[e] * rstd;
          acc[I][e] = fmaf(d[e], xh, acc[I][e]);
          t[e] = rstd * (d[e] * t[e] - xh * mean);
        }
        if (a.dr.p) {
          if (a.dx_f32)
            unpack8<F32>(Raw<F32>{{lo[I], hi[I]}}, g, H, f);
          else
            unpack8<Bf16>(Raw<Bf16>{{lo[I]}}, g, H, f);
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] += f[e];
        }
        if (a.dx_f32)
          store8<F32>(dx, g, H, t);
        else
          store8<Bf16>(dx, g, H, t);
      }
      slot_fence();
    });
  }
  if (!a.dw) return;
  float* out = a.part + (int64_t)blockIdx.x * H;
  static_for<NV>([&](auto I) __attribute__((always_inline)) {
    const int g = l0 + I * lanes;
    if constexpr (R > 1) {   // the rows' lanes, in order
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[threadIdx.x][e] = acc[I][e];
      __syncthreads();
      if ((int)threadIdx.x < lanes)
#pragma unroll 1
        for (int k = 1; k < R; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[I][e] += sum[k * lanes + l0][e];
    }
    if ((int)threadIdx.x < lanes) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (g * 8 + e < H) out[g * 8 + e] = acc[I][e];
    }
  });
}

// ------------------------------------------------------------------------------------------
// One workgroup per row, in passes over it, which the caches serve: 1024 rows of 32768 elements and more. With
// dweight a pass over the columns follows, which has 1677 rows of 20000 (float32 dy) in 36 us beside 77.
// ------------------------------------------------------------------------------------------
template <class X, class S, bool RES>
__global__ __launch_bounds__(kNormBlock) void cis_norm_kernel(const NormArgs a) {
  constexpr int NW = kNormBlock / 64;
  __shared__ double sh[NW];
  __shared__ uint32_t shm[NW];
  const int H = a.H, n8 = (H + 7) / 8;
  const int xv = (H + X::kPerVec - 1) / X::kPerVec, sv = (H + S::kPerVec - 1) / S::kPerVec;
  const int tid = threadIdx.x;
  const uint32_t row = a.row0 + blockIdx.x;
  const RowPtr x = row_of<false>(a.x, row, a.N, xv), y = row_of<false>(a.y, row, a.N, 0);
  RowPtr r{}, s{};
  if (RES) r = row_of<false>(a.r, row, a.N, sv);
  if (RES && a.s.p) s = row_of<false>(a.s, row, a.N, sv);
  auto sum8 = [&](int g, float (&f)[8]) {
    unpack8<X>(load_raw<X>(x, g), g, H, f);
    if constexpr (RES) {
      float t[8];
      unpack8<S>(load_raw<S>(r, g), g, H, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] += t[e];
      round_to<S>(f);
    }
  };
  double ss = 0.0;
  for (int g = tid; g < n8; g += kNormBlock) {
    float f[8];
    sum8(g, f);
    if (s.p) store8<S>(s, g, H, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[e], (double)f[e], ss);
  }
  const float rstd = rstd_of(block_sum<NW>(ss, sh), 1.0 / (double)H, a.eps);
  // y's group; of lanes past the row zeros. (The sum is read again as it was stored, by the thread that
  // stored it: it may have replaced what it was made from.)
  auto out8 = [&](int g, float (&f)[8]) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 0.f;
    if (g >= n8) return;
    if (s.p)
      unpack8<S>(load_raw<S>(s, g), g, H, f);
    else
      sum8(g, f);
    load_weight(a.w, a.w_f32, g, H, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] * rstd * w[e];
  };
  double inv = 0.0;
  if (a.ydt == CIS_E4M3 && a.group == 0) {
    uint32_t m = 0;
    for (int g = tid; g < n8; g += kNormBlock) {
      float f[8];
      out8(g, f);
      const uint32_t b = size_of8(f);
      m = b > m ? b : m;
    }
    const float scale = e4m3_scale(row_max<kNormBlock>(m, shm));
    if (tid == 0) a.scale[row] = scale;
    inv = e4m3_inverse(scale);
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
        inv = e4m3_inverse(scale);
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
  const RowPtr dy = row_of<false>(a.dy, row, a.N, dv), x = row_of<false>(a.x, row, a.N, xv);
  const RowPtr dx = row_of<false>(a.dx, row, a.N, 0);
  RowPtr dr{};
  if (a.dr.p) dr = row_of<false>(a.dr, row, a.N, a.dx_f32 ? (H + 3) / 4 : n8);
  auto load = [&](int g, float (&f)[8], float (&d)[8]) {
    float w[8];
    unpack8<X>(load_raw<X>(x, g), g, H, f);
    unpack8<D>(load_raw<D>(dy, g), g, H, d);
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
  const float rstd = rstd_of(ss, 1.0 / (double)H, a.eps),
              mean = (float)(dot * (double)rstd / (double)H);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
  for (int g = threadIdx.x; g < n8; g += kNormBlock) {
    float f[8], d[8];
    load(g, f, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = rstd * (d[e] - f[e] * rstd * mean);
    if (dr.p) {
      float t[8];
      if (a.dx_f32)
        unpack8<F32>(load_raw<F32>(dr, g), g, H, t);
      else
        unpack8<Bf16>(load_raw<Bf16>(dr, g), g, H, t);
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
  const RowPtr x = row_of<false>(a.x, row, a.N, xv);
  double ss = 0.0;
  for (int g = threadIdx.x; g < n8; g += kNormBlock) {
    float f[8];
    unpack8<X>(load_raw<X>(x, g), g, H, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma((double)f[e], (double)f[e], ss);
  }
  ss = block_sum<NW>(ss, sh);
  if (threadIdx.x == 0) a.rstd[row] = rstd_of(ss, 1.0 / (double)H, a.eps);
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
#pragma unroll 4
  for (uint64_t row = part; row < a.rows; row += a.parts) {
    float f[8], d[8];
    unpack8<X>(load_raw<X>(row_of<false>(a.x, (uint32_t)row, a.N, xv), g), g, H, f);
    unpack8<D>(load_raw<D>(row_of<false>(a.dy, (uint32_t)row, a.N, dv), g), g, H, d);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = fmaf(d[e], f[e] * rstd, acc[e]);
  }
  float* out = a.part + (int64_t)part * H;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (g * 8 + e < H) out[g * 8 + e] = acc[e];
}

// dweight from the parts, in double: kNormReduceCols columns to a workgroup, the parts in turn over its
// threads. 1280 parts of 2048 columns in 6 us, by latency (8.5 with 8 columns to a workgroup).
__global__ __launch_bounds__(kNormReduce) void cis_norm_reduce_kernel(const NormGradArgs a) {
  constexpr int C = kNormReduceCols, P = kNormReduce / C;
  __shared__ double sh[P][C + 1];
  const int col = threadIdx.x % C, at = threadIdx.x / C;
  const int h = blockIdx.x * C + col;
  double s = 0.0;
  if (h < a.H) {
#pragma unroll 8
    for (uint32_t p = at; p < a.parts; p += P) s += (double)a.part[(int64_t)p * a.H + h];
  }
  sh[at][col] = s;
#pragma unroll
  for (int half = P / 2; half > 0; half /= 2) {
    __syncthreads();
    if (at < half) sh[at][col] += sh[at + half][col];
  }
  if (at == 0 && h < a.H) a.dw[h] = (float)sh[0][col];
}

namespace {
template <int LANES, int NV>
NormVariant row_variant(bool x_f32, bool stream_f32, bool res) {
#define CIS_NORM(X, S, RES) {LANES, (const void*)&cis_norm_row_kernel<X, S, RES, LANES, NV>}
  if (!res) return x_f32 ? NormVariant CIS_NORM(F32, F32, false) : NormVariant CIS_NORM(Bf16, Bf16, false);
  if (x_f32) return CIS_NORM(F32, F32, true);
  return stream_f32 ? NormVariant CIS_NORM(Bf16, F32, true) : NormVariant CIS_NORM(Bf16, Bf16, true);
#undef CIS_NORM
}
template <int LANES>
NormVariant grad_variant(bool dy_f32, bool x_f32) {
#define CIS_NORM(D, X) NormVariant{LANES, (const void*)&cis_norm_grad_row_kernel<D, X, LANES>}
  if (dy_f32) return x_f32 ? CIS_NORM(F32, F32) : CIS_NORM(F32, Bf16);
  return x_f32 ? CIS_NORM(Bf16, F32) : CIS_NORM(Bf16, Bf16);
#undef CIS_NORM
}
}  // namespace

// Rows of up to 512 elements share a wave, of 4 lanes and more, or have one (524288 rows of 64 in 40 us with 8
// lanes, 50 with 16); of more, few rows take as many waves as a row fills,
// for the shortest chain, and many a wave or a workgroup of several groups to a lane, for more loads on their
// way. us (bf16, with a residual) in waves and in groups:
//   H = 640   256 rows 2.7, 3.0; 1024 3.2, 3.2; 4096 6.0, 5.7
//   H = 2048  1 row 2.3, 3.5; 256 2.8, 4.0; 1024 4.4, 4.8; 4096 12.5, 11.4
//   H = 4096  1 row 2.4, 2.6; 256 3.3, 3.4; 512 4.4, 4.4; 2048 12.9, 11.7
//   H = 8192  1 row 3.1, 3.5; 512 7.1, 7.5; 1024 13.2, 12.1
// Groups to a lane, 16384 rows of 2048: 64 lanes of 4 47.9, 256 of 1 48.6; 8192 rows of 8192 with a float32
// stream, to e4m3: 256 lanes of 4 129, 512 of 2 130, 1024 of 1 132. In passes they take 125 and 175.
NormVariant norm_kernel(int32_t H, int64_t rows, bool x_f32, bool stream_f32, bool res) {
  const int n8 = (H + 7) / 8;
#define CIS_NORM(L, V) return row_variant<L, V>(x_f32, stream_f32, res)
  if (n8 > 64 && n8 <= 1024 && rows <= 512) {
    NormVariant v = row_variant<0, 1>(x_f32, stream_f32, res);
    v.lanes = (n8 + 63) / 64 * 64;
    return v;
  }
  if (n8 <= 4) CIS_NORM(4, 1);
  if (n8 <= 8) CIS_NORM(8, 1);
  if (n8 <= 16) CIS_NORM(16, 1);
  if (n8 <= 32) CIS_NORM(32, 1);
  if (n8 <= 64) CIS_NORM(64, 1);
  if (n8 <= 128) CIS_NORM(64, 2);
  if (n8 <= 256) CIS_NORM(64, 4);
  if (n8 <= 512) CIS_NORM(256, 2);
  if (n8 <= 1024) CIS_NORM(256, 4);
  if (n8 <= 2048) CIS_NORM(512, 4);
  if (n8 <= 4096) CIS_NORM(1024, 4);
#undef CIS_NORM
  if (!res)
    return {0, x_f32 ? (const void*)&cis_norm_kernel<F32, F32, false>
                     : (const void*)&cis_norm_kernel<Bf16, Bf16, false>};
  if (x_f32) return {0, (const void*)&cis_norm_kernel<F32, F32, true>};
  return {0, stream_f32 ? (const void*)&cis_norm_kernel<Bf16, F32, true>
                        : (const void*)&cis_norm_kernel<Bf16, Bf16, true>};
}
NormVariant norm_grad_kernel(int32_t H, bool dy_f32, bool x_f32) {
  const int lanes = norm_grad_lanes(H);
  NormVariant v{};
  if (lanes == 4)
    v = grad_variant<4>(dy_f32, x_f32);
  else if (lanes == 8)
    v = grad_variant<8>(dy_f32, x_f32);
  else if (lanes == 16)
    v = grad_variant<16>(dy_f32, x_f32);
  else if (lanes == 32)
    v = grad_variant<32>(dy_f32, x_f32);
  else if (lanes == 64)
    v = grad_variant<64>(dy_f32, x_f32);
  else if (lanes)
    v = grad_variant<0>(dy_f32, x_f32);
  v.lanes = lanes;
  if (lanes) return v;
  if (dy_f32)
    return {0, x_f32 ? (const void*)&cis_norm_grad_kernel<F32, F32>
                     : (const void*)&cis_norm_grad_kernel<F32, Bf16>};
  return {0, x_f32 ? (const void*)&cis_norm_grad_kernel<Bf16, F32>
                   : (const void*)&cis_norm_grad_kernel<Bf16, Bf16>};
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
