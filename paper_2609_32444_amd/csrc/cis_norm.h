// Internal interface of the RMS norm (cis_norm.h): kernel arguments and the shape of a launch.
#pragma once

#include "../../include/cis_norm.h"
#include "cis_internal.h"

namespace cis {

// T * N rows, as in cis_rows_t, with strides in bytes.
struct NormRows {
  char* p;             // nullable
  int64_t st, sn;
};

struct NormArgs {
  NormRows x, r, s, y;   // input, residual, sum, output (r, s nullable)
  uint32_t rows, N, row0;   // row0: the first row of a launch
  int32_t H;
  const void* w;         // nullable
  int32_t w_f32;
  float eps;
  int32_t ydt;           // cis_dtype_t or CIS_E4M3
  int32_t group;         // columns of a block of e4m3 values; 0: the row
  int32_t blocks;        // per row
  float* scale;
};

struct NormGradArgs {
  NormRows dy, x, dr, dx;   // dr nullable
  uint32_t rows, N, row0;   // row0: the first row of a launch
  int32_t H;
  const void* w;            // nullable
  int32_t w_f32;
  float eps;
  int32_t dx_f32;           // type of dr and dx
  float* rstd;              // [rows]
  float* part;              // [parts, H] sums of dweight
  uint32_t parts;
  float* dw;
};

constexpr int kNormBlock = 1024;
constexpr int kNormColumns = 256;             // threads of 8 columns each in a part of dweight's sums
constexpr uint32_t kNormParts = 256;
constexpr int kNormReduce = 1024, kNormReduceCols = 64;

// x and stream in float32 or bf16; res: a residual is added
const void* norm_kernel(bool x_f32, bool stream_f32, bool res);
const void* norm_grad_kernel(bool dy_f32, bool x_f32);
const void* norm_rstd_kernel(bool x_f32);
const void* norm_part_kernel(bool dy_f32, bool x_f32);
const void* norm_reduce_kernel();

}  // namespace cis
