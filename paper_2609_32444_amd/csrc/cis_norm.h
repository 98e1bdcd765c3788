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

constexpr int kNormBlock = 1024;              // threads to a row that goes in passes
constexpr int kNormColumns = 256;             // threads of 8 columns each in a part of dweight's sums
constexpr int kNormReduce = 1024, kNormReduceCols = 16;
constexpr int32_t kNormGradResident = 8192;   // elements of a row up to which dweight's sums stay in registers

// The kernel for rows of H elements, with `lanes` lanes to a row (up to 64 in workgroups of 256, else a
// workgroup), or in passes over it (0: one workgroup of kNormBlock threads per row).
struct NormVariant {
  int lanes;
  const void* fn;
};
inline int norm_block(int lanes) { return lanes == 0 ? kNormBlock : lanes > 64 ? lanes : 256; }
inline int norm_block_rows(int lanes) { return lanes == 0 ? 1 : norm_block(lanes) / lanes; }
// x and stream in float32 or bf16; res: a residual is added
NormVariant norm_kernel(int32_t H, int64_t rows, bool x_f32, bool stream_f32, bool res);
NormVariant norm_grad_kernel(int32_t H, bool dy_f32, bool x_f32);
// Lanes to a row in the backward pass, a group of 8 elements each: a part of a wave, or whole waves. (0: in
// passes. Of two groups to a lane, 3355 rows of 10000, the registers leave so few waves that they are no
// faster than passes: 76 us of 115.)
inline int norm_grad_lanes(int32_t H) {
  const int n8 = (H + 7) / 8;
  if (H > kNormGradResident) return 0;
  return n8 <= 4 ? 4 : n8 <= 8 ? 8 : n8 <= 16 ? 16 : n8 <= 32 ? 32 : (n8 + 63) / 64 * 64;
}
const void* norm_rstd_kernel(bool x_f32);
const void* norm_part_kernel(bool dy_f32, bool x_f32);
const void* norm_reduce_kernel();

}  // namespace cis
