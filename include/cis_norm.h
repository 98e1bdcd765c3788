/*
 * cis_norm.h — C ABI of the RMS norm on MI355X (gfx950): the operator that makes the hidden states in
 * front of the LM head (and the inputs of a model's layers, and the queries and keys of its heads),
 * with the residual's addition, outputs in 8 bits with scales, and the backward pass.
 *
 * The conventions of cis.h hold here too: device pointers owned by the caller, asynchronous calls
 * on `stream` that launch kernels only (no allocation, memset or copy; they can be captured into a
 * HIP graph), arguments checked before the first launch, identical bits for identical calls.
 */
#ifndef CIS_NORM_H
#define CIS_NORM_H

#include "cis.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of 8-bit outputs, beside cis_dtype_t: OCP e4m3 (no infinities, largest 448). */
enum { CIS_E4M3 = 2 };

/* T * N rows of H elements: row (t, n) starts at data + (t * stride_t + n * stride_n) elements. N = 1
 * for a matrix; N heads of a packed projection are rows of their own. Elements of a row are adjacent.
 * In bf16 and float32, the base address and both strides are whole 16-byte vectors; the bytes up to the
 * end of a row's last vector are read and ignored, and belong to the caller. In e4m3 they are whole
 * 8-byte vectors. (A stride along an extent of 1 is not looked at.) */
typedef struct cis_rows {
  void* data;
  int32_t dtype;
  int64_t stride_t, stride_n;   /* elements, >= 0 */
} cis_rows_t;

#define CIS_NORM_MAX_H (1 << 22)

/* =========================================================================================
 * cis_rms_norm_fwd
 *
 *   s    = x + residual, rounded to the residual's type (without a residual: x)
 *   rstd = 1 / sqrt(mean(s^2) + eps)          the mean in double
 *   y    = (s * rstd) * weight                in float32, rounded once
 *
 * and with y in e4m3, for every block of `group` columns (the last one may be shorter), or for the
 * whole row (group = 0):
 *
 *   scale = max(max |y| / 448, 2^-126),   values e4m3(y / scale)
 *
 * so that y is about value * scale. The quotient is rounded to float32, and that to the nearest value, ties
 * to even. A block with a NaN has a NaN scale and its NaN; with an infinity an infinite
 * scale, NaN in its place and zeros elsewhere.
 *
 *   T, N, H       T >= 0, N >= 1, T * N < 2^31, 1 <= H <= CIS_NORM_MAX_H
 *   x             bf16 or float32
 *   residual      NULL, or rows of x's type or float32
 *   weight        [H] bf16 or float32 (weight_dtype), 16-byte aligned; NULL = ones
 *   eps           >= 0, finite (0: a row of zeros gives NaN, and rstd, a float32, is infinite where the root is
 *                 below 2^-128, which takes subnormal elements throughout)
 *   residual_out  s, in the residual's type; NULL = not written. Needs a residual.
 *   y             bf16, float32 or e4m3
 *   scale_out     [T * N, ceil(H / group)] float, with y in e4m3 (else NULL); [T * N] for group = 0
 *   group         0, 32, 64 or 128 (0 unless y is e4m3)
 * Columns from H on are not written. An output may be an input itself (the same address, type and
 * strides); other overlaps, of one output's rows among themselves too, are CIS_ERR_ALIAS, where the
 * whole range from a tensor's first to its last row counts.
 * Errors: CIS_ERR_NULL, CIS_ERR_SHAPE (a stride < 0, group included), CIS_ERR_DTYPE, CIS_ERR_PARAM,
 * CIS_ERR_ALIGN, CIS_ERR_ALIAS, CIS_ERR_LAUNCH, CIS_ERR_DEVICE.
 * ========================================================================================= */
int cis_rms_norm_fwd(int64_t T, int64_t N, int64_t H, const cis_rows_t* x,
                     const cis_rows_t* residual, const void* weight, int weight_dtype, float eps,
                     const cis_rows_t* residual_out, const cis_rows_t* y, float* scale_out,
                     int64_t group, hipStream_t stream);

/* =========================================================================================
 * cis_rms_norm_bwd — the gradients of a loss with respect to s and the weight, from that with respect
 * to y (of the values before they are rounded; with y in e4m3 too). With xh = s * rstd and
 * g = dy * weight:
 *
 *   dx      = rstd * (g - xh * mean(g * xh)) + dresidual
 *   dweight = sum over the rows of dy * xh
 *
 * The gradient of s is that of x and of the residual both. The means are formed in double, dweight in
 * float32 for a part of the rows each, and the parts in double; all in a fixed order.
 *
 *   dy         bf16 or float32 (cis_lmhead_loss_bwd's dhidden is float32)
 *   x          the rows that were normalised: residual_out, or x where there was no residual
 *   dresidual  NULL, or rows of dx's type: the gradient that reaches s by itself (along the residual)
 *   dx         bf16 or float32. May be dy, x or dresidual itself.
 *   dweight    [H] float (overwritten; zeros when T = 0); NULL = not formed
 *   workspace  >= cis_rms_norm_workspace_bytes(T, N, H) bytes, 256-byte aligned; NULL where there is no
 *              dweight
 * Other arguments, overlaps (dweight and the workspace included) and errors as for cis_rms_norm_fwd, and
 * CIS_ERR_WORKSPACE.
 * ========================================================================================= */
size_t cis_rms_norm_workspace_bytes(int64_t T, int64_t N, int64_t H);

int cis_rms_norm_bwd(int64_t T, int64_t N, int64_t H, const cis_rows_t* dy, const cis_rows_t* x,
                     const void* weight, int weight_dtype, float eps, const cis_rows_t* dresidual,
                     const cis_rows_t* dx, float* dweight, void* workspace, size_t workspace_bytes,
                     hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CIS_NORM_H */
