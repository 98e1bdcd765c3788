// Internal interface of the token operators (cis_tokens.h): kernel arguments, workspace layouts and
// what their kernels share.
#pragma once

#include "../../include/cis_tokens.h"
#include "cis_internal.h"

namespace cis {

// Rows of logits, as every token operator reads them.
struct TokRows {
  const void* logits;
  int64_t row_bytes;
  const uint8_t* mask;   // nullable
  int64_t T;
  int32_t V, nvec;       // nvec = ceil(V / elements per 16-byte vector)
};

// Weights of a draw are whole multiples of 1 / kDrawOne of the row's largest. 8 weights of a vector
// add up within 32 bits, and the 2^28 of the longest row within 64.
constexpr uint32_t kDrawOne = 1u << 28;

// What a scan of the rows leaves in the workspace: the row in chunks of kScanVecs vectors (one wave's),
// each with its largest logit m and the sum of exp2((z - m) c) over its tokens, added up in double
// from the float32 sums of its vectors; and the largest logit of every group of `gv` vectors, in the
// logits' format. A chunk with a NaN or a +inf has a NaN sum; one without tokens the largest logit
// -inf.
constexpr int kScanVecs = 512;
constexpr int kScanBlock = 256;
struct TokScan {
  void* gmax;      // [T, ngrp]
  float* cmax;     // [T, nch]
  double* csum;    // [T, nch]
  int32_t nch, ngrp, gv;   // gv = 0: no groups
};
// Vectors per group, for the K largest logits of a row of nvec vectors: 8 (a 128-byte line),
// where that leaves four times as many groups as logits are asked for, or each by itself. (The
// groups whose largest logit is among the K largest of those hold the row's K largest logits; the
// fewer groups, the more else they hold.)
inline int32_t scan_group(int32_t nvec, int64_t K) { return nvec / 8 >= 4 * K ? 8 : 1; }

struct ScanLayout {
  size_t gmax, cmax, csum, total;
  int32_t nch, ngrp, gv;
};
inline ScanLayout scan_layout(int64_t T, int32_t nvec, int elem_bytes, int32_t gv) {
  ScanLayout L{};
  L.nch = (nvec + kScanVecs - 1) / kScanVecs;
  L.gv = gv;
  L.ngrp = gv > 0 ? (nvec + gv - 1) / gv : 0;
  L.csum = 0;
  L.cmax = L.csum + align_up((size_t)T * L.nch * 8, 256);
  L.gmax = L.cmax + align_up((size_t)T * L.nch * 4, 256);
  L.total = L.gmax + align_up((size_t)T * L.ngrp * elem_bytes, 256);
  return L;
}

// The factor of a logit's exponent in base 2.
inline float scan_c(float temperature) { return 1.44269504088896340736f / temperature; }

struct ScanArgs {
  TokRows r;
  TokScan s;
  float c;         // log2(e) / temperature
};

// Where the running sum of a row's weights, in falling order of its logits, reaches top_p of the whole:
// the step of the histogram of weights, what the step has to bring, and how many tokens it holds.
struct DrawStep {
  unsigned long long left;
  int32_t step;      // kFineSteps: the row has no token
  uint32_t count;
};
constexpr int kFine = 64;                  // histogram steps per octave
constexpr int kFineSteps = 29 * kFine;     // (a weight's exponent is at least -28, or it is 0)
constexpr int kHistBlock = 1024;
constexpr int kStepTokens = 8192;          // tokens of its step that a row's list holds

struct SampleArgs {
  TokRows r;
  TokScan s;                  // of the rows at temperature 1
  unsigned long long* draw;   // [T, nch] the chunks' weights
  uint32_t* ties;             // [T, nch] their tokens of a cut's key
  DrawStep* steps;            // [rows]
  uint32_t* step_ids;         // [rows, step_ld] the tokens of the rows' steps
  unsigned long long* hist;   // [rows, parts, kFineSteps] with parts > 1
  int32_t step_ld, parts;
  int32_t weigh_parts;        // workgroups of a row in cis_weigh_kernel
  int64_t row0, rows;         // the launch's first row, and how many
  const float* u;
  cis_sample_params_t prm;
  const float* temperature;   // nullable, as the next three
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int64_t* ids;
  float* logp;                // nullable
  float* logp_kept;           // nullable
};

struct TopArgs {
  TokRows r;
  TokScan s;
  int32_t K;
  float temperature, c;       // c = scan_c(temperature)
  int64_t row0;               // the launch's first row
  int32_t* ids;
  float* values;
  float* tail;                // nullable
};

// The gradient of a row's tokens that are not listed: exp2((z - m) c + up) g.
struct RestGrad {
  float m, up, g;
};

struct DistillArgs {
  TokRows r;
  TokScan s;                  // in parts: the scan at this temperature, without groups
  RestGrad* rest;             // [T] in parts, with the gradient, as the next two
  uint8_t* valid;             // [T]
  uint32_t* grads;            // [T, K] the listed tokens' gradients
  int64_t row0;               // the launch's first row (cis_distill_grad_kernel: segment)
  int32_t nseg;               // segments per row
  float c;                    // scan_c(temperature)
  float inv_t;                // 1 / temperature, and the same in double
  double inv_t64;
  void* dlogits;              // nullable (forward)
  int64_t grow_bytes;
  const int32_t* ids;
  const float* values;
  int64_t ld_top;             // elements
  int32_t K;
  const float* tail;          // nullable
  const float* weight;        // nullable
  int32_t reverse;
  float temperature, scale;
  float* terms_user;          // nullable
  float* terms_ws;            // the loss workspace's arrays (cis_internal.h)
  uint8_t* flags_ws;
  float* logk_ws;
  float* excess_ws;
  FinalizeArgs fin;           // in parts with the gradient: where the statistics go
};

constexpr int kTokBlock = 1024;
constexpr int kTopBlock = 256;
constexpr int kWeighBlock = 256;
constexpr int kDrawK = 1024;      // top_k up to which a row is drawn from a list
constexpr int kDrawListK = 128;   // top_k that the kernel for short lists takes
// keep: the logits stay in the caches for a later kernel's read
const void* scan_kernel(int dtype, int32_t gv, bool keep);
// wide: any parameters; else top_k in [1, 128] for every row or nothing to cut but min_p
const void* sample_kernel(int dtype, bool wide);
const void* weigh_kernel(int dtype, bool step);
const void* hist_kernel(int dtype);
const void* step_kernel();
const void* top_kernel(int dtype, int64_t K);
int top_block(int64_t K);
constexpr int kDistillGradBlock = 128, kDistillGradVecs = 1024;   // 16 KiB of logits per workgroup
struct DistillVariant {
  int block;
  const void* fn;
};
// The fused pass for rows of nvec vectors, and the kernels of the pass in parts.
DistillVariant distill_fused(int dtype, int32_t nvec, int64_t K);
// few: rows that do not fill the chip with a wave each (with bwd all calls are)
const void* distill_row_kernel(int dtype, bool bwd, int64_t K, bool few);
const void* distill_grad_kernel(int dtype);

}  // namespace cis
