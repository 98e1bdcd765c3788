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

struct SampleArgs {
  TokRows r;
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
  int32_t K;
  float temperature;
  int32_t* ids;
  float* values;
  float* tail;                // nullable
};

struct DistillArgs {
  TokRows r;
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
};

constexpr int kTokBlock = 1024;
const void* sample_kernel(int dtype);
const void* top_kernel(int dtype);
const void* distill_kernel(int dtype, bool bwd);

}  // namespace cis
