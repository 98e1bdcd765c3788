/*
 * cis_tokens.h — C ABI of the per-token operators around the CIS loss on MI355X (gfx950): drawing
 * a token from each row of logits, the list of a row's largest logits, and the distillation loss
 * against such a list, forward and backward.
 *
 * The conventions of cis.h hold here too: device pointers owned by the caller, asynchronous calls
 * on `stream` that launch kernels only (no allocation, memset or copy; they can be captured into a
 * HIP graph), arguments checked before the first launch, identical bits for identical calls, masks
 * read as aligned 4-byte words. Logits are [T, ld] bf16 or float32, row-major; base address and
 * ld * sizeof(element) are multiples of 16 bytes; columns [V, ld) are never used.
 *
 * A logit of -inf is no token: it is never drawn and never listed. Equal logits are ordered by
 * their ids, the lowest first (+0 and -0 are equal).
 */
#ifndef CIS_TOKENS_H
#define CIS_TOKENS_H

#include "cis.h"

#ifdef __cplusplus
extern "C" {
#endif

/* =========================================================================================
 * Sampling. For a row z with its parameters (temperature, top_k, top_p, min_p) and its random
 * number u in [0, 1):
 *
 *   M    = max_j z_j
 *   q_j  = floor(2^28 * exp2((z_j - M) * c)),  c = log2(e) / temperature; the difference, c and the
 *          product are rounded to float32, and exp2 is the device's own in float32 (within a unit in
 *          the last place: 16 of 2^28 for a token near the largest)
 *   cuts, each a first part of the tokens in order of (z_j descending, j ascending):
 *     top_k   the first top_k tokens                                         (0: all)
 *     top_p   of those, the fewest whose sum of q reaches top_p times the sum over those (1: all)
 *     min_p   the tokens with q_j >= min_p * 2^28                             (0: all)
 *   kept = the tokens in every cut, N = sum of q over kept
 *   y    = the lowest id whose running sum of q over the kept ids <= y exceeds floor(u * N)
 *
 * The weights q are whole numbers, so with them the sums and the draw are exact and do not depend on an
 * order of summation; a token of probability below 2^-28 of the row's largest has weight 0. (top_p * sum,
 * min_p * 2^28 and u * N are formed in double.)
 * temperature = 0, or one so small that c is not finite, keeps the first token alone (greedy).
 *
 *   logp      = log softmax(z)_y over the whole row at temperature 1: the value that the loss entry
 *               points take as logp_infer
 *   logp_kept = log(q_y / N): under the distribution that y was drawn from
 *
 * Not drawn, with id -1 and log-probabilities 0: masked rows, rows without a token, with a NaN or
 * a +inf, and rows whose own parameters are out of range (u outside [0, 1) included). The loss entry
 * points count such an id as out of range and give its row no gradient.
 * ========================================================================================= */
typedef struct cis_sample_params {
  float temperature; /* >= 0, finite                                                    */
  int32_t top_k;     /* >= 0; 0: no limit                                               */
  float top_p;       /* in (0, 1]; 1: no limit                                          */
  float min_p;       /* in [0, 1]; 0: no limit                                          */
} cis_sample_params_t;

/* Bytes of device workspace for cis_sample. Returns 0 for T < 0, V outside [1, 2^28] or an
 * unknown dtype. */
size_t cis_sample_workspace_bytes(int64_t T, int64_t V, int dtype);

/*
 * cis_sample — one token per row.
 *
 *   u      [T] float       the rows' random numbers
 *   mask   [T] uint8       nonzero = draw for this row; NULL = for every row
 *   params                 the parameters of every row (a host struct, read during the call) ...
 *   temperature [T] float, top_k [T] int32, top_p [T] float, min_p [T] float
 *                          ... except those given here, one per row (NULL = the one in params)
 *   ids_out [T] int64      the drawn ids
 *   logp_out, logp_kept_out [T] float   NULL = not written
 *   workspace              >= cis_sample_workspace_bytes(T, V, dtype) bytes, 256-byte aligned
 * Errors: CIS_ERR_NULL, CIS_ERR_SHAPE, CIS_ERR_DTYPE, CIS_ERR_PARAM (a value of params out of its
 * range, where no array replaces it), CIS_ERR_ALIGN, CIS_ERR_WORKSPACE, CIS_ERR_LAUNCH,
 * CIS_ERR_DEVICE.
 */
int cis_sample(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const float* u,
               const uint8_t* mask, const cis_sample_params_t* params, const float* temperature,
               const int32_t* top_k, const float* top_p, const float* min_p, int64_t* ids_out,
               float* logp_out, float* logp_kept_out, void* workspace, size_t workspace_bytes,
               hipStream_t stream);

/* =========================================================================================
 * The largest logits of each row, and what is left of its distribution.
 *
 *   ids    [T, K] int32   the ids of the K largest logits, in order; -1 past the row's last token
 *   values [T, K] float   their logits; -inf past the row's last token
 *   tail   [T]    float   log sum exp(z_j / temperature) over the tokens that are not listed, summed
 *                         without the listed ones (-inf where there are none)
 * so that the list and the tail hold the row's softmax at that temperature: what a teacher leaves
 * behind for a distillation step. Rows that are masked or hold a NaN or a +inf list nothing: ids
 * -1, values -inf, and tail -inf (masked) or NaN.
 * ========================================================================================= */
#define CIS_TOP_MAX_K 1024

size_t cis_top_logits_workspace_bytes(int64_t T, int64_t V, int64_t K, int dtype);

/*
 * cis_top_logits
 *   mask        [T] uint8     NULL = every row counts
 *   K           entries per row, 1 <= K <= CIS_TOP_MAX_K (K may exceed V)
 *   temperature               in [2^-64, 2^64]; moves the tail only
 *   ids_out     [T, K] int32, values_out [T, K] float
 *   tail_out    [T] float     NULL = not written
 * Errors: CIS_ERR_NULL, CIS_ERR_SHAPE (K out of range included), CIS_ERR_DTYPE, CIS_ERR_PARAM,
 * CIS_ERR_ALIGN, CIS_ERR_WORKSPACE, CIS_ERR_LAUNCH, CIS_ERR_DEVICE.
 */
int cis_top_logits(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                   const uint8_t* mask, int64_t K, float temperature, int32_t* ids_out,
                   float* values_out, float* tail_out, void* workspace, size_t workspace_bytes,
                   hipStream_t stream);

/* =========================================================================================
 * Distillation against a teacher's largest logits.
 *
 * A row's list (i_k, v_k), k < K, and its tail give the teacher's distribution over the listed
 * tokens and "everything else":
 *
 *   q_k = exp(v_k / temperature) / S,  q_rest = exp(tail) / S,  S = the sum of all of them
 *   (tail = NULL: q_rest = 0, the teacher's softmax over its list alone)
 *
 * The student p = softmax(z / temperature) is collapsed to the same classes: p_k = p[i_k] and
 * p_rest, the sum over the tokens that are not listed (summed by itself, so that it keeps its
 * relative accuracy as the list takes all of the mass). With weight a_t of the row:
 *
 *   CIS_KL_FORWARD  term = scale * a_t * sum_b q_b log(q_b / p_b)
 *   CIS_KL_REVERSE  term = scale * a_t * sum_b p_b log(p_b / q_b)       (needs the tail)
 *
 * over the classes b, each evaluated as a sum of a log(a/b) - a + b >= 0, whose terms do not
 * cancel. The gradient is that of the sum of the terms with respect to the logits:
 *
 *   forward  dz_j = scale * a_t / temperature * (p_j - q_j)                  listed
 *                   scale * a_t / temperature * p_j (1 - q_rest / p_rest)    others
 *   reverse  dz_j = scale * a_t / temperature * p_j (log(p_b / q_b) - KL)    b the class of j
 *
 * Ids of -1 are empty entries. A row is valid when it is not masked, its list has an entry, and its
 * ids are -1 or in [0, V) and do not repeat; other rows have term 0 and a zero gradient row, and
 * those with ids out of range or repeated are counted as n_bad_id. A row whose weight is 0 has term
 * 0 and a zero gradient. Valid rows whose sums or term are not finite (a NaN or +inf logit or value,
 * no token, a class that the first argument has and the second has not) are counted as n_nonfinite.
 * ========================================================================================= */
typedef enum { CIS_KL_FORWARD = 0, CIS_KL_REVERSE = 1 } cis_kl_t;

typedef struct cis_distill_params {
  int32_t kind;      /* cis_kl_t                                                          */
  float temperature; /* in [2^-64, 2^64]                                                 */
  float scale;       /* loss normalisation (finite)                                      */
} cis_distill_params_t;

/* Returns 0 for T < 0, V outside [1, 2^28], K outside [1, CIS_TOP_MAX_K] or an unknown dtype. */
size_t cis_distill_workspace_bytes(int64_t T, int64_t V, int64_t K, int dtype);

/*
 * cis_distill_fwd / cis_distill_bwd — the loss, and the loss with its gradient.
 *
 *   top_ids    [T, ld_top] int32, top_values [T, ld_top] float   the first K columns are the lists
 *              (K <= ld_top); what cis_top_logits writes has ld_top = K
 *   top_tail   [T] float   NULL: the list is all that the teacher has (CIS_KL_FORWARD only)
 *   row_weight [T] float   a_t; NULL = 1 for every row
 *   mask       [T] uint8   NULL = every row counts
 *   dlogits    [T, ld_g]   like logits; every row is written, columns [V, ld_g) are not. May be the
 *              logits buffer itself when ld_g == ld; other overlaps are CIS_ERR_ALIAS. Gradient
 *              values of magnitude below 2^-126 may be flushed to zero.
 *   terms_out  [T] float   NULL = not written
 *   loss_out   [1] float   the sum of the terms; NULL = not written
 *   workspace  >= cis_distill_workspace_bytes(T, V, K, dtype) bytes, 256-byte aligned; receives a
 *              cis_stats_t (loss, n_valid, n_bad_id, n_nonfinite; the other fields are 0)
 * Errors: CIS_ERR_NULL, CIS_ERR_SHAPE (K outside [1, CIS_TOP_MAX_K], ld_top < K), CIS_ERR_DTYPE,
 * CIS_ERR_PARAM (CIS_KL_REVERSE without a tail included), CIS_ERR_ALIGN, CIS_ERR_WORKSPACE,
 * CIS_ERR_ALIAS, CIS_ERR_LAUNCH, CIS_ERR_DEVICE.
 */
int cis_distill_fwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                    const int32_t* top_ids, const float* top_values, int64_t K, int64_t ld_top,
                    const float* top_tail, const float* row_weight, const uint8_t* mask,
                    const cis_distill_params_t* params, float* terms_out, float* loss_out,
                    void* workspace, size_t workspace_bytes, hipStream_t stream);

int cis_distill_bwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                    const int32_t* top_ids, const float* top_values, int64_t K, int64_t ld_top,
                    const float* top_tail, const float* row_weight, const uint8_t* mask,
                    const cis_distill_params_t* params, void* dlogits, int64_t ld_g,
                    float* terms_out, float* loss_out, void* workspace, size_t workspace_bytes,
                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CIS_TOKENS_H */
