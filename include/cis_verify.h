/*
 * cis_verify.h — C ABI of the verification of drafted tokens on MI355X (gfx950): a cheap draft proposes the
 * next tokens of each sequence, the target model scores them all at once, and the accepted ones and
 * one token more are distributed as the target's own draws (cis_sample) would be.
 *
 * The conventions of cis.h and cis_tokens.h hold here too: device pointers owned by the caller,
 * asynchronous calls on `stream` that launch kernels only, arguments checked before the first launch,
 * identical bits for identical calls; logits with rows of whole 16-byte vectors, -inf for no token.
 */
#ifndef CIS_VERIFY_H
#define CIS_VERIFY_H

#include "cis_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/* =========================================================================================
 * Sequence s has the target's rows [seq_offsets[s], seq_offsets[s+1]): at each but the last a token was
 * drafted, and row t's draft is entry t - s of the drafts (one after the other, no gaps). The last row
 * holds the target's logits after the last draft; a sequence of one row has no drafts, and is a draw. A
 * sequence without rows yields nothing, and comes behind all others that have some (an entry of the
 * drafts would be its own otherwise).
 *
 * A row's weights are those of cis_sample (cis_tokens.h), under the sequence's temperature, top_k, top_p
 * and min_p: whole numbers, 0 for tokens that a cut leaves out. P are the target's and N their sum; Q
 * and N' the same of the draft's logits, and rho = N / N' (Without draft logits the drafts are certain:
 * Q is N' for the drafted token.) In double, rounded at each step:
 *
 *   row by row, draft d is accepted when   u * (Q_d * rho) < P_d
 *   the first that is not ends the sequence: a token is drawn in its place from the weights
 *                       max(P_j - floor(Q_j * rho), 0)     (from P where all of them are 0)
 *   after the last draft a token is drawn from P
 *
 * with the row's own random number u for a draft, and that of the sequence's last row for the draw, by
 * the rule of cis_sample: the lowest id whose running sum exceeds floor(u * sum).
 *
 *   ids        the accepted drafts and the drawn token; -1 for the sequence's other rows, and for rows
 *              that no sequence has
 *   accepted   how many drafts were accepted (-1: the sequence's offsets are out of range; where offsets fall,
 *              the others that share its rows are undefined)
 *   logp       log softmax of the target's row at its token, at temperature 1: what the loss entry
 *              points take as logp_infer
 *   logp_kept  log(P_y / N)
 *
 * A sequence ends before a row that cannot be drawn from (cis_sample), whose draft's row cannot, or
 * whose draft is no id in [0, V): accepted counts the drafts ahead of it, and the row has id -1.
 * Log-probabilities of rows without an id are 0.
 * ========================================================================================= */

/* Bytes of device workspace for T rows of the target and D drafts with logits (0 without them) in
 * n_seq sequences. Returns 0 for a negative count, T + D > 2^31, V outside [1, 2^28] or an unknown dtype. */
size_t cis_verify_workspace_bytes(int64_t T, int64_t D, int64_t n_seq, int64_t V, int dtype);

/*
 * cis_verify
 *   logits       [T, ld]    the target's, bf16 or float32
 *   draft_logits [D, ld_d]  the draft's, of the same type; NULL: the drafts are certain
 *   draft_ids    [D] int64
 *   u            [T] float  in [0, 1)
 *   seq_offsets  [n_seq+1] int64, rising; rows from seq_offsets[n_seq] on belong to no sequence and
 *                are not read
 *   params                  the parameters of every sequence (a host struct, read during the call) ...
 *   temperature [n_seq] float, top_k [n_seq] int32, top_p [n_seq] float, min_p [n_seq] float
 *                           ... except those given here, one per sequence (NULL = the one in params)
 *   ids_out [T] int64, accepted_out [n_seq] int32
 *   logp_out, logp_kept_out [T] float   NULL = not written
 *   workspace               >= cis_verify_workspace_bytes(T, draft_logits ? D : 0, n_seq, V, dtype)
 *                           bytes, 256-byte aligned
 * No output overlaps another argument, nor does the workspace (as many bytes of it as are needed):
 * CIS_ERR_ALIAS.
 * Errors: CIS_ERR_NULL, CIS_ERR_SHAPE (n_seq < 1 with T > 0 included), CIS_ERR_DTYPE, CIS_ERR_PARAM (as
 * for cis_sample), CIS_ERR_ALIGN, CIS_ERR_WORKSPACE, CIS_ERR_LAUNCH, CIS_ERR_DEVICE, CIS_ERR_ALIAS.
 */
int cis_verify(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
               const void* draft_logits, int64_t D, int64_t ld_d, const int64_t* draft_ids,
               const float* u, const int64_t* seq_offsets, int64_t n_seq,
               const cis_sample_params_t* params, const float* temperature, const int32_t* top_k,
               const float* top_p, const float* min_p, int64_t* ids_out, int32_t* accepted_out,
               float* logp_out, float* logp_kept_out, void* workspace, size_t workspace_bytes,
               hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CIS_VERIFY_H */
