/*
 * lookat_search.h -- beam search's selection over beams and vocabulary.
 *
 * The general rules, status codes and error text of lookat.h hold here too.
 */
#ifndef LOOKAT_SEARCH_H
#define LOOKAT_SEARCH_H

#include "lookat.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The n best continuations of each of Q requests.  Rows q*beams .. q*beams + beams - 1 of logits are the beams of request q, scores their
 * log-probabilities so far; token v of row r makes
 *     scores[r] + logits[r,v] - log sum_u exp(logits[r,u])
 * Candidates of a request are ordered by that, falling, equal ones by (row, token), rising; the first n are written.  A row's candidates are ordered
 * as its logits are whatever the rounding of the sum.  Candidates are compared in 64 bits; the log of a row's sum is good to 2^-18 (to 5.4e-7 in
 * what was measured: rows with most of their weight in equal logits far below the maximum), so that two beams' candidates whose scores lie closer
 * than 2^-17 may change places.  The score that is written is rounded to fp32 once, below its range to its lowest number.
 * A logit of -inf is a token that cannot be chosen, a score of -inf a beam that has none (one that ended; all but the first of a request that
 * begins).  A row that has a NaN or +inf among its logits, or whose score is NaN or +inf, gives no candidate either.  Where a request has fewer than n
 * candidates the rest is -inf, -1, -1.
 *   logits        fp16 or fp32, element (r,v) at logits[r*logit_stride + v], logit_stride >= V; any alignment of its type
 *   scores        [Q*beams] fp32
 *   scores_out    [Q,n] fp32, which may be scores where n = beams;  tokens [Q,n] int32
 *   parents       [Q,n] int32: first_parent + r, what lookat_pages_fork takes as sources if the beams' sequences are the slots from first_parent on
 *                 (a -1 is passed over there)
 *   workspace     lookat_beam_select_workspace_bytes(Q, beams, V, n) bytes, 16-byte aligned; calls in flight at once must not share one
 * Supported: 1 <= n <= 64, 1 <= beams <= 1024, Q*beams <= 65535, V <= 2^24; otherwise LOOKAT_ERR_UNSUPPORTED or LOOKAT_ERR_SHAPE.
 */
size_t lookat_beam_select_workspace_bytes(int32_t Q, int32_t beams, int32_t V, int32_t n);

int lookat_beam_select(int32_t Q, int32_t beams, int32_t V, int32_t n,
                       const void *logits, lookat_dtype logit_dtype, int64_t logit_stride,
                       const float *scores, int32_t first_parent,
                       float *scores_out, int32_t *parents, int32_t *tokens,
                       void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LOOKAT_SEARCH_H */
