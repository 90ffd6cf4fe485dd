/*
 * stom_sample.h -- the choice of the next token from a row of logits, on
 * NVIDIA B200 (sm_100a); part of libstom_oqm.so.  Conventions as in stom_kv.h.
 */
#ifndef STOM_SAMPLE_H
#define STOM_SAMPLE_H

#include "stom_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* For every row, with the tokens in descending order of their logits (equal
 * logits: the lower index first), T its temperature and
 *     w_j = exp((x_j - x_max) / T),
 * the tokens kept are a prefix of that order, the shortest that
 *     top_k > 0:  has at most top_k tokens;
 *     top_p < 1:  has a mass (sum of w) of at least top_p times that of what
 *                 top_k left;
 *     min_p > 0:  ends before the first w_j < min_p;
 * ask for, and at least one token.  The token drawn is the first whose mass,
 * with that of all before it, exceeds u times the mass of the kept.  T <= 0
 * takes the first token of the order.
 * Each of temperature, top_k, top_p and min_p may be NULL (1, 0, 1 and 0 for
 * all rows).  u [rows] are the given random numbers, in [0, 1) (values outside
 * are taken to its nearest end); u may be NULL if temperature is given: rows
 * with T > 0 then draw with u = 0, that is, take the first token.
 * A logit of -inf, or one with (x_max - x) / T > 700 (a w below 1e-304), is
 * never kept.  If the largest logit is +inf, the tokens at +inf share the mass.  A NaN logit
 * counts as -inf, a NaN setting as NULL; both set STOM_FLAG_BAD_VALUE.  A row
 * that has nothing to draw from gives token -1, kept 0 and logprob -inf.
 * Masses are exact sums, in no order, of the masses of up to 4 096 ranges of
 * logits, each rounded once to a whole multiple of 2^-43 or less (by n), and
 * binary64 sums over the last few tokens: a token is off only where u falls
 * within 2^-34 (n <= 131 072; else 2^-32) of a border between two.
 * logits (dtype): element (r, j) at r*row_stride + j; any alignment of a
 *   whole element.  1 <= n <= STOM_SAMPLE_MAX_N.
 * token [rows] int32; kept [rows] int32, the number of tokens kept, or NULL;
 * logprob [rows] float, ln(w / mass of the kept) of the token, or NULL.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, CUDA. */
#define STOM_SAMPLE_MAX_N 500000
int32_t stom_sample_tokens(const void *logits, int32_t dtype, int32_t rows, int32_t n, int64_t row_stride,
                           const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                           const float *u, int32_t *token, int32_t *kept, float *logprob, uint32_t *dev_flags,
                           void *stream);

#ifdef __cplusplus
}
#endif
#endif /* STOM_SAMPLE_H */
