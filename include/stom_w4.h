/*
 * stom_w4.h -- products with 4-bit weights, on NVIDIA B200 (sm_100a); part of
 * libstom_oqm.so.  Conventions as in stom_kv.h.
 *
 * A pass over one or a few tokens reads every weight once and does little else,
 * and a weight of 4 bits is a quarter of one of 16.  More than 64 tokens are taken
 * 64 at a time.
 */
#ifndef STOM_W4_H
#define STOM_W4_H

#include "stom_oqm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A matrix of n rows (outputs) and k columns (inputs), in groups of `group`
 * adjacent columns:
 *     W[r][c] = code[r][c] * scale[r][c / group] + zero[r][c / group]
 * or, where zero is NULL, (code[r][c] - 8) * scale[r][c / group].  Two codes a
 * byte, that of the even column in the low half. */
typedef struct stom_w4_matrix {
    const uint8_t *codes;   /* [n][k/2] bytes, rows code_stride bytes apart; 16-byte aligned rows          */
    const void *scale;      /* [n][k/group] of meta_dtype, rows meta_stride elements apart                 */
    const void *zero;       /* like scale, or NULL                                                         */
    int32_t n, k;           /* k: a multiple of group                                                      */
    int32_t group;          /* 32, 64 or 128                                                               */
    int32_t meta_dtype;     /* STOM_BF16 | STOM_FP16 | STOM_FP32                                           */
    int64_t code_stride;    /* bytes, a multiple of 16                                                     */
    int64_t meta_stride;    /* elements                                                                    */
} stom_w4_matrix;

/* y[t][r] = sum_c x[t][c] W[r][c] + bias[r] + add[t][r] for `rows` tokens t.
 * Products of a token's 16-bit values with codes are summed in binary32 group
 * by group, the groups' sums scaled and summed in binary32, and the result is
 * rounded once to dtype.
 * x, add, y (dtype: STOM_BF16 | STOM_FP16): element (t, i) at t*stride + i; x
 * and its stride 16-byte aligned, the others any alignment of an element.
 * x values below 2^-24 (fp16) or 2^-27 (bf16) of the largest of their token and
 * group may lose bits, 2^-35 of that at most; a token with a value that is no finite
 * number gives no finite numbers.
 * bias [n] (dtype) and add may be NULL; add may be y; x and y do not overlap.
 * STOM_FLAG_TIMEOUT in the optional dev_flags: a bounded wait inside a kernel
 * ran out, y is not to be used.
 * workspace: 128-byte aligned, of at least stom_w4_workspace_bytes() bytes, asked
 * for with the same device current; its contents do not matter, and it may be used
 * by one call at a time.  None is needed for few tokens, whose operands of all
 * columns fit into a multiprocessor's shared memory: up to 8 (16 of the smallest
 * and largest matrices) of 3 840 columns, 5 of 5 632, one of 17 408 in groups of
 * 32, and of 4 096, 6 400 and 27 648 in groups of 128.  k <= 2^24, n < 2^23 - 127, rows <= 524 280.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED, ALIGNMENT, WORKSPACE, CUDA. */
int64_t stom_w4_workspace_bytes(const stom_w4_matrix *w, int32_t rows);
int32_t stom_w4_linear(const stom_w4_matrix *w, int32_t dtype, int32_t rows, const void *x, int64_t x_stride,
                       const void *bias, const void *add, int64_t add_stride, void *y, int64_t y_stride,
                       void *workspace, int64_t workspace_bytes, uint32_t *dev_flags, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* STOM_W4_H */
