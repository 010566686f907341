/*
 * libenec, third part -- the end of a decoding step, on AMD MI355X (gfx950): one token for each row of logits, drawn with temperature,
 * top-k, top-p and min-p from random numbers that the caller gives.
 *
 * Conventions are those of enec.h and enec_lowbit.h: plain pointers and sizes, status codes of enec_status, all work enqueued on
 * `stream`, no device memory allocated by the library, errors that the host can see return before anything is enqueued, a workspace is
 * scratch memory, and a call can be captured into a graph.  Results do not depend on the timing of a run: weights are summed as whole numbers.
 */
#ifndef ENEC_SAMPLING_H
#define ENEC_SAMPLING_H

#include "enec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What a row is drawn with: arrays on the DEVICE, an entry for each row; NULL leaves a filter out. */
typedef struct {
    const float *temperature;      /* NULL: 1 */
    const int32_t *top_k;          /* 0 and below, or vocab and above: all tokens */
    const float *top_p;            /* 1 and above: all; 0 and below: the first token only */
    const float *min_p;            /* 0 and below: all; over 1: the first token only */
    const float *uniform;          /* from 0 to below 1; not NULL */
} enec_sampling;

/* A token for each row.
 *   logits  DEVICE, rows x vocab values (bf16, fp16 or fp32), row_stride elements from row to row (>= vocab)
 *   tokens  DEVICE, int32, rows entries
 *   log_probs  DEVICE, fp32, rows entries, or NULL: the natural logarithm of the probability that the token was drawn with
 *   workspace  DEVICE, 16-byte aligned, or NULL if workspace_bytes = enec_sample_workspace(rows, vocab) is 0.  What it says serves every
 *           call with no more rows and the same vocab as well.  It is 57 KB for each part of a row and 16 bytes a row; a row has 16 parts,
 *           all rows no more than 1024 together, but one for each 65536 tokens of a row (16 at most) in any case: 0.9 MB for one row, 59 MB for 64
 *           to 1024 rows of up to 65536 tokens, 471 MB for 4096 rows of 131072.
 * With l a row's logits, L the largest, T the temperature: w[i] = exp((l[i] - L) / T), 0 where l[i] is minus infinity (L plus infinity: 1 where
 * l[i] is, 0 elsewhere).  The tokens in descending order of l, ties in ascending order of i (0 and -0 are a tie), are cut three times:
 *   top_k   the first top_k of them
 *   top_p   of those the fewest first whose w reach top_p times the sum of those
 *   min_p   of those the first, and the others with w[i] >= min_p
 * and the token is the least i at which the sum of the kept w[0 ... i] exceeds uniform times the sum of all kept.  T = 0: the first of the order.
 * Weights are computed in 64 bits and held as multiples of 2^-46 (a vocabulary beyond 65536 tokens: of 2^-62 times it, rounded up to a power of
 * two); smaller ones than half of that are never drawn.
 * The token is -1, and log_probs NaN, of a row that has a NaN, nothing but minus infinities, or a temperature, top_p, min_p or uniform out of
 * range (T below zero or not finite, NaN, uniform outside [0, 1)).
 * ENEC_E_ARG also if vocab is 0 or exceeds 2^22, or rows, or rows times the vocabulary's pieces of 65536 (at most 16), exceed 2^22. */
size_t enec_sample_workspace(size_t rows, size_t vocab);
int enec_sample(const void *logits, size_t rows, size_t vocab, size_t row_stride, int dtype, const enec_sampling *how, int32_t *tokens,
                float *log_probs, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ENEC_SAMPLING_H */
