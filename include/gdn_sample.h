/*
 * gdn_sample.h - C ABI of the choice of the next token from a model's logits.
 * Same library as gdn.h, whose status codes, data types and conventions
 * (ownership, streams, checks before the first launch) hold here too.
 *
 * For each row, with logits l_i, temperature T and a given random number u:
 *
 *  - Tokens are ordered by falling l_i, the lowest index first among equals.  A
 *    NaN is never drawn; +infinity takes all there is.
 *  - T <= 0 (or NaN): the first of them, with probability 1.
 *  - Else w_i = exp((l_i - max l) / T), and w_i below 2^-43 counts as 0.
 *    top_k > 0 keeps the first top_k; then top_p < 1 the shortest prefix of these
 *    that holds at least top_p of their sum (at least one token); then min_p > 0
 *    those with w_i >= min_p (at least one).
 *  - The drawn token is the first of the kept ones up to which the sum of w passes u
 *    times the sum of all kept; its logprob is log(w / that sum).
 *  - A row without anything to draw (only NaN and -infinity) gives token -1 and logprob
 *    -infinity.
 *
 * Sums are of whole multiples of 2^-42 held in 64 bits: they do not depend on an order,
 * and the same call gives the same tokens.
 */
#ifndef GDN_SAMPLE_H_
#define GDN_SAMPLE_H_

#include "gdn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t rows;       /* 1 to 2^22 - 1                                    */
  int32_t vocab;      /* 1 to 2^20                                        */
  gdn_dtype dtype;    /* of the logits                                    */
  const void *logits; /* [rows, vocab], aligned to an element             */
  int64_t row_stride; /* elements from a row to the next                  */
  /* device arrays [rows], or NULL                                        */
  const float *temperature; /* NULL: 1                                    */
  const int32_t *top_k;     /* <= 0 (or NULL): off                        */
  const float *top_p;       /* >= 1, NaN (or NULL): off; <= 0: one token  */
  const float *min_p;       /* <= 0, NaN (or NULL): off                   */
  const float *u;           /* [rows], in [0, 1); outside: the nearest of
                             * them; may be NULL if temperature is given
                             * and no row of it is above 0                */
} gdn_sampling;

/*   out: tokens int32 [rows]; logprob float32 [rows], or NULL to skip. */
gdn_status gdn_sample(const gdn_sampling *s, int32_t *tokens, float *logprob,
                      void *stream);

#ifdef __cplusplus
}
#endif
#endif /* GDN_SAMPLE_H_ */
