/*
 * gdn_linear.h - C ABI of linear attention with a decay for each head, the other
 * recurrent layer of the paper's hybrid models (Sec. 3.4: blocks of this kind
 * beside those of the gated delta rule and window attention).  Same library
 * as gdn.h, whose status codes, problem description, layouts and conventions
 * (ownership, streams, checks before the first launch) hold here too; what
 * differs is said below.
 *
 * The operation, for each sequence and head, with the state a dk x dv matrix:
 *
 *     S_t = alpha_t S_{t-1} + k_t v_t^T,    o_t = S_t^T q_t,    alpha_t = exp(log_alpha_t)
 *
 * (the rule of gdn.h without its correction, Sec. 2.1, Eq. mamba2-update-o).  No scale is applied to q.
 * These are the forms that serve a model: prompts in chunks, and token by
 * token.
 *
 *  - Head dims: dk in {64, 128, 256} and dv in {64, 128, 256, 512}, any pair,
 *    in bfloat16 (fp32 sums and states) and in float32.  In chunks of bfloat16 the products
 *    for o take the state and the tokens' weights to 2^-16 of their values, and o is
 *    rounded once; what a token adds to the state keeps all 24 bits.
 *  - log_alpha: float32 [B, T, H], or with per_head != 0 float32 [H], the same
 *    decay for every token of a head; NULL: alpha == 1.  Values are expected
 *    to be <= 0; -infinity forgets all that came before the token.
 *  - An infinity or NaN in a token reaches no earlier token of its sequence and no
 *    other sequence or head; one in v stays in its column, one in k in its row of the
 *    state, as the infinity that its product with v is (chunks make it a NaN where the
 *    alphas behind it, multiplied together, fall below what float32 holds), and one in q in
 *    its token's row of o (in chunks as an infinity or NaN).
 *  - Outputs must not overlap inputs, but ht may be h0 (updated in place).
 *  - The same call on the same inputs gives the same bits; a sequence's results
 *    can differ in rounding between calls whose B, H or boundaries differ
 *    (where there are few sequences, their chunks are walked in several pieces
 *    at a time).
 */
#ifndef GDN_LINEAR_H_
#define GDN_LINEAR_H_

#include "gdn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Prompts: all tokens of the call, in chunks of 64.
 *   in : q, k [B, T, H, dk], v [B, T, H, dv]; log_alpha (see above); h0 = initial
 *        states [Nseq, H, dk, dv] or NULL (zero)
 *   out: o [B, T, H, dv]; ht = final states, or NULL to skip (of a sequence without
 *        tokens: its initial state).
 * workspace: gdn_linear_chunk_fwd_workspace_size(p) bytes (0 if none is needed, or if the
 * problem is invalid). */
size_t gdn_linear_chunk_fwd_workspace_size(const gdn_problem *p);
gdn_status gdn_linear_chunk_fwd(const gdn_problem *p, const void *q, const void *k,
                                const void *v, const float *log_alpha,
                                int32_t per_head, const float *h0, void *o,
                                float *ht, void *workspace,
                                size_t workspace_bytes, void *stream);

/* Token by token: the same operation for few tokens (T = 1: one decode step).  The state is
 * read once and written once, whatever T.  No workspace. */
gdn_status gdn_linear_recurrent_fwd(const gdn_problem *p, const void *q, const void *k,
                                    const void *v, const float *log_alpha,
                                    int32_t per_head, const float *h0, void *o,
                                    float *ht, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* GDN_LINEAR_H_ */
