/*
 * gdn_paged.h - C ABI of the attention layer that stands beside the gated
 * delta rule in a hybrid model (Sec. 3.4: the rule's layers alternate with
 * sliding-window attention): rotary positions, a cache of keys and values in
 * pages, attention of new tokens over it, and the management of its pages.
 * Same library as gdn.h, whose status codes, data types and conventions
 * (ownership, streams, checks before the first launch) hold here too; what
 * differs is said below.
 *
 * Tokens.  A call works on the tokens of num_seqs sequences, either dense,
 * [B, T, heads, d] with one sequence per row of B, or packed, B == 1 and
 * T tokens in all with the boundaries cu_seqlens (as in gdn_problem; a
 * sequence may have none).  Row tensors are described by gdn_rows: the
 * innermost dim is contiguous, the strides between heads and between tokens
 * are free (q, k and v may be slices of one projection), in dense input the
 * rows of B follow each other at T token strides.
 *
 * Cache.  Sequence n holds kv_lens[n] tokens; token j's key and value stand
 * in slot j % page_size of page table[n][j / page_size].  A page of k (and
 * the page of the same index of v) holds [Hk, page_size, d], with free
 * strides.  A table entry outside [0, num_pages) is a hole: no token sees
 * its keys, nothing is stored there and nothing of it is read, so pages that
 * have left a window can be freed and their entries set to -1.  kv_lens and
 * table live in device memory and are read when the kernels run; values
 * outside [0, max_blocks * page_size] are taken as the nearest bound, so a
 * longer length would put new tokens over the last ones: lengths come from
 * gdn_pages_extend, which does not let them pass the table's room.
 *
 * Where pages may run out, skip (or NULL) is the short_of of the
 * gdn_pages_extend before: a sequence with a non-zero entry there did not get
 * the room for the call's tokens, its kv_lens does not count them, and the
 * places that its length gives them are those of older tokens, perhaps in
 * pages that other sequences share.  It is taken as one that holds no tokens:
 * nothing of it is stored, its tokens see nothing (o = 0, lse = -infinity) and
 * its queries are rotated as the tokens before position 0.  Without skip, the
 * caller has to see to it that no such sequence is in the call.
 *
 * Alignment.  Device pointers are 16-byte aligned and every row (a head of a
 * token, a slot of a page) starts at a multiple of 16 bytes (GDN_ERR_ALIGN).
 * Pointers to int32 arrays are 4-byte aligned.
 */
#ifndef GDN_PAGED_H_
#define GDN_PAGED_H_

#include "gdn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t B, T;     /* tokens: [B, T], packed: B == 1                        */
  int32_t Hq, Hk;   /* query heads, cache heads (attention: Hk divides Hq)   */
  int32_t d;        /* channels of a head: 64, 128 or 256                    */
  int32_t num_seqs; /* packed input: sequences; dense: ignored (B)           */
  const int32_t *cu_seqlens;      /* packed: device int32[num_seqs + 1]      */
  const int32_t *cu_seqlens_host; /* packed: the same values on the host     */
  gdn_dtype dtype;
} gdn_tokens;

typedef struct {
  void *data;
  int64_t token_stride, head_stride; /* elements */
} gdn_rows;

typedef struct {
  void *k, *v;          /* [num_pages, Hk, page_size, d] each                */
  int64_t page_stride, head_stride, token_stride; /* elements, of both       */
  int32_t num_pages;    /* >= 1                                              */
  int32_t page_size;    /* a power of two, 16 to 1024                        */
  int32_t max_blocks;   /* columns of table, >= 1; times page_size at most
                         * 2^31 - 2^18                                       */
  const int32_t *table;   /* device int32[N, max_blocks]                     */
  const int32_t *kv_lens; /* device int32[N]: tokens of each sequence, those
                           * of the call included                            */
  const int32_t *skip;    /* device int32[N] or NULL: sequences to leave alone */
} gdn_cache;

/* ---- rotary positions
 *
 * Pair i of a head's first `rot` channels (rot even, 2..d) is turned by the
 * angle position * theta_i, and scaled:
 *     y1 = s (x1 cos a - x2 sin a),  y2 = s (x2 cos a + x1 sin a);
 * the channels from rot on pass unchanged.  The pair is (i, i + rot / 2) in
 * GDN_ROTARY_HALVES and (2 i, 2 i + 1) in GDN_ROTARY_INTERLEAVED.  The angle
 * is formed as a fraction of a turn in 64 bits, so it keeps full accuracy at
 * any position. */
enum { GDN_ROTARY_HALVES = 0, GDN_ROTARY_INTERLEAVED = 1 };

typedef struct {
  int32_t rot, layout;
  float scale;         /* s; finite                                          */
  const double *turns; /* device double[rot / 2]: theta_i / (2 pi), 8-byte
                        * aligned                                            */
} gdn_rotary;

/* turns[i] = theta_i / (2 pi) on the host, theta_i = base^(-2 i / rot), for a
 * context `factor` times longer than the `original` one the model learnt:
 *   GDN_ROTARY_PLAIN   as it is;
 *   GDN_ROTARY_LINEAR  theta_i / factor (positions interpolated);
 *   GDN_ROTARY_BASE    base * factor^(rot / (rot - 2)) for base (rot > 2);
 *   GDN_ROTARY_PARTS   with r = original * theta_i / (2 pi) turns over the
 *                      original context and g = clamp((r - slow) /
 *                      (fast - slow), 0, 1): theta_i ((1 - g) / factor + g),
 *                      and *scale = 0.1 ln(factor) + 1 (Peng et al. 2023,
 *                      "YaRN", Sec. 3.2-3.4, whose alpha and beta are slow
 *                      and fast).
 * *scale is 1 otherwise.  GDN_ERR_VALUE: rot odd or < 2, base <= 1,
 * factor < 1, original < 1 or fast <= slow (PARTS), values not finite. */
enum { GDN_ROTARY_PLAIN = 0, GDN_ROTARY_LINEAR = 1, GDN_ROTARY_BASE = 2, GDN_ROTARY_PARTS = 3 };
gdn_status gdn_rotary_turns(int32_t rot, double base, int32_t scaling, double factor,
                            double original, double slow, double fast, double *turns,
                            float *scale);

/* Rotation of q [.., Hq, d] and k [.., Hk, d] (k optional, NULL: q alone) into
 * q_out and k_out, which may be the inputs (in place).  positions: device
 * int32[B * T], or NULL: a token's place within its sequence.  The backward
 * turns the gradients of q_out and k_out back (the angle negated, the same
 * scale), which is the transpose of the forward. */
gdn_status gdn_rotary_fwd(const gdn_tokens *t, const gdn_rotary *r, const gdn_rows *q,
                          const gdn_rows *k, const int32_t *positions, const gdn_rows *q_out,
                          const gdn_rows *k_out, void *stream);
gdn_status gdn_rotary_bwd(const gdn_tokens *t, const gdn_rotary *r, const gdn_rows *dq_out,
                          const gdn_rows *dk_out, const int32_t *positions, const gdn_rows *dq,
                          const gdn_rows *dk, void *stream);

/* ---- the cache
 *
 * Stores a call's new tokens: token i of sequence n's m new ones is at
 * position kv_lens[n] - m + i; its k, rotated there, and v go to that slot of
 * the sequence's pages (nowhere if the position is negative or a hole), and q,
 * rotated, to q_out (which may be q).  r == NULL: no rotation; q == NULL (then
 * q_out too): only k and v. */
gdn_status gdn_cache_append(const gdn_tokens *t, const gdn_rotary *r, const gdn_rows *q,
                            const gdn_rows *k, const gdn_rows *v, const gdn_cache *cache,
                            const gdn_rows *q_out, void *stream);

/* Attention of the new tokens over their sequences' cached keys:
 *     o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i k_j) / sum_j' exp(scale q_i k_j')
 * over the keys j that token i sees: 0 <= j < kv_lens[n], no hole; with
 * causal != 0 also j <= its own position kv_lens[n] - m + i; with window > 0
 * (causal only) also j > its position - window.  Query head h reads cache head
 * h / (Hq / Hk).  A token that sees nothing gets o = 0 and lse = -infinity.
 * What is not seen has no influence, whatever bits it holds (infinities and
 * NaN among them).  Scores, the softmax and the sums over keys are in 32 bits.
 * In bfloat16 problems p is rounded to bfloat16 for its product with v (2^-8 of
 * each p v at most; over many keys about as much as the rounding of o); where
 * every sequence has few rows (new tokens x Hq / Hk at most 32; not in batches of
 * over 256 sequences x Hk with at most 1024 keys), it enters as two bfloat16
 * values (2^-16).
 *   lse      fp32 [B * T, Hq] or NULL: log of the sum of exp(scale q k)
 *   max_kv   how many tokens kv_lens is expected to hold at most: the launches
 *            are sized by it (a longer cache costs time, not results); 0:
 *            max_blocks * page_size
 *   scale    > 0, finite
 * A launch holds less than 2^24 workgroups (GDN_ERR_SHAPE past that): one for
 * each sequence and cache head and one for each 64 rows (new tokens x Hq), at
 * most; keys are split only where those are few.
 * The workspace (gdn_cache_attn_workspace_size bytes, 0 where none is needed)
 * holds partial results of keys split over several workgroups.  The same call
 * gives the same bits. */
typedef struct {
  float scale;
  int32_t causal, window, max_kv;
} gdn_attn;

size_t gdn_cache_attn_workspace_size(const gdn_tokens *t, const gdn_cache *cache,
                                     const gdn_attn *a);
gdn_status gdn_cache_attn(const gdn_tokens *t, const gdn_attn *a, const gdn_rows *q,
                          const gdn_cache *cache, const gdn_rows *o, float *lse, void *workspace,
                          size_t workspace_bytes, void *stream);

/* ---- management of the pages, on the device
 *
 * A book of S sequences: table int32[S, max_blocks], lens int32[S] (tokens of
 * each), refs int32[num_pages] (how many rows, or other holders, hold a page;
 * 0: free).  Sequence s holds blocks 0 .. ceil(lens[s] / page_size) - 1; an
 * entry of those outside [0, num_pages) is a hole.  Full pages may be shared
 * between sequences; the last, partly filled page of a sequence is its own.
 * The calls keep that so.  Each reads one book and writes another, whose
 * arrays may be the first's own (in place) and must not overlap it otherwise.
 * Pages are given out lowest index first, to sequences in order: results are
 * whole numbers that depend on the inputs alone.
 *
 * Pool: the data of the pages.  `parts` arrays (k and v of each layer, say) of
 * num_pages pages of page_bytes bytes (a multiple of 16), page p of part i at
 * data + i * part_stride + p * page_stride (bytes, multiples of 16).  A pool
 * of recurrent states is one too (a page: a sequence's state). */
typedef struct {
  int32_t S, max_blocks, num_pages, page_size; /* S, num_pages <= 2^20 */
  const int32_t *table, *lens, *refs;
  int32_t *table_out, *lens_out, *refs_out;
} gdn_book;

typedef struct {
  void *data;
  int32_t parts, num_pages;
  int64_t part_stride, page_stride, page_bytes;
} gdn_pool;

size_t gdn_pages_workspace_size(const gdn_book *b);

/* Room for add[s] more tokens (< 0 is taken as 0) in each sequence: new pages
 * where its blocks do not suffice.  Sequences are served in order while free
 * pages last: one whose new pages, after those of all before it, exceed what
 * was free, or whose blocks exceed max_blocks, keeps its row and length and
 * gets short_of[s] = the new pages it asked for (0: served).  Sequences past
 * max_blocks take no pages from those behind them; those that need no new
 * page are always served.  The cache calls that follow take short_of as the
 * cache's skip, or leave the refused sequences out: what they stored for them
 * would go over older tokens. */
gdn_status gdn_pages_extend(const gdn_book *b, const int32_t *add, int32_t *short_of,
                            void *workspace, size_t workspace_bytes, void *stream);

/* New row i goes on from old row parents[i] (outside [0, S): an empty row):
 * freeing, forking and reordering sequences in one call.  Full pages are
 * shared; the partly filled last page goes to the lowest new row of its
 * parent, every further one gets a free page and a copy of the data in every
 * part of the pool (pool == NULL: no data is copied).  Pages free before the
 * call are given out, in the order of the rows; a row that finds none left
 * becomes empty with short_of[i] = 1 (0 elsewhere).  refs loses the old rows'
 * references and gains the new rows'. */
gdn_status gdn_pages_select(const gdn_book *b, const int32_t *parents, const gdn_pool *pool,
                            int32_t *short_of, void *workspace, size_t workspace_bytes,
                            void *stream);

/* Moves the pages in use (refs > 0) into the lowest indexes: with n of them,
 * the i-th free page below n receives the i-th page in use from n on; its data
 * moves in every part of the pool (pool == NULL: none).  The table and refs
 * are renumbered, map[p] (int32[num_pages]) is the new index of page p, -1 if
 * it was free.  Entries past a sequence's blocks and holes become -1.  lens is
 * unchanged and lens_out not used. */
gdn_status gdn_pages_compact(const gdn_book *b, const gdn_pool *pool, int32_t *map,
                             void *workspace, size_t workspace_bytes, void *stream);

/* Copies pages src[i] to dst[i], i < n, in every part of the pool (device
 * int32 arrays).  A pair with an index outside [0, num_pages) is skipped.  No
 * page may be both a source and a destination, or a destination twice. */
gdn_status gdn_pages_copy(const gdn_pool *pool, const int32_t *src, const int32_t *dst, int32_t n,
                          void *stream);

#ifdef __cplusplus
}
#endif
#endif /* GDN_PAGED_H_ */
