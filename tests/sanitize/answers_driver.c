/* The host side of linear attention, of attention over a shared prefix and of the choice of tokens
 * without a GPU: sizes over the range of what is allowed, and refusals. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../../include/gdn_linear.h"
#include "../../include/gdn_paged.h"
#include "../../include/gdn_sample.h"

static uint64_t state = 12345;
static int below(int n) {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return (int)((state >> 33) % (uint64_t)n);
}
static void expect(int ok, const char *what) {
  if (ok) return;
  printf("answers driver: %s\n", what);
  exit(1);
}

int main(void) {
  void *const x = (void *)0x10000;
  const int dks[] = {64, 128, 256}, dvs[] = {64, 128, 256, 512};
  for (int i = 0; i < 3000; ++i) {
    gdn_problem p;
    memset(&p, 0, sizeof p);
    p.B = 1 + below(i % 3 ? 64 : 2);
    p.T = 1 + below(i % 5 ? 20000 : 20000000);
    p.H = 1 + below(i % 7 ? 16 : 200);
    p.dk = dks[below(3)];
    p.dv = dvs[below(4)];
    p.dtype = below(2) ? GDN_BF16 : GDN_F32;
    int32_t *host = NULL;
    if (below(2)) {
      p.B = 1;
      p.num_seqs = 1 + below(100);
      host = malloc((size_t)(p.num_seqs + 1) * sizeof *host);
      host[0] = 0;
      for (int n = 1; n < p.num_seqs; ++n)
        host[n] = host[n - 1] + (below(3) ? below((p.T - host[n - 1]) / 2 + 1) : 0);
      host[p.num_seqs] = p.T;
      p.cu_seqlens = x;
      p.cu_seqlens_host = host;
    }
    const size_t need = gdn_linear_chunk_fwd_workspace_size(&p);
    if (need) {
      /* a state for each segment at least */
      expect(need >= (size_t)2 * p.H * p.dk * p.dv * 4, "a workspace of less than two segments");
      expect(gdn_linear_chunk_fwd(&p, x, x, x, NULL, 0, NULL, x, NULL, NULL, 0, NULL) ==
                 GDN_ERR_WORKSPACE, "no workspace");
      expect(gdn_linear_chunk_fwd(&p, x, x, x, NULL, 0, NULL, x, NULL, x, need - 1, NULL) ==
                 GDN_ERR_WORKSPACE, "a short workspace");
    }
    expect(gdn_linear_chunk_fwd(&p, NULL, x, x, NULL, 0, NULL, x, NULL, x, need, NULL) != GDN_OK,
           "no q");
    expect(gdn_linear_recurrent_fwd(&p, x, x, NULL, NULL, 0, NULL, x, NULL, NULL) != GDN_OK, "no v");
    if (host) host[p.num_seqs] = p.T + 1;
    if (host) expect(gdn_linear_chunk_fwd_workspace_size(&p) == 0, "boundaries past the end");
    free(host);
  }
  expect(gdn_linear_chunk_fwd_workspace_size(NULL) == 0, "no problem");

  for (int i = 0; i < 3000; ++i) {
    gdn_tokens t;
    gdn_cache c;
    gdn_attn a;
    memset(&t, 0, sizeof t);
    memset(&c, 0, sizeof c);
    memset(&a, 0, sizeof a);
    t.B = 1 + below(i % 3 ? 256 : 4);
    t.T = 1 + below(i % 4 ? 4 : 3000);
    t.Hk = 1 + below(8);
    t.Hq = t.Hk * (1 + below(8));
    t.d = 64 << below(3);
    t.dtype = below(2) ? GDN_BF16 : GDN_F32;
    c.k = c.v = x;
    c.table = c.kv_lens = x;
    c.page_size = 16 << below(7);
    c.num_pages = 1 + below(1000);
    c.max_blocks = 1 + below((1 << (i % 5 ? 12 : 20)) / c.page_size * 16);
    c.token_stride = t.d;
    c.head_stride = (int64_t)t.d * c.page_size;
    c.page_stride = c.head_stride * t.Hk;
    a.scale = 0.1f;
    a.causal = 1;
    a.window = below(2) ? 0 : 1 + below(5000);
    a.max_kv = below(2) ? 0 : below(c.max_blocks * c.page_size);
    const int room = c.max_blocks * c.page_size, prefix = 1 + below(room);
    const size_t need = gdn_cache_attn_shared_workspace_size(&t, &c, &a, prefix);
    const size_t row = (size_t)t.B * t.T * t.Hq * (t.d + 2) * 4;
    expect(need == 0 || (need >= 2 * row && need <= 512 * row + 512), "sums of a row");
    expect(gdn_cache_attn_shared_workspace_size(&t, &c, &a, room + 1) == 0, "past the cache");
    gdn_rows r;
    memset(&r, 0, sizeof r);
    r.data = x;
    r.token_stride = (int64_t)t.Hq * t.d;
    r.head_stride = t.d;
    if (need)
      expect(gdn_cache_attn_shared(&t, &a, &r, &c, x, prefix, &r, NULL, x, need - 1, NULL) ==
                 GDN_ERR_WORKSPACE, "a short workspace");
    expect(gdn_cache_attn_shared(&t, &a, &r, &c, NULL, prefix, &r, NULL, x, need, NULL) != GDN_OK,
           "no pages");
  }

  gdn_sampling s;
  memset(&s, 0, sizeof s);
  expect(gdn_sample(NULL, x, x, NULL) == GDN_ERR_NULL, "no sampling");
  expect(gdn_sample(&s, x, x, NULL) != GDN_OK, "no rows");
  s.rows = s.vocab = 5;
  s.dtype = GDN_BF16;
  expect(gdn_sample(&s, x, x, NULL) == GDN_ERR_NULL, "no logits");
  s.logits = x;
  expect(gdn_sample(&s, x, x, NULL) == GDN_ERR_NULL, "no random numbers");
  s.row_stride = INT64_MIN;
  expect(gdn_sample(&s, x, x, NULL) == GDN_ERR_SHAPE, "a far row");
  printf("answers driver: ok\n");
  return 0;
}
