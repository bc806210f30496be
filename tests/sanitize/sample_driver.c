/* The host side of the choice of tokens without a GPU: its refusals (but that of an unknown type,
 * whose value the enumeration does not hold: tests/test_sample_abi.py), over the range of what a
 * description can hold. */
#include <limits.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../../include/gdn_sample.h"

static uint64_t state = 4321;
static int below(int n) {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return (int)((state >> 33) % (uint64_t)n);
}
static void expect(int got, int want, const char *what) {
  if (got == want) return;
  printf("sample driver: %s gives %d, not %d\n", what, got, want);
  exit(1);
}

int main(void) {
  char *const x = (char *)0x10000;
  const int32_t odd_rows[] = {0, -1, INT32_MIN, 1 << 22, INT32_MAX};
  const int32_t odd_vocab[] = {0, -7, INT32_MIN, (1 << 20) + 1, INT32_MAX};
  const int64_t far[] = {INT64_MIN, INT64_MAX, ((int64_t)1 << 40) + 1, -((int64_t)1 << 40) - 1};
  for (int i = 0; i < 20000; ++i) {
    gdn_sampling s;
    memset(&s, 0, sizeof s);
    s.rows = 1 + below(i % 2 ? 300 : (1 << 22) - 1);
    s.vocab = 1 + below(i % 3 ? 200000 : 1 << 20);
    s.dtype = below(2) ? GDN_BF16 : GDN_F32;
    s.logits = x + 16 * below(8);
    s.row_stride = (int64_t)(below(3) - 1) * (((int64_t)1 << below(41)));
    s.temperature = below(2) ? (float *)x : NULL;
    s.top_k = below(2) ? (int32_t *)x : NULL;
    s.top_p = below(2) ? (float *)x : NULL;
    s.min_p = below(2) ? (float *)x : NULL;
    s.u = s.temperature && below(2) ? NULL : (float *)x;
    int32_t *tokens = (int32_t *)x;
    float *logprob = below(2) ? (float *)x : NULL;
    int want = GDN_OK;
    switch (below(12)) {
      case 0: s.logits = x + (s.dtype == GDN_F32 ? 2 : 1); want = GDN_ERR_ALIGN; break;
      case 1: s.rows = odd_rows[below(5)]; want = GDN_ERR_SHAPE; break;
      case 2: s.vocab = odd_vocab[below(5)]; want = GDN_ERR_SHAPE; break;
      case 3: s.row_stride = far[below(4)]; want = GDN_ERR_SHAPE; break;
      case 4: s.logits = NULL; want = GDN_ERR_NULL; break;
      case 5: tokens = NULL; want = GDN_ERR_NULL; break;
      case 6: s.u = s.temperature = NULL; want = GDN_ERR_NULL; break;
      case 7: s.logits = x + 1; want = GDN_ERR_ALIGN; break;
      case 8: s.u = (float *)(x + 2); want = GDN_ERR_ALIGN; break;
      case 9: s.top_k = (int32_t *)(x + 1 + below(3)); want = GDN_ERR_ALIGN; break;
      case 10: tokens = (int32_t *)(x + 2); want = GDN_ERR_ALIGN; break;
      default: logprob = (float *)(x + 3); want = GDN_ERR_ALIGN; break;
    }
    expect(gdn_sample(&s, tokens, logprob, NULL), want, "a call");
  }
  expect(gdn_sample(NULL, (int32_t *)x, NULL, NULL), GDN_ERR_NULL, "no description");
  printf("sample driver: ok\n");
  return 0;
}
