/* The host side of the attention layer's entry points (gdn_paged_api.hip) without a GPU:
 * workspace sizes of many problems up to the limits (so the plan of an attention call, whose
 * rule counts blocks, keys and splits), refusals, and the table of a rotation.  No call
 * reaches a HIP call. */
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../../include/gdn_paged.h"

#define FAIL(...) (fprintf(stderr, __VA_ARGS__), exit(1))

static unsigned long long state = 88172645463325252ull;
static unsigned next(unsigned n) {
  state ^= state << 13;
  state ^= state >> 7;
  state ^= state << 17;
  return (unsigned)((state >> 20) % n);
}
/* of any size up to most, small ones as often as large ones */
static int32_t any(int bits) { return (int32_t)((1u << next((unsigned)bits)) + next(1u << next((unsigned)bits))); }

static void plans(void) {
  const int32_t dims[] = {64, 128, 256};
  long sized = 0, none = 0, refused = 0;
  for (int i = 0; i < 20000; ++i) {
    const int n = 1 + (int)next(70);
    int32_t* cu = malloc(sizeof(int32_t) * (size_t)(n + 1));
    gdn_tokens t;
    memset(&t, 0, sizeof t);
    t.Hk = any(5);
    t.Hq = t.Hk * any(5);
    t.d = dims[next(3)];
    t.dtype = next(2) ? GDN_F32 : GDN_BF16;
    if (next(2)) {
      cu[0] = 0;
      for (int j = 0; j < n; ++j) cu[j + 1] = cu[j] + (next(3) ? any(12) - 1 : 0);
      t.B = 1;
      t.T = cu[n];
      t.num_seqs = n;
      t.cu_seqlens = (const int32_t*)256;
      t.cu_seqlens_host = cu;
    } else {
      t.B = any(10);
      t.T = any(14);
    }
    gdn_cache c;
    memset(&c, 0, sizeof c);
    c.num_pages = any(20);
    c.page_size = 16 << next(7);
    c.max_blocks = any(27);
    gdn_attn a;
    a.scale = 0.1f;
    a.causal = next(4) != 0;
    a.window = a.causal && next(2) ? (next(8) ? any(17) : INT32_MAX) : 0;
    a.max_kv = next(3) ? any(24) : next(2) ? INT32_MAX : 0;
    const size_t need = gdn_cache_attn_workspace_size(&t, &c, &a);
    if (need % 256) FAIL("workspace of %zu bytes\n", need);
    need ? ++sized : ++none;
    /* without tensors nothing runs */
    if (gdn_cache_attn(&t, &a, NULL, &c, NULL, NULL, NULL, 0, NULL) == GDN_OK)
      FAIL("a call without tensors was taken\n");
    ++refused;
    free(cu);
  }
  if (!sized || !none || !refused) FAIL("the problems do not cover the plans\n");
}

static void pages(void) {
  gdn_book b;
  memset(&b, 0, sizeof b);
  for (int i = 0; i < 2000; ++i) {
    b.S = any(21);
    b.max_blocks = any(27);
    b.num_pages = any(21);
    b.page_size = any(11);
    const size_t need = gdn_pages_workspace_size(&b);
    const int ok = b.S <= 1 << 20 && b.num_pages <= 1 << 20;
    if ((need != 0) != ok || need % 256) FAIL("workspace of %zu bytes\n", need);
    if (gdn_pages_extend(&b, NULL, NULL, NULL, 0, NULL) == GDN_OK ||
        gdn_pages_select(&b, NULL, NULL, NULL, NULL, 0, NULL) == GDN_OK ||
        gdn_pages_compact(&b, NULL, NULL, NULL, 0, NULL) == GDN_OK)
      FAIL("a call without arrays was taken\n");
  }
  if (gdn_pages_copy(NULL, NULL, NULL, 0, NULL) == GDN_OK) FAIL("no pool\n");
}

static void turns(void) {
  for (int32_t rot = -2; rot <= 256; ++rot)
    for (int32_t kind = -1; kind <= 4; ++kind) {
      const size_t n = rot > 1 ? (size_t)rot / 2 : 1;
      double* f = malloc(sizeof(double) * n);
      float s = 0;
      const gdn_status st = gdn_rotary_turns(rot, 10000., kind, 4., 4096., 1., 32., f, &s);
      const int good = rot >= 2 && rot % 2 == 0 && kind >= 0 && kind <= 3;
      if ((st == GDN_OK) != good) FAIL("rot %d, kind %d: status %d\n", rot, kind, (int)st);
      for (size_t i = 0; good && i < n; ++i)
        if (!(f[i] > 0) || !(f[i] < 0.2) || (i && f[i] > f[i - 1])) FAIL("turn %g\n", f[i]);
      free(f);
    }
}

int main(void) {
  plans();
  pages();
  turns();
  puts("paged driver: ok");
  return 0;
}
