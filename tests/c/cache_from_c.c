/* A plain C99 caller of the cache's entry points that need no device. */
#include <stdio.h>
#include <string.h>

#include "ssba_cache.h"

#define CHECK(x) do { if (!(x)) { printf("failed: %s\n", #x); return 1; } } while (0)

int main(void) {
  ssba_cache c;
  ssba_cache_batch b;
  ssba_cache_query q;
  ssba_pages p;
  size_t n = 0;
  memset(&c, 0, sizeof c);
  memset(&b, 0, sizeof b);
  memset(&q, 0, sizeof q);
  memset(&p, 0, sizeof p);
  c.layers = 1;
  c.pages = 8;
  c.kv_heads = 2;
  c.head_dim = 64;
  c.page = 16;
  b.seqs = 2;
  b.max_pages = 4000;
  b.rows = 2;
  b.max_new = 1;
  q.heads = 4;
  q.causal = 1;
  q.keep = 3;
  q.first = q.last = 1;
  p.rows = 2;
  p.max_pages = 4;
  CHECK(ssba_cache_select_workspace_size(&c, &b, &q, &n) == SSBA_OK && n > 0);
  CHECK(ssba_cache_attend_workspace_size(&c, &b, &q, 1, &n) == SSBA_OK);
  CHECK(ssba_pages_workspace_size(&c, &p, 2, &n) == SSBA_OK && n > 0);
  CHECK(ssba_cache_append(&c, 0, &b, SSBA_DT_BF16, NULL, NULL, 0, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_cache_select(&c, 0, &b, &q, NULL, NULL, 0, NULL, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_cache_attend(&c, 0, &b, &q, NULL, NULL, 0, NULL, NULL, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_pages_reserve(&c, &p, NULL, NULL, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_pages_fork(&c, &p, 1, NULL, NULL, NULL, NULL, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_pages_release(&c, &p, 1, NULL, NULL, NULL, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_pages_compact(&c, &p, NULL, NULL, NULL, NULL, 0, NULL) == SSBA_ERR_ARG);
  CHECK(ssba_pages_copy(&c, &c, 1, NULL, NULL, NULL) == SSBA_ERR_ARG);
  c.page = 17;
  CHECK(ssba_pages_workspace_size(&c, &p, 2, &n) == SSBA_ERR_UNSUPPORTED);
  puts("ok");
  return 0;
}
