/* The entry points of the paged cache, of the attention over it and of the log-probabilities for the sanitizer build (tests/test_host_sanitizers_generation.py): calls that
 * the argument validation must turn down, and the queries of sizes.  Nothing here reaches a kernel launch. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../include/dlayer.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
  do {                                                                      \
    if (!(cond)) { printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } \
  } while (0)
#define EXPECT_INVALID(call)                                                \
  do {                                                                      \
    int rc_ = (call);                                                       \
    if (rc_ != DLAYER_ERR_INVALID || strlen(dlayer_last_error()) == 0) {    \
      printf("FAILED line %d: %s returned %d (%s)\n", __LINE__, #call, rc_, dlayer_last_error()); \
      ++failures;                                                           \
    }                                                                       \
  } while (0)

int main(void) {
  static char arena[1 << 16] __attribute__((aligned(256)));
  void *a = arena, *b = arena + (1 << 14), *odd = arena + 2;   /* never dereferenced */
  float* f = (float*)b;
  const int64_t big = INT64_MAX;
  const dlayer_kv_cache good = {arena + 0x8000, arena + 0x9000, arena + 0xa000, arena + 0xb000, (int32_t*)(arena + 0xc000), 1, 1, 16, 32, 1, 1, DLAYER_CACHE_E4M3};
  dlayer_kv_cache c = good;
  int i, s;

  EXPECT_INVALID(kv_cache_append(NULL, a, a, a, NULL, NULL, 1, 1, 1e4f, 0, b, NULL));
  EXPECT_INVALID(kv_cache_append(&good, a, a, a, NULL, NULL, 0, 1, 1e4f, 0, b, NULL));
  EXPECT_INVALID(kv_cache_append(&good, a, a, a, NULL, NULL, big, 1, 1e4f, 0, b, NULL));
  EXPECT_INVALID(kv_cache_append(&good, a, a, a, NULL, NULL, 1, big, 1e4f, 0, b, NULL));
  EXPECT_INVALID(kv_cache_append(&good, a, odd, a, NULL, NULL, 1, 1, 1e4f, 0, b, NULL));
  EXPECT_INVALID(kv_cache_append(&good, a, a, a, NULL, NULL, 1, 1, NAN, 0, b, NULL));
  EXPECT_INVALID(kv_cache_append(&good, NULL, a, a, NULL, NULL, 1, 1, 1e4f, -1, NULL, NULL));
  EXPECT_INVALID(kv_cache_read(&good, NULL, NULL, -1, a, b, NULL));
  EXPECT_INVALID(kv_cache_read(&good, NULL, NULL, 1, a, a, NULL));
  EXPECT_INVALID(kv_cache_read(&good, NULL, NULL, 1, good.k, b, NULL));
  EXPECT_INVALID(paged_attention_forward(&good, a, NULL, NULL, 1, 0, 1.f, b, NULL, a, NULL));
  EXPECT_INVALID(paged_attention_forward(&good, a, NULL, NULL, big, 1, 1.f, b, NULL, a, NULL));
  EXPECT_INVALID(paged_attention_forward(&good, a, NULL, NULL, 1, big, 1.f, b, NULL, a, NULL));
  EXPECT_INVALID(paged_attention_forward(&good, a, NULL, NULL, 1, 1, INFINITY, b, NULL, a, NULL));
  EXPECT_INVALID(paged_attention_forward(&good, a, NULL, NULL, 1, 1, 1.f, a, NULL, b, NULL));
  for (i = 0; i < 7; ++i) {                                        /* every size of the handle at the ends of its type */
    int32_t* size[7] = {&c.n_pages, &c.n_kv_heads, &c.page_size, &c.head_dim, &c.batch, &c.max_pages, &c.dtype};
    const int32_t ends[3] = {INT32_MIN, -1, INT32_MAX};
    for (s = 0; s < 3; ++s) {
      c = good;
      *size[i] = ends[s];
      (void)paged_attention_workspace_bytes(&c, 1, 1);
      if (s < 2 || (i != 0 && i != 4)) EXPECT(paged_attention_workspace_bytes(&c, 1, 1) == 0);
      if (s < 2) EXPECT_INVALID(kv_cache_read(&c, NULL, NULL, 1, a, b, NULL));
    }
  }
  c = good;
  c.batch = INT32_MAX;
  EXPECT(paged_attention_workspace_bytes(&c, INT32_MAX, 65535) == 0);
  EXPECT(paged_attention_workspace_bytes(&good, 1, 4) > 0 && paged_attention_workspace_bytes(&good, 1 << 20, 8) > 0 && paged_attention_workspace_bytes(NULL, 1, 1) == 0);

  EXPECT_INVALID(token_logprobs_forward(a, (int64_t*)a, 0, 8, 8, 1.f, 0, f, f, f, NULL, NULL, b, NULL));
  EXPECT_INVALID(token_logprobs_forward(a, (int64_t*)a, big, big, big, 1.f, 0, f, f, f, NULL, NULL, b, NULL));
  EXPECT_INVALID(token_logprobs_forward(a, (int64_t*)a, 1, 9, 8, 1.f, 0, f, f, f, NULL, NULL, b, NULL));
  EXPECT_INVALID(token_logprobs_forward(a, (int64_t*)a, 1, 8, 8, 1.f, big, f, f, f, NULL, NULL, b, NULL));
  EXPECT_INVALID(token_logprobs_forward(a, NULL, 1, 8, 8, 1.f, 0, f, f, f, NULL, NULL, b, NULL));
  EXPECT_INVALID(token_logprobs_backward(a, (int64_t*)a, f, f, f, f, big, 8, 8, 1.f, b, NULL));
  EXPECT_INVALID(token_logprobs_backward(a, (int64_t*)a, f, f, NULL, NULL, 1, 8, 8, 1.f, b, NULL));
  EXPECT_INVALID(token_logprobs_backward(a, (int64_t*)a, f, f, f, f, 1, 8, 8, -1.f, b, NULL));
  EXPECT_INVALID(token_logprobs_backward(a, (int64_t*)a, f, f, f, f, 2, 8, 8, 1.f, (char*)a + 16, NULL));
  EXPECT(token_logprobs_workspace_bytes(big, 8, 0) == 0 && token_logprobs_workspace_bytes(1, big, 0) == 0 && token_logprobs_workspace_bytes(1, 8, big) == 0);
  EXPECT(token_logprobs_workspace_bytes(1, 128256, 64) > 0);

  if (failures) return 1;
  printf("all calls rejected as expected\n");
  return 0;
}
