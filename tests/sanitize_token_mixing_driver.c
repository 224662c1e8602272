/* The entry points of the norm of queries and keys and of linear attention for the sanitizer build (tests/test_host_sanitizers_token_mixing.py):
 * calls that the argument validation must turn down, and the queries of sizes and plans.  Nothing here reaches a kernel launch. */
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
  static char arena[4096] __attribute__((aligned(256)));
  void *a = arena, *b = arena + 1024, *odd = arena + 2;   /* never dereferenced */
  float* f = (float*)b;
  const int64_t big = INT64_MAX;
  int32_t plan[3];
  int dh, backward;

  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, 0, 1, 1, 1, 64, 1e-5f, 1e4f, 0, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, 1, 1, 1, 1, 96, 1e-5f, 1e4f, 0, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, big, big, big, big, 64, 1e-5f, 1e4f, 0, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, 1, 1, 1, 1, 64, -1.f, 1e4f, 0, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e-5f, 0.f, 0, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e-5f, 1e4f, 2, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, odd, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e-5f, 1e4f, 0, b, b, NULL, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_forward(a, a, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e-5f, 1e4f, 0, b, b, f, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_backward(a, a, a, a, NULL, f, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e4f, 0, b, b, b, b, 0, b, NULL));
  EXPECT_INVALID(qk_norm_rope_backward(a, a, a, a, f, f, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e4f, 0, b, b, b, b, 0, NULL, NULL));
  EXPECT_INVALID(qk_norm_rope_backward(a, a, a, a, f, f, a, a, NULL, NULL, 1, 1, 1, 1, 64, 1e4f, 7, b, b, b, b, 0, b, NULL));
  EXPECT(qk_norm_rope_backward_workspace_bytes(2, 8192, 32, 8, 128) > 0 && qk_norm_rope_backward_workspace_bytes(2, 8192, 32, 8, 80) == 0);
  EXPECT(qk_norm_rope_backward_workspace_bytes(big, big, 1, 1, 64) == 0);

  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, 1, 1, 3, 2, 64, 1.f, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, 1, -1, 2, 2, 64, 1.f, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, big, 1, 2, 2, 64, 1.f, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, 1, big, 2, 2, 64, 1.f, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, NULL, NULL, NULL, 1, 1, 2, 2, 64, 1.f, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, odd, 1, 1, 2, 2, 64, 1.f, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, 1, 1, 2, 2, 64, 1.f, b, NULL, NULL, NULL));
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, 1, 1, 2, 2, 64, 1.f, a, NULL, b, NULL));            /* o over q, k and v */
  EXPECT_INVALID(linear_attention_forward(a, a, a, f, NULL, NULL, 1 << 20, 1 << 29, 2, 2, 128, 1.f, b, NULL, a, NULL));   /* b is inside a's 2^58 bytes */
  EXPECT_INVALID(linear_attention_backward(a, a, a, f, NULL, NULL, NULL, NULL, 1, 1, 2, 2, 64, 1.f, b, b, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_backward(a, a, a, f, NULL, NULL, a, NULL, 1, 1, 2, 2, 64, 1.f, b, a, b, NULL, b, NULL));
  EXPECT_INVALID(linear_attention_backward(a, a, a, f, NULL, f, a, NULL, 1, 1, 2, 2, 64, 1.f, b, b, b, f, b, NULL));  /* d_state_in is state_in */
  EXPECT_INVALID(linear_attention_step(a, a, a, f, NULL, NULL, 1, 2, 2, 64, 1.f, b, NULL));
  EXPECT_INVALID(linear_attention_step(a, a, a, f, NULL, f, 1, 2, 2, 48, 1.f, b, NULL));
  EXPECT_INVALID(linear_attention_step(a, a, a, f, NULL, f, 1, 2, 2, 64, 1.f, a, NULL));
  EXPECT(linear_attention_workspace_bytes(1, 0, 2, 2, 64) == 0 && linear_attention_backward_workspace_bytes(1, 5, 3, 2, 64) == 0);
  EXPECT_INVALID(linear_attention_plan(1, 64, 2, 2, 64, 2, plan));
  EXPECT_INVALID(linear_attention_plan(1, 64, 2, 2, 64, 0, NULL));

  /* plans of the whole range of sizes: whole, without an empty segment or part, within the workspaces */
  for (dh = 32; dh <= 128; dh *= 2)
    for (backward = 0; backward < 2; ++backward)
      for (int64_t batch = 1; batch < (1 << 22); batch = batch * 5 + 1)
        for (int64_t seq = 1; seq < (1 << 30); seq = seq * 3 + 1)
          for (int64_t hkv = 1; hkv <= 64 && batch * hkv < (1 << 22); hkv = hkv * 3 + 1)
            for (int64_t group = 1; group <= 64 && group * hkv < 65536; group = group * 2 + 1) {
              const int64_t chunks = (seq + 63) / 64, pairs = batch * hkv;
              const size_t room = (backward ? linear_attention_backward_workspace_bytes : linear_attention_workspace_bytes)(batch, seq, group * hkv, hkv, dh);
              if (linear_attention_plan(batch, seq, group * hkv, hkv, dh, backward, plan) != DLAYER_OK) {
                printf("FAILED: no plan for %lld %lld %lld %lld\n", (long long)batch, (long long)seq, (long long)hkv, (long long)group);
                return 1;
              }
              const int64_t n = plan[1], per = (group + plan[2] - 1) / plan[2];
              if (!(n >= 1 && plan[0] >= 1 && (n - 1) * plan[0] < chunks && chunks <= n * plan[0] && plan[2] >= 1 && per * (plan[2] - 1) < group) ||
                  ((n > 1 || plan[2] > 1) && (size_t)(pairs * n * dh * dh * 4 * (backward ? 2 : 1)) > room) ||
                  pairs * n * (backward + plan[2]) * 512 >= ((int64_t)1 << 32)) {
                printf("FAILED: plan %d %d %d of %lld %lld %lld %lld %d\n", plan[0], plan[1], plan[2], (long long)batch, (long long)seq, (long long)hkv,
                       (long long)group, backward);
                return 1;
              }
            }
  printf(failures ? "sanitize driver: %d FAILED\n" : "sanitize driver: all calls rejected as expected (%d failures)\n", failures);
  return failures ? 1 : 0;
}
