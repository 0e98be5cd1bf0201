/* The host side of grpo_top.h and grpo_linear.h under the sanitizers: refusals and size queries at the ends of their
 * ranges.  Device pointers are numbers that nothing reads. */
#include <stdio.h>
#include <string.h>

#include "grpo_linear.h"
#include "grpo_top.h"

#define CHECK(x)                             \
  do {                                       \
    if (!(x)) {                              \
      printf("line %d: %s\n", __LINE__, #x); \
      return 1;                              \
    }                                        \
  } while (0)

static void* at(unsigned long a) { return (void*)a; }

int main(void) {
  const int64_t big = INT64_MAX;
  void* D = at(0x100000);
  CHECK(grpo_token_logp_top_workspace_bytes(big, big, 5) == 0 && grpo_token_logp_top_workspace_bytes(1, 5, INT32_MIN) == 0);
  for (int64_t T = 0; T < 3000; T += 7)
    for (int n = 0; n <= GRPO_TOP_MAX; ++n)
      CHECK(grpo_token_logp_top_workspace_bytes(T, GRPO_TOP_MAX_V, n) < (size_t)1 << 20);
  CHECK(grpo_token_logp_top(D, GRPO_BF16, big, 1, 1, NULL, 1.f, D, 1, D, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_SHAPE);
  CHECK(grpo_token_logp_top(D, GRPO_BF16, 1, big, big, NULL, 1.f, D, 1, D, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_SHAPE);
  CHECK(grpo_token_logp_top(D, 1 << 30, 1, 5, 5, NULL, 1.f, D, 1, D, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_DTYPE);
  CHECK(grpo_token_logp_top(D, GRPO_F32, 1, 50000, 50000, NULL, 1.f, D, 1, D, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_WORKSPACE);
  CHECK(grpo_token_logp_top_bwd(D, GRPO_F32, 1, 5, INT64_MIN, D, 1, D, D, D, D, D, D, NULL) == GRPO_ERR_SHAPE);
  CHECK(grpo_token_logp_top_bwd(D, GRPO_F32, 4, 5, 5, D, 1, D, D, D, D, D, at(0x100004), NULL) == GRPO_ERR_ARG);

  const int64_t most = 8388352, sizes[] = {1, 7, 8, 9, 31, 33, 64, 65, 257, 3584, 151936, most};
  const int n_sizes = (int)(sizeof sizes / sizeof *sizes);
  grpo_linear_op op;
  grpo_linear_grads g;
  memset(&op, 0, sizeof op);
  memset(&g, 0, sizeof g);
  CHECK(grpo_linear_workspace_bytes(NULL) == 0 && grpo_linear_workspace_bytes(&op) == 0);
  op.x = at(0x1000002);
  op.w = at(0x2000002);
  g.dx = at(0x3000000);
  g.dw = at(0x4000000);
  g.dbias = at(0x5000000);
  for (int i = 0; i < n_sizes; ++i)
    for (int j = 0; j < n_sizes; ++j)
      for (int k = 0; k < n_sizes; ++k)
        for (int form = 0; form < 8; ++form) {
          op.M = sizes[i];
          op.K = sizes[j];
          op.N = sizes[k];
          op.w_out_in = form & 1;
          op.act = form & 2 ? GRPO_ACT_SILU : GRPO_ACT_NONE;
          op.ldx = form & 4 ? big : op.K;
          op.ldw = form & 4 ? big : op.w_out_in ? op.K : op.N;
          const size_t f = grpo_linear_workspace_bytes(&op);
          const size_t b = grpo_linear_bwd_workspace_bytes(&op, at(0x6000000), form & 4 ? big : op.N, GRPO_F32, &g);
          CHECK(f % 256 == 0 && b % 256 == 0 && b > 0);
          if (f > 0)
            CHECK(grpo_linear(&op, NULL, 0, at(0x7000000), op.N, GRPO_F32, NULL, NULL, 0, NULL) == GRPO_ERR_WORKSPACE);
          CHECK(grpo_linear_bwd(&op, at(0x6000000), op.N, GRPO_F32, at(0x8000000), &g, NULL, 0, NULL) == GRPO_ERR_WORKSPACE);
        }
  op.M = op.K = op.N = 64;
  op.ldx = op.ldw = 64;
  op.M = big;
  CHECK(grpo_linear_workspace_bytes(&op) == 0);
  op.M = 64;
  op.act = INT32_MAX;
  CHECK(grpo_linear(&op, NULL, 0, D, 64, GRPO_F32, NULL, NULL, 0, NULL) == GRPO_ERR_ARG);
  op.act = 0;
  CHECK(grpo_linear(&op, NULL, 0, D, INT64_MIN, GRPO_F32, NULL, NULL, 0, NULL) == GRPO_ERR_SHAPE);
  g.accumulate_dw = 7;
  CHECK(grpo_linear_bwd(&op, D, 64, GRPO_F32, NULL, &g, D, (size_t)1 << 40, NULL) == GRPO_ERR_ARG);
  CHECK(grpo_linear_bwd(&op, D, 64, GRPO_F32, NULL, NULL, D, (size_t)1 << 40, NULL) == GRPO_ERR_ARG);
  printf("argument checks ok\n");
  return 0;
}
