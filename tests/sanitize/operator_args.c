/* The host side of grpo_sampling.h and grpo_clip.h under the sanitizers: refusals, size queries at the ends of their
 * ranges, and clipping tables of valid, empty and overlapping tensors.  Device pointers are numbers that nothing reads. */
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "grpo_clip.h"
#include "grpo_sampling.h"

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      printf("line %d: %s\n", __LINE__, #x);                  \
      return 1;                                               \
    }                                                         \
  } while (0)

static void* at(unsigned long a) { return (void*)a; }

int main(void) {
  const int64_t big = INT64_MAX;
  grpo_sampling p;
  memset(&p, 0, sizeof p);
  p.temperature_all = 1.f;
  p.top_p_all = 1.f;
  void* D = at(0x100000);
  CHECK(grpo_sampling_workspace_bytes(big, big) == 0 && grpo_sampling_workspace_bytes(-1, 1) == 0);
  CHECK(grpo_sampling_workspace_bytes(191, GRPO_SAMPLING_MAX_V) > 0);
  CHECK(grpo_sample(D, GRPO_BF16, big, 1, 1, &p, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_SHAPE);
  CHECK(grpo_sample(D, GRPO_BF16, 1, big, big, &p, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_SHAPE);
  CHECK(grpo_sample(D, GRPO_BF16, 1, 50000, 50000, &p, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_WORKSPACE);
  CHECK(grpo_sample(D, 1 << 30, 1, 5, 5, &p, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_DTYPE);
  CHECK(grpo_sampled_logp(D, GRPO_F32, 1, 5, 5, NULL, D, D, D, D, D, D, 0, NULL) == GRPO_ERR_ARG);
  CHECK(grpo_sampled_logp_bwd(D, GRPO_F32, 1, 5, INT64_MIN, D, D, D, D, NULL) == GRPO_ERR_SHAPE);
  CHECK(grpo_sampled_logp_bwd(D, GRPO_F32, 4, 5, 5, D, D, D, at(0x100004), NULL) == GRPO_ERR_ARG);

  CHECK(grpo_grad_table_bytes(INT32_MIN) == 0 && grpo_grad_table_bytes(INT32_MAX) == 0);
  enum { N = 1000 };
  grpo_grad* g = malloc(N * sizeof *g);
  void* table = malloc(grpo_grad_table_bytes(N));
  grpo_grad_layout l;
  for (int i = 0; i < N; ++i) {
    g[i] = (grpo_grad){at(0x1000000ul + 0x10000ul * i), at(0x1000000ul + 0x10000ul * i), i % 7 ? 100 * i % 16384 : 0,
                       GRPO_F32, GRPO_F32};
  }
  CHECK(grpo_grad_table(g, N, table, grpo_grad_table_bytes(N), &l) == GRPO_OK && l.n == N && l.in_place == 1);
  CHECK(grpo_grad_table(g, N, table, grpo_grad_table_bytes(N) - 1, &l) == GRPO_ERR_WORKSPACE);
  g[N - 1] = g[1];
  CHECK(grpo_grad_table(g, N, table, grpo_grad_table_bytes(N), &l) == GRPO_ERR_SHAPE);
  g[N - 1].n = INT64_MAX;
  CHECK(grpo_grad_table(g, N, table, grpo_grad_table_bytes(N), &l) == GRPO_ERR_SHAPE);
  g[N - 1].dtype = INT32_MIN;
  CHECK(grpo_grad_table(g, N, table, grpo_grad_table_bytes(N), &l) == GRPO_ERR_DTYPE);
  CHECK(grpo_grad_table(NULL, 0, table, grpo_grad_table_bytes(0), &l) == GRPO_OK && l.units == 0);
  CHECK(grpo_grad_sumsq(&l, table, NULL, NULL) == GRPO_ERR_ARG);
  CHECK(grpo_grad_clip(&l, table, table, -1.0, NULL, NULL, NULL) == GRPO_ERR_ARG);
  free(table);
  free(g);
  printf("operator argument checks ok\n");
  return 0;
}
