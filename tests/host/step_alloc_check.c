/* The calls of a training step around the gradients take no memory from the heap: counts malloc (operator new goes there too) while they
 * check their arguments, up to a refusal that they make after all lists have been built.  No GPU call is made. */
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "caramel.h"

extern void* __libc_malloc(size_t);
static unsigned long calls;
void* malloc(size_t n) {
  ++calls;
  return __libc_malloc(n);
}

enum { WORLD = CARAMEL_MAX_WORLD, LISTS = 13 };

static void* at[LISTS][WORLD]; /* pointers of every worker, 1 MiB apart */
#define IN(k) ((const void* const*)at[k])
#define F32(k) ((float* const*)at[k])
#define F32_IN(k) ((const float* const*)at[k])

int main(void) {
  const uint64_t elems[1] = {16};
  caramel_config cfg;
  caramel_plan* plan = NULL;
  uint64_t tokens[WORLD], sequences[WORLD];
  void* ws = (void*)((uintptr_t)1 << 40);
  const uint64_t ws_bytes = (uint64_t)1 << 30;
  int w, k, pass;
  memset(&cfg, 0, sizeof cfg);
  cfg.world = WORLD;
  cfg.dtype = CARAMEL_F32;
  cfg.batch_threshold_bytes = 65536;
  cfg.split_mode = CARAMEL_SPLIT_NONE;
  cfg.max_depth = 8;
  cfg.align_bytes = 16;
  cfg.num_streams = 2;
  cfg.pattern = CARAMEL_PATTERN_RING;
  if (caramel_plan_create(&cfg, elems, 1, &plan) != CARAMEL_OK) return 1;
  for (w = 0; w < WORLD; ++w) {
    for (k = 0; k < LISTS; ++k) at[k][w] = (void*)(((uintptr_t)k * WORLD + w + 1) << 20);
    tokens[w] = 500;
    sequences[w] = 3;
  }
  at[12][WORLD - 1] = at[12][0]; /* two outputs in one place: refused, and last of all checks */
  for (pass = 0; pass < 2; ++pass) { /* the first one makes room for the message */
    calls = 0;
    if (caramel_residual_norm(plan, IN(0), 16, 1e-5f, tokens, IN(1), IN(2), CARAMEL_F32, 16, at[3], at[4], F32(12), at[5], NULL) != CARAMEL_EINVAL)
      return 2;
    if (caramel_recurrence(plan, 16, tokens, sequences, IN(0), 8, IN(1), IN(2), CARAMEL_F32, 16, F32_IN(3), at[4], 16, F32(12), ws, ws_bytes,
                           NULL) != CARAMEL_EINVAL)
      return 3;
    if (caramel_recurrence_gradient(plan, 16, tokens, sequences, IN(0), 8, IN(1), IN(2), CARAMEL_F32, 16, F32_IN(3), IN(4), IN(5), 16, F32_IN(6),
                                    at[7], at[8], F32(12), ws, ws_bytes, NULL) != CARAMEL_EINVAL)
      return 4;
    if (caramel_distillation(plan, 16, tokens, IN(0), CARAMEL_F32, 16, IN(1), IN(2), 8, IN(3), CARAMEL_F32, 4, 2.0f, 1.0f, 0.5f, 1.0f, F32(4),
                             at[12], 16, ws, ws_bytes, NULL) != CARAMEL_EINVAL)
      return 5;
    if (strstr(caramel_last_error(), "overlap") == NULL) return 6;
    /* (its outputs are checked against a bound plan's; this one is not) */
    if (caramel_residual_norm_gradient(plan, 0, IN(0), tokens, IN(1), F32_IN(2), IN(3), IN(4), CARAMEL_F32, 16, at[12], 0, ws, ws_bytes, NULL) !=
        CARAMEL_ESTATE)
      return 7;
  }
  if (calls) {
    printf("%lu allocations: %s\n", calls, caramel_last_error());
    return 8;
  }
  caramel_plan_destroy(plan);
  printf("step_alloc_check ok\n");
  return 0;
}
