/* The calls that fill gradient tensors take no memory from the heap: counts malloc (operator new goes there too) while they check
 * their arguments, up to a refusal that they make after all lists have been built.  No GPU call is made. */
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

enum { WORLD = CARAMEL_MAX_WORLD };

int main(void) {
  const uint64_t elems[1] = {64};
  caramel_config cfg;
  caramel_plan* plan = NULL;
  const void* in[WORLD];
  const void* ids[WORLD];
  void* out[WORLD];
  uint64_t tokens[WORLD];
  int w, pass;
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
    in[w] = (const void*)(((uintptr_t)w + 1) << 20);
    ids[w] = (const void*)(((uintptr_t)w + 100) << 20);
    out[w] = (void*)(((uintptr_t)w + 200) << 20);
    tokens[w] = 5;
  }
  out[WORLD - 1] = out[0]; /* two outputs in one place: refused, and last of all checks */
  for (pass = 0; pass < 2; ++pass) { /* the first one makes room for the message */
    calls = 0;
    if (caramel_embedding_lookup(plan, in, 8, 16, 1.0f, ids, 8, tokens, out, 16, NULL) != CARAMEL_EINVAL) return 2;
    if (caramel_checkpoint_store(plan, tokens, 16, in, CARAMEL_F32, 16, out, NULL) != CARAMEL_EINVAL) return 3;
    if (caramel_checkpoint_load(plan, tokens, 16, in, out, CARAMEL_F32, 16, NULL) != CARAMEL_EINVAL) return 4;
  }
  if (calls) {
    printf("%lu allocations: %s\n", calls, caramel_last_error());
    return 5;
  }
  caramel_plan_destroy(plan);
  printf("alloc_check ok\n");
  return 0;
}
