/* Drives the host side of the calls of requests (pages, prompts, sampling rules) through its error paths and its planning, under
 * AddressSanitizer and UndefinedBehaviorSanitizer.  No call reaches a launch. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include "hb.h"

#define WANT(call, rc)                                                                        \
  do {                                                                                        \
    int32_t got = (call);                                                                     \
    if (got != (rc)) {                                                                        \
      printf("%s:%d: got %d, want %d: %s\n", __FILE__, __LINE__, got, (rc), hb_last_error()); \
      return 1;                                                                               \
    }                                                                                         \
  } while (0)

static hb_attn_desc desc(void) {
  hb_attn_desc d;
  memset(&d, 0, sizeof d);
  d.dtype = HB_BF16;
  d.batch = 2;
  d.num_q_heads = 28;
  d.num_kv_heads = 4;
  d.head_dim = 128;
  d.page_size = 16;
  d.max_blocks_per_seq = 64;
  d.num_blocks = 200;
  d.total_nodes = 120;
  d.max_nodes_per_tree = 1;
  d.softmax_scale = 0.1f;
  return d;
}

int main(void) {
  /* addresses that nothing reads */
  char *at = (char *)0x1000;
  void *p = at, *far = (void *)((uintptr_t)1 << 46);
  int32_t *i = p, *j = far;
  float *f = p;
  hb_attn_desc d;
  /* plans over the whole range of what a descriptor may say */
  static const int32_t some[] = {0, 1, 2, 7, 64, 1000, 65535, 1 << 20, 1 << 25, INT32_MAX};
  const unsigned n = sizeof some / sizeof *some;
  for (unsigned a = 0; a < n; ++a)
    for (unsigned b = 0; b < n; ++b)
      for (unsigned c = 0; c < n; ++c)
        for (int s = 0; s < 4; ++s) {
          d = desc();
          d.batch = some[a];
          d.max_blocks_per_seq = some[b];
          d.total_nodes = some[c];
          d.num_splits = s == 2 ? some[b] : s & 1;
          d.max_prefix_len_hint = some[c];
          if (s == 3) d.dtype = HB_F32;
          const size_t bytes = hb_prompt_attn_workspace_bytes(&d);
          if (d.num_splits == 1 && bytes) {
            printf("%zu bytes for one part\n", bytes);
            return 1;
          }
          if (hb_rules_probs_workspace_bytes(some[a], some[b]) && (!some[a] || !some[b])) return 1;
        }
  /* sizes at the ends of their types */
  WANT(hb_pages_take(INT32_MAX, 1, 1, 1, 0, 0, i, i, i, i, i, j, NULL, NULL, j, NULL, j, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_pages_take(1, INT32_MAX, INT32_MAX, INT32_MAX, 0, 0, i, i, i, i, i, j, NULL, NULL, j, NULL, j, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_pages_take(1, 1, 1, INT32_MAX, INT32_MAX, INT32_MAX, i, i, i, i, i, j, NULL, NULL, j, NULL, j, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_pages_take(1, 1, 1, 1, -1, 0, i, i, i, i, i, j, NULL, NULL, j, NULL, j, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_pages_give(8192, 1, 1 << 30, INT32_MAX, i, i, i, j, i, j, j, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_pages_give(0, 1, 1, 1, NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL), HB_OK);
  d = desc();
  WANT(hb_kv_append(NULL, 1, p, p, i, p, p, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv_append(&d, INT32_MIN, p, p, i, p, p, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv_append(&d, INT32_MAX, p, p, i, p, NULL, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv_append(&d, 1, p, p, i, p, at + 8, NULL), HB_ERR_INVALID_ARG);
  d.page_size = d.num_blocks = 1 << 16;
  WANT(hb_kv_append(&d, 1, p, p, i, p, p, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_prompt_attn(NULL, p, p, p, p, p, i, i, i, far, NULL, p, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  d = desc();
  WANT(hb_prompt_attn(&d, p, p, p, NULL, p, i, i, i, far, NULL, p, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_prompt_attn(&d, p, p, p, p, p, i, i, i, p, NULL, p, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_prompt_attn(&d, p, p, p, p, p, i, i, i, far, (float *)far, p, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  d.num_splits = 4;
  WANT(hb_prompt_attn(&d, p, p, p, p, p, i, i, i, far, NULL, NULL, SIZE_MAX, NULL), HB_ERR_WORKSPACE);
  WANT(hb_prompt_attn(&d, p, p, p, p, p, i, i, i, far, NULL, far, hb_prompt_attn_workspace_bytes(&d) - 1, NULL), HB_ERR_WORKSPACE);
  WANT(hb_prompt_attn(&d, p, p, p, p, p, i, i, i, far, NULL, far, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  d.total_nodes = INT32_MAX;
  WANT(hb_prompt_attn(&d, p, p, p, p, p, i, i, i, far, NULL, p, SIZE_MAX, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_rules_count(INT32_MAX, INT32_MAX, INT32_MAX, NULL, i, 2, j, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_rules_count(2, INT32_MAX, INT32_MAX, NULL, i, 0, j, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_rules_logits(HB_BF16, 1, 64, INT32_MAX, 1 << 30, p, i, i, i, i, f, i, 1, i, f, 1, (uint32_t *)p, i, at + 16, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_rules_logits(HB_BF16, 1, 64, 1, INT32_MAX, p, i, i, i, i, f, i, 1, i, f, 1, (uint32_t *)p, i, p, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_rules_probs(HB_F32, 1, 64, 1000, 100000, p, i, i, i, i, f, i, 1, i, f, 1, (uint32_t *)p, i, f, far, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_rules_probs(HB_F32, 1, 64, 1000, 100000, p, i, i, i, i, f, i, 1, i, f, 1, (uint32_t *)p, i, far, NULL, 0, NULL), HB_ERR_WORKSPACE);
  printf("host shim checks passed\n");
  return 0;
}
