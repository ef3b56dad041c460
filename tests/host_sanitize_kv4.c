/* Drives the host side of the 4-bit cache's calls through its error paths and its planning, under
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
  d.max_nodes_per_tree = 60;
  d.softmax_scale = 0.1f;
  return d;
}

int main(void) {
  void *p = (void *)0x1000;
  const int32_t *i = p;
  hb_attn_desc d = desc();
  /* plans over the whole range of what a descriptor may say */
  static const int32_t some[] = {0, 1, 2, 7, 64, 1000, 65535, 1 << 20, INT32_MAX};
  for (unsigned a = 0; a < sizeof some / sizeof *some; ++a)
    for (unsigned b = 0; b < sizeof some / sizeof *some; ++b)
      for (unsigned c = 0; c < sizeof some / sizeof *some; ++c)
        for (int s = 0; s < 3; ++s) {
          d = desc();
          d.batch = some[a];
          d.max_blocks_per_seq = some[b];
          d.total_nodes = some[c];
          d.num_splits = s == 2 ? some[b] : s;
          d.max_prefix_len_hint = some[c];
          size_t bytes = hb_tree_verify_attn_kv4_workspace_bytes(&d);
          int32_t splits = hb_tree_verify_attn_kv4_num_splits(&d);
          if ((splits <= 1) != (bytes == 0)) {
            printf("%zu bytes for %d slots\n", bytes, splits);
            return 1;
          }
          if (some[c] > 0) hb_kv4_evict_workspace_bytes(&d, some[c] > 1 << 30 ? 1 << 30 : some[c]);
        }
  d = desc();
  WANT(hb_kv4_append(NULL, 1, p, p, p, p, p, p, i, i, i, NULL, NULL, NULL, NULL, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv4_append(&d, INT32_MAX, p, p, p, p, p, p, i, i, i, NULL, NULL, NULL, NULL, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_kv4_append(&d, -1, p, p, p, p, p, p, i, i, i, NULL, NULL, NULL, NULL, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv4_compact(&d, p, p, p, p, p, p, i, i, i, i, i, INT32_MAX, NULL, NULL, NULL, NULL, NULL, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_kv4_read(&d, INT32_MAX, p, p, p, p, i, i, i, p, p, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_tree_verify_attn_kv4(&d, p, p, p, p, p, p, p, i, i, i, i, p, NULL, NULL, 0, NULL), HB_ERR_WORKSPACE);
  WANT(hb_kv4_attn_weight(&d, p, p, p, i, i, i, i, i, 6, NULL, 1.f, p, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv4_evict(&d, INT32_MAX, 1, 1, p, p, p, p, i, i, i, p, i, p, p, p, NULL, p, SIZE_MAX, NULL), HB_ERR_UNSUPPORTED);
  WANT(hb_kv4_evict(&d, 10, INT32_MAX, INT32_MAX, p, p, p, p, i, i, i, p, i, p, p, p, NULL, p, SIZE_MAX, NULL), HB_ERR_INVALID_ARG);
  WANT(hb_kv4_evict(&d, 10, 1, 1, p, p, p, p, i, i, i, p, i, p, p, p, NULL, p, 8, NULL), HB_ERR_WORKSPACE);
  printf("host shim checks passed\n");
  return 0;
}
