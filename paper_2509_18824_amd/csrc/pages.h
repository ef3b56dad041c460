// Arguments of the page calls (pages.hip).
#pragma once
#include "hb_internal.h"

namespace hb {

struct PagesArgs {
  int32_t batch, page, max_blocks, num_blocks, n_rows, reserve;
  const int32_t *len;         // take: positions there; give: positions to keep
  const int32_t *row_offset;  // take
  const int32_t *have, *free_pages, *free_count;
  int32_t *table;             // take: written
  int32_t *free_out;          // give: written
  int32_t *slots, *new_len, *have_out, *granted, *left;  // slots, new_len and granted may be null
};
hipError_t launch_pages_take(const PagesArgs &a, hipStream_t s);
hipError_t launch_pages_give(const PagesArgs &a, hipStream_t s);
hipError_t launch_kv_append(const hb_attn_desc &d, int32_t n, const void *k, const void *v, const int32_t *slots, void *k_pool,
                            void *v_pool, hipStream_t s);

}  // namespace hb
