// Arguments of the calls that apply a request's sampling rules to logits (rules.hip).
#pragma once
#include "hb_internal.h"

namespace hb {

constexpr int32_t kPromptFlag = 1 << 30;  // of a count: the token is in the prompt

struct RulesArgs {
  int32_t dtype, batch, max_nodes, rows, V, n_bias, num_masks;
  const void *logits;
  const int32_t *node_offset;        // null: row t is sequence t's
  const int32_t *parent, *draft_ids;  // null: no paths
  const int32_t *counts;             // null: no tokens so far
  const float *rules;                // null: temperature 1, no penalties
  const int32_t *bias_offset, *bias_id;
  const float *bias_value;
  const uint32_t *mask;
  const int32_t *mask_row;
  void *out;
  uint32_t *marks;  // null, or [batch][(V + 31) / 32]: where rows have a workgroup each, and are several to a sequence
  float *stats;  // [rows][parts][4]: largest, sum, its token (as an integer), nothing
  int32_t parts, chunk;  // of a row: workgroups (0: one, without stats), and tokens of each
};
bool rules_marks(int32_t B, int32_t T);
int32_t rules_parts(int32_t rows, int32_t V, int32_t *chunk);
hipError_t launch_rules_logits(RulesArgs a, hipStream_t s);
hipError_t launch_rules_probs(RulesArgs a, hipStream_t s);
hipError_t launch_rules_count(int32_t B, int32_t V, int32_t n, const int32_t *row_offset, const int32_t *tokens, int32_t prompt,
                              int32_t *counts, hipStream_t s);

}  // namespace hb
