// Host side of the calls that bring requests in and apply their sampling rules: argument validation, plans, dispatch.
#include <initializer_list>

#include "pages.h"
#include "prompt.h"
#include "rules.h"

namespace hb {

static size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
static bool misaligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// What a call writes while other workgroups read, or write something else
struct Span {
  const void *at;
  int64_t bytes;
};
// a pool's bytes, and no more than an address space has
static int64_t pool_bytes(const hb_attn_desc &d) {
  const double n = (double)d.num_blocks * d.page_size * d.num_kv_heads * d.head_dim * (d.dtype == HB_F32 ? 4 : 2);
  return n < 1e18 ? (int64_t)n : (int64_t)1e18;
}
template <typename List = std::initializer_list<Span>>
static int32_t check_apart(const char *name, Span out, const List &in) {
  for (const Span &x : in) {
    const uintptr_t o = (uintptr_t)out.at, i = (uintptr_t)x.at;
    if (o && i && out.bytes > 0 && x.bytes > 0 && o < i + (uint64_t)x.bytes && i < o + (uint64_t)out.bytes)
      return fail(HB_ERR_INVALID_ARG, "%s must not overlap another argument of the call", name);
  }
  return HB_OK;
}

static int32_t check_pages(int32_t B, int32_t page_size, int32_t max_blocks, int32_t num_blocks) {
  if (B < 0) return fail(HB_ERR_INVALID_ARG, "negative batch");
  if (page_size <= 0 || max_blocks <= 0 || num_blocks <= 0)
    return fail(HB_ERR_INVALID_ARG, "page_size, max_blocks_per_seq and num_blocks must be positive");
  if (B > 8192) return fail(HB_ERR_UNSUPPORTED, "batch %d: at most 8192", B);
  if ((int64_t)page_size * max_blocks > (int64_t)1 << 30)
    return fail(HB_ERR_UNSUPPORTED, "page table covers more than 2^30 positions");
  if ((int64_t)page_size * num_blocks > INT32_MAX)
    return fail(HB_ERR_UNSUPPORTED, "%d pages of %d: slots are 32-bit numbers", num_blocks, page_size);
  return HB_OK;
}

// the descriptor as calls without trees read it
static int32_t check_rows_desc(const hb_attn_desc *desc) {
  if (!desc) return fail(HB_ERR_INVALID_ARG, "desc is NULL");
  hb_attn_desc d = *desc;
  d.max_nodes_per_tree = 1;
  int32_t rc = check_attn_desc(&d);
  if (rc) return rc;
  if (d.num_kv_heads > 65535) return fail(HB_ERR_UNSUPPORTED, "num_kv_heads %d: at most 65535", d.num_kv_heads);
  return HB_OK;
}

struct PromptPlan {
  bool mfma;
  int32_t rows;  // of a tile
  int32_t tiles, parts, units;
  size_t ml_offset, heads_offset, bytes;
};

static int32_t make_prompt_plan(const hb_attn_desc *d, PromptPlan *p) {
  int32_t rc = check_rows_desc(d);
  if (rc) return rc;
  if ((int64_t)d->total_nodes * d->num_q_heads > 1 << 30)
    return fail(HB_ERR_UNSUPPORTED, "total_nodes * num_q_heads %lld: at most 2^30", (long long)d->total_nodes * d->num_q_heads);
  const bool can = prompt_mfma_supports(*d);
  if (d->algo == HB_ATTN_MFMA && !can)
    return fail(HB_ERR_UNSUPPORTED, "HB_ATTN_MFMA for prompts needs bf16, head_dim 64 or 128, page_size a power of two and a positive "
                "softmax_scale");
  p->mfma = can && d->algo != HB_ATTN_SCALAR;
  const int64_t G = d->num_q_heads / d->num_kv_heads;
  int64_t span = (int64_t)d->page_size * d->max_blocks_per_seq;
  if (d->max_prefix_len_hint > 0 && d->max_prefix_len_hint < span) span = d->max_prefix_len_hint;
  span += d->total_nodes;
  p->rows = p->mfma ? prompt_mfma_rows(*d) : kPromptAnyRows;
  p->units = p->mfma ? 256 : 512;
  const int64_t least = p->mfma ? 256 : 64;  // keys of a part, about
  const int64_t tiles = d->total_nodes * G / p->rows + (d->batch < d->total_nodes ? d->batch : d->total_nodes);
  p->tiles = (int32_t)tiles;
  int64_t parts = d->num_splits;
  if (parts == 0) {
    // More find nothing to do, at some cost: 64 sequences of a token over 8 K whole 198 us, in at most 3, 7, 15 parts 267, 356, 530
    parts = tiles > 0 ? 2 * p->units / (tiles * d->num_kv_heads) : 1;
    // A join costs 2 to 4 us, as much as a few tiles.  bf16, whole and cut: 4 prompts of 64 rows over 256 positions 20.3 and 24.9,
    // one of 512 24.4 and 27.2; one of 256 over 512 30.7 and 29.3, over 768 37.8 and 31.9.  Float32: 2 prompts of 200 to 256 rows 11.7 and
    // 14.2, one of 512 18.1 and 20.8; one row over 512 20.7 and 14.9.
    if (p->mfma ? span <= 768 : parts < 8 || span <= 512) parts = 1;
  }
  if (parts > span / least) parts = span / least;
  if (parts > 256) parts = 256;
  if (parts < 1) parts = 1;
  p->parts = (int32_t)parts;
  p->ml_offset = p->heads_offset = p->bytes = 0;
  if (parts > 1) {
    const size_t slots = (size_t)tiles * d->num_kv_heads * parts * p->rows;
    p->ml_offset = round_up(slots * d->head_dim * sizeof(float), 256);
    p->heads_offset = p->ml_offset + round_up(slots * 4 * sizeof(float), 256);
    p->bytes = p->heads_offset + round_up((size_t)tiles * sizeof(PromptArgs::Head), 256);
  }
  return HB_OK;
}

struct RulesCall {
  const int32_t *node_offset, *parent, *draft_ids, *counts;
  const float *rules;
  const int32_t *bias_offset;
  int32_t n_bias;
  const int32_t *bias_id;
  const float *bias_value;
  int32_t num_masks;
  const uint32_t *mask;
  const int32_t *mask_row;
};

// What a call with sampling rules writes, apart from what it reads beside the logits
static int32_t check_rules_apart(const char *name, Span out, int32_t B, int32_t T, int32_t V, const RulesCall &r) {
  const int64_t b = B, t = T, n = r.n_bias, words = ((int64_t)V + 31) / 32;
  return check_apart(name, out, {{r.node_offset, 4 * b + 4}, {r.parent, 4 * t}, {r.draft_ids, 4 * t}, {r.counts, 4 * b * V}, {r.rules, 16 * b},
                                 {n ? r.bias_offset : nullptr, 4 * b + 4}, {r.bias_id, 4 * n}, {r.bias_value, 4 * n},
                                 {r.mask, 4 * words * r.num_masks}, {r.mask_row, 4 * t}});
}

static int32_t check_rules(int32_t dtype, int32_t B, int32_t max_nodes, int32_t T, int32_t V, const void *logits, const RulesCall &r,
                           const void *out, RulesArgs *a) {
  if (dtype != HB_F32 && dtype != HB_BF16) return fail(HB_ERR_UNSUPPORTED, "dtype %d: only HB_F32 and HB_BF16 are supported", dtype);
  if (B < 0 || T < 0 || V <= 0 || max_nodes <= 0 || r.n_bias < 0 || r.num_masks < 0)
    return fail(HB_ERR_INVALID_ARG, "batch, rows, biases and masks must not be negative, V and max_nodes_per_tree positive");
  if (max_nodes > 64) return fail(HB_ERR_UNSUPPORTED, "max_nodes_per_tree %d: trees of more than 64 nodes are not supported", max_nodes);
  if (V > 1 << 30) return fail(HB_ERR_UNSUPPORTED, "V %d: at most 2^30", V);
  if (T == 0 || B == 0) return HB_OK;
  if (!logits || !out) return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (!r.node_offset && T != B) return fail(HB_ERR_INVALID_ARG, "without node_offset every sequence has one row: %d of %d", T, B);
  if (!r.parent != !r.draft_ids || (r.parent && !r.node_offset))
    return fail(HB_ERR_INVALID_ARG, "node_offset, parent and draft_ids come together");
  if (r.n_bias > 0 && (!r.bias_offset || !r.bias_id || !r.bias_value))
    return fail(HB_ERR_INVALID_ARG, "bias_offset, bias_id and bias_value come together");
  if (!r.mask && r.mask_row) return fail(HB_ERR_INVALID_ARG, "mask_row without masks");
  if (r.mask && !r.mask_row && r.num_masks < T) return fail(HB_ERR_INVALID_ARG, "without mask_row there is a mask for every row");
  if (misaligned(logits, 16) || misaligned(out, 16) || misaligned(r.counts, 16) || misaligned(r.rules, 16) || misaligned(r.mask, 16))
    return fail(HB_ERR_INVALID_ARG, "logits, out, counts, rules and masks must be 16-byte aligned");
  *a = {dtype, B, max_nodes, T, V, r.n_bias, r.num_masks, logits, r.node_offset, r.parent, r.draft_ids, r.counts, r.rules,
        r.n_bias > 0 ? r.bias_offset : nullptr, r.bias_id, r.bias_value, r.mask, r.mask_row, (void *)out, nullptr, nullptr, 0, 0};
  return HB_OK;
}

}  // namespace hb

using namespace hb;

extern "C" {

int32_t hb_pages_take(int32_t B, int32_t page_size, int32_t max_blocks_per_seq, int32_t num_blocks, int32_t n_rows, int32_t reserve,
                      const int32_t *prefix_len, const int32_t *row_offset, const int32_t *pages, const int32_t *free_pages,
                      const int32_t *free_count, int32_t *block_table, int32_t *slots, int32_t *new_len, int32_t *pages_out,
                      int32_t *granted, int32_t *free_left, void *stream) {
  int32_t rc = check_pages(B, page_size, max_blocks_per_seq, num_blocks);
  if (rc) return rc;
  if (n_rows < 0 || reserve < 0) return fail(HB_ERR_INVALID_ARG, "n_rows and reserve must not be negative");
  if (B == 0) return HB_OK;
  if (!prefix_len || !row_offset || !pages || !free_pages || !free_count || !block_table || !pages_out || !free_left)
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  const Span table = {block_table, (int64_t)B * max_blocks_per_seq * 4}, s = {slots, (int64_t)n_rows * 4}, len = {new_len, (int64_t)B * 4},
             have = {pages_out, (int64_t)B * 4}, ok = {granted, (int64_t)B * 4}, left = {free_left, 4};
  const Span in[] = {{prefix_len, (int64_t)B * 4}, {row_offset, (int64_t)B * 4 + 4}, {pages, (int64_t)B * 4},
                     {free_pages, (int64_t)num_blocks * 4}, {free_count, 4}};
  const Span out[] = {table, s, len, have, ok, left};
  static const char *const names[] = {"block_table", "slots", "new_len", "pages_out", "granted", "free_left"};
  for (int i = 0; i < 6; ++i) {
    if ((rc = check_apart(names[i], out[i], {in[0], in[1], in[2], in[3], in[4]}))) return rc;
    for (int k = 0; k < i; ++k)
      if ((rc = check_apart(names[i], out[i], {out[k]}))) return rc;
  }
  PagesArgs a = {B, page_size, max_blocks_per_seq, num_blocks, n_rows, reserve, prefix_len, row_offset, pages, free_pages, free_count,
                 block_table, nullptr, slots, new_len, pages_out, granted, free_left};
  HB_HIP_TRY(launch_pages_take(a, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_pages_give(int32_t B, int32_t page_size, int32_t max_blocks_per_seq, int32_t num_blocks, const int32_t *keep_len,
                      const int32_t *pages, const int32_t *block_table, int32_t *free_pages, const int32_t *free_count,
                      int32_t *pages_out, int32_t *free_now, void *stream) {
  int32_t rc = check_pages(B, page_size, max_blocks_per_seq, num_blocks);
  if (rc) return rc;
  if (B == 0) return HB_OK;
  if (!keep_len || !pages || !free_pages || !free_count || !block_table || !pages_out || !free_now)
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  const Span in[] = {{keep_len, (int64_t)B * 4}, {pages, (int64_t)B * 4}, {block_table, (int64_t)B * max_blocks_per_seq * 4}, {free_count, 4}};
  const Span out[] = {{free_pages, (int64_t)num_blocks * 4}, {pages_out, (int64_t)B * 4}, {free_now, 4}};
  static const char *const names[] = {"free_pages", "pages_out", "free_now"};
  for (int i = 0; i < 3; ++i) {
    if ((rc = check_apart(names[i], out[i], {in[0], in[1], in[2], in[3]}))) return rc;
    for (int k = 0; k < i; ++k)
      if ((rc = check_apart(names[i], out[i], {out[k]}))) return rc;
  }
  PagesArgs a = {B, page_size, max_blocks_per_seq, num_blocks, 0, 0, keep_len, nullptr, pages, nullptr, free_count,
                 (int32_t *)block_table, free_pages, nullptr, nullptr, pages_out, nullptr, free_now};
  HB_HIP_TRY(launch_pages_give(a, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_kv_append(const hb_attn_desc *desc, int32_t n_rows, const void *k_rows, const void *v_rows, const int32_t *slots, void *k_pool,
                     void *v_pool, void *stream) {
  int32_t rc = check_rows_desc(desc);
  if (rc) return rc;
  if (n_rows < 0) return fail(HB_ERR_INVALID_ARG, "negative n_rows");
  if ((int64_t)desc->page_size * desc->num_blocks > INT32_MAX)
    return fail(HB_ERR_UNSUPPORTED, "%d pages of %d: slots are 32-bit numbers", desc->num_blocks, desc->page_size);
  if (n_rows == 0) return HB_OK;
  if (!k_rows || !v_rows || !slots || !k_pool || !v_pool) return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (misaligned(k_rows, 16) || misaligned(v_rows, 16) || misaligned(k_pool, 16) || misaligned(v_pool, 16))
    return fail(HB_ERR_INVALID_ARG, "rows and pools must be 16-byte aligned");
  const int64_t bytes = (int64_t)n_rows * desc->num_kv_heads * desc->head_dim * (desc->dtype == HB_F32 ? 4 : 2);
  const Span k = {k_pool, pool_bytes(*desc)}, v = {v_pool, k.bytes}, kr = {k_rows, bytes}, vr = {v_rows, bytes}, s = {slots, (int64_t)n_rows * 4};
  if ((rc = check_apart("k_pool", k, {v, kr, vr, s})) || (rc = check_apart("v_pool", v, {kr, vr, s}))) return rc;
  HB_HIP_TRY(launch_kv_append(*desc, n_rows, k_rows, v_rows, slots, k_pool, v_pool, (hipStream_t)stream));
  return HB_OK;
}

size_t hb_prompt_attn_workspace_bytes(const hb_attn_desc *desc) {
  PromptPlan p;
  return make_prompt_plan(desc, &p) ? 0 : p.bytes;
}

int32_t hb_prompt_attn(const hb_attn_desc *desc, const void *q, const void *k_rows, const void *v_rows, const void *k_pool,
                       const void *v_pool, const int32_t *block_table, const int32_t *prefix_len, const int32_t *row_offset, void *out,
                       float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  PromptPlan p;
  int32_t rc = make_prompt_plan(desc, &p);
  if (rc) return rc;
  if (desc->batch == 0 || desc->total_nodes == 0) return HB_OK;
  if (!q || !k_rows || !v_rows || !row_offset || !out) return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (prefix_len && (!k_pool || !v_pool || !block_table))
    return fail(HB_ERR_INVALID_ARG, "prefix_len without pools and block_table");
  if (misaligned(q, 16) || misaligned(k_rows, 16) || misaligned(v_rows, 16) || misaligned(k_pool, 16) || misaligned(v_pool, 16) ||
      misaligned(out, 16))
    return fail(HB_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  const int64_t el = desc->dtype == HB_F32 ? 4 : 2, rows = (int64_t)desc->total_nodes * desc->head_dim;
  const Span in[] = {{q, rows * desc->num_q_heads * el}, {k_rows, rows * desc->num_kv_heads * el}, {v_rows, rows * desc->num_kv_heads * el}},
             o = {out, rows * desc->num_q_heads * el}, l = {lse, (int64_t)desc->total_nodes * desc->num_q_heads * 4};
  if ((rc = check_apart("out", o, {in[0], in[1], in[2], l})) || (rc = check_apart("lse", l, {in[0], in[1], in[2]}))) return rc;
  if (p.bytes) {
    if (!workspace || workspace_bytes < p.bytes)
      return fail(HB_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", p.bytes, workspace ? workspace_bytes : (size_t)0);
    if (misaligned(workspace, 256)) return fail(HB_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if ((rc = check_apart("workspace", {workspace, (int64_t)p.bytes}, {in[0], in[1], in[2], o, l}))) return rc;
  }
  const int64_t B = desc->batch, pool = prefix_len ? pool_bytes(*desc) : 0;
  const Span cache[] = {{k_pool, pool}, {v_pool, pool}, {block_table, prefix_len ? B * desc->max_blocks_per_seq * 4 : 0}, {prefix_len, 4 * B},
                        {row_offset, 4 * B + 4}};
  if ((rc = check_apart("out", o, cache)) || (rc = check_apart("lse", l, cache)) ||
      (p.bytes && (rc = check_apart("workspace", {workspace, (int64_t)p.bytes}, cache))))
    return rc;
  PromptArgs a = {*desc, q, k_rows, v_rows, k_pool, v_pool, block_table, prefix_len, row_offset, out, lse,
                  p.bytes ? (float *)workspace : nullptr, p.bytes ? (float *)((char *)workspace + p.ml_offset) : nullptr,
                  p.bytes ? (PromptArgs::Head *)((char *)workspace + p.heads_offset) : nullptr, p.tiles, p.parts, p.units};
  if (p.mfma)
    HB_HIP_TRY(launch_prompt_mfma(a, (hipStream_t)stream));
  else
    HB_HIP_TRY(launch_prompt_any(a, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_rules_count(int32_t B, int32_t V, int32_t n, const int32_t *row_offset, const int32_t *tokens, int32_t prompt, int32_t *counts,
                       void *stream) {
  if (B < 0 || n < 0 || V <= 0) return fail(HB_ERR_INVALID_ARG, "batch and n must not be negative, V positive");
  if (prompt != 0 && prompt != 1) return fail(HB_ERR_INVALID_ARG, "prompt must be 0 or 1");
  if (B == 0 || n == 0) return HB_OK;
  if (!tokens || !counts) return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (!row_offset && n % B) return fail(HB_ERR_INVALID_ARG, "without row_offset every sequence has as many tokens: %d of %d", n, B);
  int32_t rc;
  if ((rc = check_apart("counts", {counts, (int64_t)B * V * 4}, {{tokens, (int64_t)n * 4}, {row_offset, (int64_t)B * 4 + 4}}))) return rc;
  HB_HIP_TRY(launch_rules_count(B, V, n, row_offset, tokens, prompt, counts, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_rules_logits(int32_t dtype, int32_t B, int32_t max_nodes_per_tree, int32_t T, int32_t V, const void *logits,
                        const int32_t *node_offset, const int32_t *parent, const int32_t *draft_ids, const int32_t *counts,
                        const float *rules, const int32_t *bias_offset, int32_t n_bias, const int32_t *bias_id, const float *bias_value,
                        int32_t num_masks, const uint32_t *mask, const int32_t *mask_row, void *out, void *stream) {
  RulesArgs a;
  const RulesCall r = {node_offset, parent, draft_ids, counts, rules, bias_offset, n_bias, bias_id, bias_value, num_masks, mask, mask_row};
  int32_t rc = check_rules(dtype, B, max_nodes_per_tree, T, V, logits, r, out, &a);
  if (rc || T == 0 || B == 0) return rc;
  const int64_t bytes = (int64_t)T * V * (dtype == HB_F32 ? 4 : 2);
  if (out != logits && (rc = check_apart("out", {out, bytes}, {{logits, bytes}}))) return rc;
  if ((rc = check_rules_apart("out", {out, bytes}, B, T, V, r))) return rc;
  HB_HIP_TRY(launch_rules_logits(a, (hipStream_t)stream));
  return HB_OK;
}

size_t hb_rules_probs_workspace_bytes(int32_t T, int32_t V) {
  if (T <= 0 || V <= 0 || V > 1 << 30) return 0;
  int32_t chunk;
  const int32_t parts = rules_parts(T, V, &chunk);
  if (parts) return (size_t)T * parts * 16;
  return (size_t)(T / 4) * (((size_t)V + 31) / 32) * 4;  // marks of at most so many sequences: with more, there are none
}

int32_t hb_rules_probs(int32_t dtype, int32_t B, int32_t max_nodes_per_tree, int32_t T, int32_t V, const void *logits,
                       const int32_t *node_offset, const int32_t *parent, const int32_t *draft_ids, const int32_t *counts,
                       const float *rules, const int32_t *bias_offset, int32_t n_bias, const int32_t *bias_id, const float *bias_value,
                       int32_t num_masks, const uint32_t *mask, const int32_t *mask_row, float *probs, void *workspace,
                       size_t workspace_bytes, void *stream) {
  RulesArgs a;
  const RulesCall r = {node_offset, parent, draft_ids, counts, rules, bias_offset, n_bias, bias_id, bias_value, num_masks, mask, mask_row};
  int32_t rc = check_rules(dtype, B, max_nodes_per_tree, T, V, logits, r, probs, &a);
  if (rc || T == 0 || B == 0) return rc;
  const size_t need = hb_rules_probs_workspace_bytes(T, V);
  if (need && (!workspace || workspace_bytes < need))
    return fail(HB_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  if (need && misaligned(workspace, 16)) return fail(HB_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  const int64_t el = dtype == HB_F32 ? 4 : 2;
  const Span in = {logits, (int64_t)T * V * el}, o = {probs, (int64_t)T * V * 4};
  if ((rc = check_apart("probs", o, {in})) || (need && (rc = check_apart("workspace", {workspace, (int64_t)need}, {in, o})))) return rc;
  if ((rc = check_rules_apart("probs", o, B, T, V, r)) || (need && (rc = check_rules_apart("workspace", {workspace, (int64_t)need}, B, T, V, r))))
    return rc;
  int32_t chunk;
  if (rules_parts(T, V, &chunk))
    a.stats = (float *)workspace;
  else if (counts && rules_marks(B, T))
    a.marks = (uint32_t *)workspace;
  HB_HIP_TRY(launch_rules_probs(a, (hipStream_t)stream));
  return HB_OK;
}

}  // extern "C"
