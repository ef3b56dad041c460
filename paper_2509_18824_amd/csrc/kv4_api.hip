// Host side of the calls over the 4-bit cache: argument validation, the cut of the prefix, dispatch.
#include "kv4.h"

#include <initializer_list>

namespace hb {

static size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
static bool misaligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

static int32_t check_kv4(const hb_attn_desc *desc) {
  int32_t rc = check_attn_desc(desc);
  if (rc) return rc;
  if (desc->head_dim % kKv4Block)
    return fail(HB_ERR_UNSUPPORTED, "head_dim %d: the 4-bit cache needs a multiple of %d", desc->head_dim, kKv4Block);
  if ((int64_t)desc->batch * desc->num_kv_heads > 65535)
    return fail(HB_ERR_UNSUPPORTED, "batch * num_kv_heads %lld: at most 65535", (long long)desc->batch * desc->num_kv_heads);
  if ((int64_t)desc->total_nodes * desc->num_q_heads > 1 << 23)
    return fail(HB_ERR_UNSUPPORTED, "total_nodes * num_q_heads %lld: at most 2^23", (long long)desc->total_nodes * desc->num_q_heads);
  return HB_OK;
}

// the cache alone: fields that only attention needs may hold anything (a bound on lengths sizes eviction's launches)
static int32_t check_kv4_cache(const hb_attn_desc *desc) {
  if (!desc) return fail(HB_ERR_INVALID_ARG, "desc is NULL");
  hb_attn_desc d = *desc;
  d.max_nodes_per_tree = 1;
  d.num_splits = d.max_prefix_len_hint = 0;
  d.algo = HB_ATTN_AUTO;
  return check_kv4(&d);
}

static int32_t check_pool(const void *k_codes, const void *k_scales, const void *v_codes, const void *v_scales) {
  if (!k_codes || !k_scales || !v_codes || !v_scales) return fail(HB_ERR_INVALID_ARG, "a pool's device pointer is NULL");
  if (misaligned(k_codes, 16) || misaligned(k_scales, 16) || misaligned(v_codes, 16) || misaligned(v_scales, 16))
    return fail(HB_ERR_INVALID_ARG, "codes and scales must be 16-byte aligned");
  return HB_OK;
}

// What a call writes while other workgroups read its integers
struct Ints {
  const int32_t *at;
  int64_t n;
};
static int32_t check_apart(const char *name, Ints out, std::initializer_list<Ints> in) {
  for (const Ints &x : in) {
    const uintptr_t o = (uintptr_t)out.at, i = (uintptr_t)x.at;
    if (o && i && o < i + (uint64_t)x.n * 4 && i < o + (uint64_t)out.n * 4)
      return fail(HB_ERR_INVALID_ARG, "%s must not overlap the lengths, offsets and paths that the call reads", name);
  }
  return HB_OK;
}

// a launch has a thread for eight elements of every row
static int32_t check_rows(int64_t rows, const hb_attn_desc *d) {
  if (rows * d->num_kv_heads * (d->head_dim / 8) > INT32_MAX)
    return fail(HB_ERR_UNSUPPORTED, "%lld rows of %d heads of %d in one call", (long long)rows, d->num_kv_heads, d->head_dim);
  return HB_OK;
}

static int64_t span_of(const hb_attn_desc *d) {
  const int64_t cap = (int64_t)d->page_size * d->max_blocks_per_seq;
  return d->max_prefix_len_hint > 0 && d->max_prefix_len_hint < cap ? d->max_prefix_len_hint : cap;
}

struct AttnCut {
  bool mfma;
  Kv4Plan plan;            // the matrix-core kernel's
  int32_t splits, chunk;   // slots of a row's partial results; the scalar kernel's chunk length
  size_t ml_offset, cut_offset, bytes;
};

static int32_t make_cut(const hb_attn_desc *d, AttnCut *cut) {
  int32_t rc = check_kv4(d);
  if (rc) return rc;
  const bool can = kv4_attn_supports(*d);
  if (d->algo == HB_ATTN_MFMA && !can)
    return fail(HB_ERR_UNSUPPORTED, "HB_ATTN_MFMA over the 4-bit cache needs head_dim 64 or 128, page_size a multiple of 16 up to "
                "1024, a positive softmax_scale and Hq/Hkv <= 512");
  cut->mfma = can && d->algo != HB_ATTN_SCALAR;
  const int64_t rows = (int64_t)d->total_nodes * d->num_q_heads, span = span_of(d);
  if (cut->mfma) {
    kv4_attn_plan(*d, span, &cut->plan);
    cut->splits = cut->plan.splits;
  } else {
    int64_t splits = d->num_splits;
    if (splits == 0) {
      splits = rows > 0 ? (2048 + rows - 1) / rows : 1;
      if (splits > (span + 255) / 256) splits = (span + 255) / 256;
    }
    if (splits > 1024) splits = 1024;
    int64_t chunk = (span + splits - 1) / splits;
    chunk = (chunk + 63) / 64 * 64;
    cut->splits = (int32_t)((span + chunk - 1) / chunk);
    cut->chunk = (int32_t)chunk;
  }
  cut->ml_offset = cut->splits > 1 ? round_up((size_t)rows * cut->splits * d->head_dim * 4, 256) : 0;
  cut->cut_offset = cut->splits > 1 ? cut->ml_offset + round_up((size_t)rows * cut->splits * 8, 256) : 0;
  cut->bytes = cut->splits > 1 ? cut->cut_offset + 256 : 0;
  return HB_OK;
}

}  // namespace hb

using namespace hb;

extern "C" {

int32_t hb_kv4_append(const hb_attn_desc *desc, int32_t n_rows, const void *k_rows, const void *v_rows, void *k_codes,
                      void *k_scales, void *v_codes, void *v_scales, const int32_t *block_table, const int32_t *prefix_len,
                      const int32_t *row_offset, const int32_t *seq_len, float *weight, int32_t *pos, int32_t *new_len,
                      void *stream) {
  int32_t rc = check_kv4_cache(desc);
  if (rc) return rc;
  if (n_rows < 0) return fail(HB_ERR_INVALID_ARG, "negative n_rows");
  if (desc->batch == 0) return HB_OK;
  if ((rc = check_rows(n_rows, desc)) || (rc = check_pool(k_codes, k_scales, v_codes, v_scales))) return rc;
  if ((n_rows && (!k_rows || !v_rows)) || !block_table || !prefix_len || !row_offset)
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  const int64_t B = desc->batch;
  if ((rc = check_apart("new_len", {new_len, B}, {{prefix_len, B}, {row_offset, B + 1}, {seq_len, B}}))) return rc;
  if (misaligned(k_rows, 16) || misaligned(v_rows, 16)) return fail(HB_ERR_INVALID_ARG, "k_rows and v_rows must be 16-byte aligned");
  Kv4AppendArgs a = {*desc, n_rows, n_rows, 0, k_rows, v_rows, (uint8_t *)k_codes, (uint8_t *)k_scales, (uint8_t *)v_codes,
                     (uint8_t *)v_scales, block_table, prefix_len, row_offset, nullptr, nullptr, seq_len, weight, pos, nullptr, new_len};
  HB_HIP_TRY(launch_kv4_append(a, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_kv4_compact(const hb_attn_desc *desc, const void *k_tree, const void *v_tree, void *k_codes, void *k_scales,
                       void *v_codes, void *v_scales, const int32_t *block_table, const int32_t *prefix_len,
                       const int32_t *node_offset, const int32_t *accept_len, const int32_t *accept_path, int32_t max_path,
                       const int32_t *seq_len, float *weight, int32_t *pos, int32_t *out_slots, int32_t *new_len, void *stream) {
  int32_t rc = check_kv4_cache(desc);
  if (rc) return rc;
  if (max_path <= 0) return fail(HB_ERR_INVALID_ARG, "max_path must be positive");
  if (desc->batch == 0) return HB_OK;
  if ((rc = check_rows((int64_t)desc->batch * max_path, desc)) || (rc = check_pool(k_codes, k_scales, v_codes, v_scales))) return rc;
  if (!block_table || !prefix_len || !node_offset || !accept_len || !accept_path)
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (desc->total_nodes && (!k_tree || !v_tree)) return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  const int64_t B = desc->batch;
  const std::initializer_list<Ints> in = {{prefix_len, B}, {node_offset, B + 1}, {accept_len, B}, {accept_path, B * max_path}, {seq_len, B}};
  if ((rc = check_apart("new_len", {new_len, B}, in)) || (rc = check_apart("out_slots", {out_slots, B * max_path}, in))) return rc;
  if (misaligned(k_tree, 16) || misaligned(v_tree, 16)) return fail(HB_ERR_INVALID_ARG, "k_tree and v_tree must be 16-byte aligned");
  Kv4AppendArgs a = {*desc, desc->batch * max_path, desc->total_nodes, max_path, k_tree, v_tree, (uint8_t *)k_codes, (uint8_t *)k_scales,
                     (uint8_t *)v_codes, (uint8_t *)v_scales, block_table, prefix_len, node_offset, accept_len, accept_path, seq_len,
                     weight, pos, out_slots, new_len};
  HB_HIP_TRY(launch_kv4_append(a, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_kv4_read(const hb_attn_desc *desc, int32_t n_rows, const void *k_codes, const void *k_scales, const void *v_codes,
                    const void *v_scales, const int32_t *block_table, const int32_t *first, const int32_t *row_offset,
                    void *k_rows, void *v_rows, void *stream) {
  int32_t rc = check_kv4_cache(desc);
  if (rc) return rc;
  if (n_rows < 0) return fail(HB_ERR_INVALID_ARG, "negative n_rows");
  if (desc->batch == 0 || n_rows == 0) return HB_OK;
  if ((rc = check_rows(n_rows, desc)) || (rc = check_pool(k_codes, k_scales, v_codes, v_scales))) return rc;
  if (!block_table || !first || !row_offset || !k_rows || !v_rows) return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (misaligned(k_rows, 16) || misaligned(v_rows, 16)) return fail(HB_ERR_INVALID_ARG, "k_rows and v_rows must be 16-byte aligned");
  HB_HIP_TRY(launch_kv4_read(*desc, n_rows, {(const uint8_t *)k_codes, (const uint8_t *)k_scales},
                             {(const uint8_t *)v_codes, (const uint8_t *)v_scales}, block_table, first, row_offset, k_rows, v_rows,
                             (hipStream_t)stream));
  return HB_OK;
}

size_t hb_tree_verify_attn_kv4_workspace_bytes(const hb_attn_desc *desc) {
  AttnCut cut;
  return make_cut(desc, &cut) ? 0 : cut.bytes;
}

int32_t hb_tree_verify_attn_kv4_num_splits(const hb_attn_desc *desc) {
  AttnCut cut;
  return make_cut(desc, &cut) ? 0 : cut.splits;
}

int32_t hb_tree_verify_attn_kv4(const hb_attn_desc *desc, const void *q, const void *k_tree, const void *v_tree,
                                const void *k_codes, const void *k_scales, const void *v_codes, const void *v_scales,
                                const int32_t *block_table, const int32_t *prefix_len, const int32_t *node_offset,
                                const int32_t *parent, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                void *stream) {
  AttnCut cut;
  int32_t rc = make_cut(desc, &cut);
  if (rc) return rc;
  if (desc->batch == 0 || desc->total_nodes == 0) return HB_OK;
  if ((rc = check_pool(k_codes, k_scales, v_codes, v_scales))) return rc;
  if (!q || !k_tree || !v_tree || !block_table || !prefix_len || !node_offset || !parent || !out)
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (misaligned(q, 16) || misaligned(k_tree, 16) || misaligned(v_tree, 16) || misaligned(out, 16))
    return fail(HB_ERR_INVALID_ARG, "q, k_tree, v_tree and out must be 16-byte aligned");
  if (cut.bytes) {
    if (!workspace || workspace_bytes < cut.bytes)
      return fail(HB_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", cut.bytes, workspace ? workspace_bytes : (size_t)0);
    if (misaligned(workspace, 256)) return fail(HB_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  }
  Kv4AttnArgs a = {*desc, cut.splits, cut.chunk, q, k_tree, v_tree, {(const uint8_t *)k_codes, (const uint8_t *)k_scales},
                   {(const uint8_t *)v_codes, (const uint8_t *)v_scales}, block_table, prefix_len, node_offset, parent, out, lse,
                   (float *)workspace, (float *)((char *)workspace + cut.ml_offset),
                   cut.bytes ? (int32_t *)((char *)workspace + cut.cut_offset) : nullptr};
  if (cut.mfma) {
    HB_HIP_TRY(launch_kv4_attn(a, cut.plan, (hipStream_t)stream));
    return HB_OK;
  }
  HB_HIP_TRY(launch_kv4_attn_scalar(a, (hipStream_t)stream));
  if (cut.splits > 1) HB_HIP_TRY(launch_kv4_merge(a, (hipStream_t)stream));
  return HB_OK;
}

int32_t hb_kv4_attn_weight(const hb_attn_desc *desc, const void *q, const void *k_codes, const void *k_scales,
                           const int32_t *block_table, const int32_t *prefix_len, const int32_t *node_offset,
                           const int32_t *accept_len, const int32_t *accept_path, int32_t max_path, const float *lse, float decay,
                           float *weight, void *stream) {
  int32_t rc = check_kv4(desc);
  if (rc) return rc;
  if (!(decay >= 0.f) || !(decay <= 1.f)) return fail(HB_ERR_INVALID_ARG, "decay must lie in [0, 1]");
  if (!accept_len != !accept_path) return fail(HB_ERR_INVALID_ARG, "accept_len and accept_path come together");
  if (accept_path && max_path <= 0) return fail(HB_ERR_INVALID_ARG, "max_path must be positive");
  if (desc->batch == 0) return HB_OK;
  if (!k_codes || !k_scales || !block_table || !prefix_len || !node_offset || !weight || (desc->total_nodes && (!q || !lse)))
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if (misaligned(q, 16) || misaligned(k_codes, 16) || misaligned(k_scales, 16))
    return fail(HB_ERR_INVALID_ARG, "q, codes and scales must be 16-byte aligned");
  Kv4WeightArgs a = {*desc, max_path, decay, q, {(const uint8_t *)k_codes, (const uint8_t *)k_scales}, block_table, prefix_len,
                     node_offset, accept_len, accept_path, lse, weight};
  if (desc->algo != HB_ATTN_SCALAR && kv4_weight_supports(*desc))
    HB_HIP_TRY(launch_kv4_weight_mfma(a, (int32_t)span_of(desc), (hipStream_t)stream));
  else
    HB_HIP_TRY(launch_kv4_weight_scalar(a, (int32_t)span_of(desc), (hipStream_t)stream));
  return HB_OK;
}

struct EvictLayout {
  int64_t parts;
  size_t counts, least, parts_at, bytes;
};
static EvictLayout evict_layout(const hb_attn_desc *d, int32_t budget) {
  const size_t units = (size_t)d->batch * d->num_kv_heads;
  EvictLayout e;
  e.parts = ((int64_t)d->page_size * d->max_blocks_per_seq + 255) / 256;
  e.counts = round_up(units * 2 * budget * 4, 256);
  e.least = e.counts + round_up(units * 4, 256);
  e.parts_at = e.least + round_up(units * 8, 256);
  e.bytes = e.parts_at + round_up(units * e.parts * 8, 256);
  return e;
}

size_t hb_kv4_evict_workspace_bytes(const hb_attn_desc *desc, int32_t budget) {
  if (check_kv4_cache(desc) || budget <= 0 || desc->batch == 0) return 0;
  return evict_layout(desc, budget).bytes;
}

int32_t hb_kv4_evict(const hb_attn_desc *desc, int32_t budget, int32_t recent, int32_t sinks, void *k_codes, void *k_scales,
                     void *v_codes, void *v_scales, const int32_t *block_table, const int32_t *prefix_len, const int32_t *seq_len,
                     const float *weight, const int32_t *pos, float *weight_out, int32_t *pos_out, int32_t *kept,
                     int32_t *new_len, void *workspace, size_t workspace_bytes, void *stream) {
  int32_t rc = check_kv4_cache(desc);
  if (rc) return rc;
  if (budget <= 0 || recent < 0 || sinks < 0 || (int64_t)recent + sinks > budget)
    return fail(HB_ERR_INVALID_ARG, "budget %d must be positive and hold the %d recent and %d first positions", budget, recent, sinks);
  if (budget > 1 << 30) return fail(HB_ERR_UNSUPPORTED, "budget %d: at most 2^30", budget);
  if (desc->batch == 0) return HB_OK;
  if ((rc = check_pool(k_codes, k_scales, v_codes, v_scales))) return rc;
  if (!block_table || !prefix_len || !seq_len || !weight || !pos || !weight_out || !pos_out || !kept)
    return fail(HB_ERR_INVALID_ARG, "a required device pointer is NULL");
  if ((rc = check_apart("new_len", {new_len, desc->batch}, {{prefix_len, desc->batch}, {seq_len, desc->batch}}))) return rc;
  const EvictLayout at = evict_layout(desc, budget);
  const size_t need = at.bytes;
  if (!workspace || workspace_bytes < need)
    return fail(HB_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  if (misaligned(workspace, 256)) return fail(HB_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  Kv4EvictArgs a = {*desc, budget, recent, sinks, (uint8_t *)k_codes, (uint8_t *)k_scales, (uint8_t *)v_codes, (uint8_t *)v_scales,
                    block_table, prefix_len, seq_len, weight, pos, weight_out, pos_out, kept, new_len, (int32_t *)workspace,
                    (int32_t *)((char *)workspace + at.counts), (int32_t *)((char *)workspace + at.least),
                    (int32_t *)((char *)workspace + at.parts_at), (int32_t)at.parts, (int32_t)span_of(desc), 0, 0};
  HB_HIP_TRY(launch_kv4_evict(a, (hipStream_t)stream));
  return HB_OK;
}

}  // extern "C"
