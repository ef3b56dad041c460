// What the kernels of the 4-bit cache share: the number format, the slot of a position, the sequence of a row.
//
// A row (one position and head of K or V) is D elements of 4 bits, E2M1 (sign, two exponent bits, one mantissa
// bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte with the even element in the low half, and one scale byte s for every 32
// of them, worth 2^(s - 127) (255: not a number).  The matrix cores of gfx950 multiply this form as it is, and every value
// that hb_kv4_append writes is exact in bf16.
#pragma once
#include "hb_internal.h"

namespace hb {

constexpr int kKv4Block = 32;       // elements under one scale
constexpr int kKv4NaN = 255;        // scale byte of a block that held something that is not finite
constexpr int kKv4MaxScale = 252;   // 6 * 2^125 is the largest value that is written

struct Kv4Pool {
  const uint8_t *codes, *scales;  // [blocks][Hkv][page][D / 2], [blocks][Hkv][page][D / 32]
};

// part_o, part_ml: of row r = node * Hq + head and chunk c at (r * splits + c) * D and * 2: sums against the chunk's
// largest score, that score (log2 units from the matrix-core kernels, natural ones from the scalar kernel), the sum of weights.
// Unused where splits is 1.
struct Kv4AttnArgs {
  hb_attn_desc d;
  int32_t splits, chunk;  // chunks of a prefix, and their length in positions
  const void *q, *k_tree, *v_tree;
  Kv4Pool kp, vp;
  const int32_t *block_table, *prefix_len, *node_offset, *parent;
  void *out;
  float *lse, *part_o, *part_ml;
  int32_t *cut;  // the matrix-core kernels' chunk length, in grains, or null where they do not cut
};
// How the matrix-core kernel cuts the prefixes, from what the host knows
struct Kv4Plan {
  int32_t row_groups;   // workgroups that share a chunk's query rows, at most
  int32_t heads;        // query heads of a kv head
  int32_t group_shift;  // log2 of the query rows of a row group
  int32_t grain_shift;  // log2 of the keys that a chunk's length is a multiple of, its grains
  int32_t target;       // workgroups per kv head, over all sequences
  int32_t fit;          // not more than these, if longer chunks can do it
  int32_t splits;       // chunks of a sequence, at most: slots of part_o and part_ml
  int32_t grid;         // workgroups that are started
  uint32_t page_magic;  // ceil(2^32 / (page_size / 16)), 0 where that is one
};
bool kv4_attn_supports(const hb_attn_desc &d);
void kv4_attn_plan(const hb_attn_desc &d, int64_t span, Kv4Plan *plan);
hipError_t launch_kv4_attn(const Kv4AttnArgs &a, const Kv4Plan &plan, hipStream_t s);

hipError_t launch_kv4_attn_scalar(const Kv4AttnArgs &a, hipStream_t s);
hipError_t launch_kv4_merge(const Kv4AttnArgs &a, hipStream_t s);

struct Kv4WeightArgs {
  hb_attn_desc d;
  int32_t max_path;
  float decay;
  const void *q;
  Kv4Pool kp;
  const int32_t *block_table, *prefix_len, *node_offset, *accept_len, *accept_path;  // the last two may be null
  const float *lse;
  float *weight;
};
hipError_t launch_kv4_weight_scalar(const Kv4WeightArgs &a, int32_t longest, hipStream_t s);
bool kv4_weight_supports(const hb_attn_desc &d);
hipError_t launch_kv4_weight_mfma(const Kv4WeightArgs &a, int32_t longest, hipStream_t s);

__device__ inline float kv4_scale(uint32_t s) {
  return __uint_as_float(s == kKv4NaN ? 0x7fc00000u : s == 0 ? 0x00400000u : s << 23);
}

typedef float kv4_f32x2 __attribute__((ext_vector_type(2)));

// A float32 as three bf16 pieces, which is all of it.  The first is cut off behind its eight bits: rounded, it would be an infinity
// from 2^128 - 2^119 on, and the others infinities and NaN with it.
__device__ __forceinline__ float kv4_cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint32_t kv4_pack_cut(float lo, float hi) {  // of two
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}

// two elements, from byte SEL of `codes`
template <int SEL>
__device__ inline kv4_f32x2 kv4_pair(uint32_t codes, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.f, SEL) * scale;
}

// the scale byte of a block whose largest magnitude is `top` (its float bits): the smallest power of two that
// brings it to 7 or less.  What is above 6 becomes 6: 7 is where that loses as much as the next larger scale
// would (N(0, 1) in blocks of 32: 19.0 dB signal to error; with 6 or 8 in its place 18.8)
__device__ inline uint32_t kv4_scale_of(uint32_t top) {
  if (top >= 0x7f800000u) return kKv4NaN;
  const int s = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)(s < 1 ? 1 : s > kKv4MaxScale ? kKv4MaxScale : s);
}

// index of position p's row among all rows of a pool, for one head; p lies in [0, max_blocks_per_seq * page_size)
__device__ inline size_t kv4_row(const hb_attn_desc &d, const int32_t *__restrict__ block_table, int b, int h, int p) {
  int blk = block_table[(size_t)b * d.max_blocks_per_seq + p / d.page_size];
  blk = blk < 0 ? 0 : (blk >= d.num_blocks ? d.num_blocks - 1 : blk);
  return ((size_t)blk * d.num_kv_heads + h) * d.page_size + p % d.page_size;
}

__device__ inline int kv4_length(const hb_attn_desc &d, const int32_t *__restrict__ prefix_len, int b) {
  const int cap = d.max_blocks_per_seq * d.page_size, L = prefix_len[b];
  return L < 0 ? 0 : L > cap ? cap : L;
}

// the last sequence whose first row is not behind r (0 where none is)
__device__ inline int kv4_sequence(const int32_t *__restrict__ offset, int batch, int r) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (offset[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

}  // namespace hb
