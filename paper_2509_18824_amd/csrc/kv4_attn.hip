// Attention over the 4-bit cache on the matrix cores of gfx950 (bf16, heads of 64 and 128, pages of a multiple of 16).
//
// Formulation (transposed, so that no score crosses lanes on its way into the second product):
//   S^T = K Q^T     v_mfma_scale_f32_16x16x128_f8f6f4: A = 16 cached keys as they lie in memory, 4 bits and a scale byte for
//                   every 32 elements (a lane holds one block: 16 bytes); B = 16 query rows in 8 bits, twice
//   O^T = V^T P^T   v_mfma_f32_16x16x32_bf16: A = V^T (16 d x 32 keys), values widened to bf16, which is exact
// A query row is cut in two 8-bit pieces: q = 2^(E-7) (hi + lo / 16), E the exponent of the row's largest element, hi and lo
// E4M3.  Eight significant bits are two times four, so the pieces are q exactly, except for elements below 2^-14 of the largest
// (what is lost lies below 2^-22 of it).  Two such products take 2.4 times a bf16 product of a quarter of the length, and
// keys are never unpacked.  The matrix core drops what lies some 2^-15 below the largest product of a sum: scores are off by
// 5e-6 of their spread (root of the mean square, N(0, 1) data), where bf16 probabilities are off by 2e-3.
// Probabilities are rounded to bf16 for the second product, sums are kept in 32 bits.
//
// A wavefront takes 32 keys at a time of its own and TPW tiles of 16 query rows (row = node * G + head of the group); the
// wavefronts of a workgroup take turns on the steps of a chunk of the prefix and join their results in LDS at its end.  Nobody
// waits for anybody in between: a step's codes go from memory to registers two steps ahead, keys to the matrix core as they
// are, values through 8 KB of LDS of the wavefront's own, where a transposing read turns them.
//
// Chunks are cut on the device from the lengths (kv4_plan below), so that about as many workgroups start as the host planned
// for, whatever the lengths are.
#include "kv4.h"
#include "wave_ops.h"

#include <type_traits>

namespace hb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4_ptr;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int swap2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;  // keys
constexpr int kWaves = 4;  // of a workgroup
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // log2 units a score may exceed its row's reference
constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// maximum over the lanes l, l^16, l^32, l^48
__device__ __forceinline__ float group_max(float x) {
  swap2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float group_sum(float x) {
  swap2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// a / b for 0 <= a < 2^16, 0 < b < 2^16
__device__ __forceinline__ int small_div(int a, int b) { return (int)(((float)a + 0.5f) * __builtin_amdgcn_rcpf((float)b)); }

// XOR on the 16-byte piece index of a key's row of values in LDS: transposing reads and the writes of 16 keys both
// spread over all banks
__device__ __forceinline__ int v_swz(int key) { return ((key & 7) << 1) | ((key >> 3) & 1); }

__device__ __forceinline__ uint32_t finite_or_zero_bf16x2(uint32_t w) {
  uint32_t lo = ((w & 0x7f80u) == 0x7f80u) ? 0u : (w & 0xffffu);
  uint32_t hi = ((w & 0x7f800000u) == 0x7f800000u) ? 0u : (w & 0xffff0000u);
  return lo | hi;
}

// 16 query rows as the B operand: lane (j, kg) holds d = 16 kg + 0 .. 15 and 64 + 16 kg + 0 .. 15 of row j
struct QTile {
  i32x8 hi, lo;
  int hi_scale, lo_scale;
};

template <int DB>
__device__ __forceinline__ void split_rows(const u32x4 (&x)[4], QTile &q) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 2 * (DB / 2); ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max((x[i][e] << 16) & 0x7fffffffu, x[i][e] & 0x7fff0000u));
  top = __float_as_uint(group_max(__uint_as_float(top > 0x7f800000u ? 0x7f800000u : top)));
  const bool fine = top < 0x7f800000u;
  int E = (int)(top >> 23) - 127;
  E = E < -115 ? -115 : E;
  const float unit = __uint_as_float((uint32_t)(127 + 7 - (fine ? E : 0)) << 23);  // 2^(7 - E)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // words 2 i and 2 i + 1 of the operand: eight elements
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      int hi = 0, lo = 0;
      if (i < 2 * (DB / 2)) {
        float a[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          a[2 * e] = __uint_as_float(x[i][2 * w + e] << 16) * unit;
          a[2 * e + 1] = __uint_as_float(x[i][2 * w + e] & 0xffff0000u) * unit;
        }
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(a[2], a[3], hi, true);
        const kv4_f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), c = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32((a[0] - b[0]) * 16.f, (a[1] - b[1]) * 16.f, lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32((a[2] - c[0]) * 16.f, (a[3] - c[1]) * 16.f, lo, true);
      }
      q.hi[2 * i + w] = fine ? hi : 0x7f7f7f7f;  // NaN
      q.lo[2 * i + w] = fine ? lo : 0;
    }
  }
  q.hi_scale = E + 120;
  q.lo_scale = E + 116;
}

// What a wavefront holds of 32 keys: lane (j, kg) the block kg of keys j and 16 + j
struct Tile {
  u32x4 k[2], v[2];
  uint32_t ks[2], vs[2];
};

// Where the workgroup's chunk lies, and the sequence's nodes
struct Chunk {
  int b, c, chunks, L, begin, end, n0, n;
};

__device__ __forceinline__ int kv4_chunks(int L, int len) { return L > 0 ? (L + len - 1) / len : 1; }

// Chunks of all sequences on one line: as many as `target`, each of the same length (a multiple of `grain` keys) and no
// sequence in more than `splits`; a sequence without a prefix has one too, for its tree.  Every workgroup finds the length by
// itself from the sequences' lengths, a sequence to a lane.
__device__ __forceinline__ int chunk_length(int grains, int longest, const Kv4Plan &plan) {
  const int target = plan.target - plan.over;
  int len = (grains + target - 1) / target;
  const int least = (longest + plan.splits - 1) / plan.splits;
  len = len < least ? least : len;
  return (len < 1 ? 1 : len) * plan.grain;
}
__device__ __forceinline__ int grains_of(int L, const Kv4Plan &plan) { return (L + plan.grain - 1) / plan.grain; }
__device__ int chunk_length(const hb_attn_desc &d, const int32_t *__restrict__ prefix_len, const Kv4Plan &plan) {
  int grains = 0, longest = 0;
  for (int b0 = 0; b0 < d.batch; b0 += 64) {
    const int b = b0 + (threadIdx.x & 63), n = b < d.batch ? grains_of(kv4_length(d, prefix_len, b), plan) : 0;
    grains += sum_lanes(n);
    longest = max(longest, max_lanes(n));
  }
  return chunk_length(grains, longest, plan);
}

// the chunk with index `unit` on the line; false behind its end
__device__ __forceinline__ bool find_chunk(const Kv4AttnArgs &a, const Kv4Plan &plan, int unit, Chunk &c) {
  const hb_attn_desc &d = a.d;
  const int lane = threadIdx.x & 63;
  // up to 64 sequences: lengths and offsets in one go
  int L = 0, n0 = 0, n1 = 0, len;
  if (lane < d.batch) {
    L = kv4_length(d, a.prefix_len, lane);
    n0 = a.node_offset[lane];
    n1 = a.node_offset[lane + 1];
  }
  if (d.batch <= 64) {
    const int n = grains_of(L, plan);
    len = chunk_length(sum_lanes(n), max_lanes(n), plan);
  } else {
    len = chunk_length(d, a.prefix_len, plan);
  }
  int before = 0;
  for (int b0 = 0; b0 < d.batch; b0 += 64) {
    const int b = b0 + lane;
    if (b0) {
      L = b < d.batch ? kv4_length(d, a.prefix_len, b) : 0;
      n0 = b < d.batch ? a.node_offset[b] : 0;
      n1 = b < d.batch ? a.node_offset[b + 1] : 0;
    }
    const int n = b < d.batch ? kv4_chunks(L, len) : 0;
    const int up = scan_lanes(n);
    const unsigned long long behind = __ballot(before + up > unit);
    if (behind) {
      const int who = __builtin_ctzll(behind);
      c.b = b0 + who;
      c.L = __builtin_amdgcn_readlane(L, who);
      c.chunks = __builtin_amdgcn_readlane(n, who);
      c.c = unit - before - __builtin_amdgcn_readlane(up - n, who);
      c.begin = c.c * len;
      c.end = min(c.L, c.begin + len);
      c.n0 = __builtin_amdgcn_readlane(n0, who);
      c.n = __builtin_amdgcn_readlane(n1, who) - c.n0;
      c.n = c.n < 0 ? 0 : c.n > d.max_nodes_per_tree ? d.max_nodes_per_tree : c.n;
      if (c.n0 < 0 || c.n0 + c.n > d.total_nodes) c.n = 0;  // malformed offsets: touch nothing
      return true;
    }
    before += __builtin_amdgcn_readlane(up, 63);
  }
  return false;
}

// Nodes on the path of node `lane`, by doubling: a node's mask and the ancestor that it does not hold yet
__device__ __forceinline__ unsigned long long path_of(int par, int lane, int n) {
  unsigned long long path = lane < n ? 1ull << lane : 0ull;
  int up = lane < n && par < lane ? par : -1;
  for (int i = 0; i < 6 && __any(up >= 0); ++i) {
    const int from = up < 0 ? 0 : up;
    const unsigned long long p = ((unsigned long long)(uint32_t)__shfl((int)(path >> 32), from, 64) << 32) | (uint32_t)__shfl((int)path, from, 64);
    const int next = __shfl(up, from, 64);
    path |= up < 0 ? 0ull : p;
    up = up < 0 ? -1 : next;
  }
  return path;
}

template <int TPW, int DB>
struct Rows {
  QTile q[TPW];
  f32x4 o[TPW][2 * DB];  // O^T: lane (j, kg) holds d = 16 dt + 4 kg + r of row j
  f32x4 lr[TPW];         // row sums of the rounded weights (every element), which is what the values are weighed with
  float l[TPW];          // of the weights as they are, the lane's own keys: a log-sum-exp of few keys would show their rounding
  float m[TPW], ref[TPW], limit[TPW];  // reference exponent (log2 units), the same or 0 where there is none yet, largest score that keeps it
};

// softmax weights of a step's scores, after moving the reference of rows that need it
template <int TPW, int DB>
__device__ __forceinline__ void weigh(Rows<TPW, DB> &w, const f32x4 (&sc)[TPW][2], float c1, f32x8 (&p)[TPW]) {
  float lm[TPW];
  bool need = false;
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    lm[t] = fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(sc[t][0][0], sc[t][0][1]), sc[t][0][2]), sc[t][0][3]), sc[t][1][0]), sc[t][1][1]), sc[t][1][2]), sc[t][1][3]);
    need |= !(lm[t] <= w.limit[t]);
  }
  if (__any(need)) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      const float mx = group_max(lm[t]) * c1;
      const float old = w.m[t] == kNegInf ? mx : w.m[t];
      const bool grow = mx > old + kSlack;
      w.m[t] = grow ? mx : old;
      w.ref[t] = w.m[t] == kNegInf ? 0.f : w.m[t];
      w.limit[t] = w.m[t] == kNegInf ? kNegInf : (w.m[t] + kSlack) / c1;
      if (__any(grow)) {
        const float alpha = grow ? fast_exp2(old - mx) : 1.f;
        w.l[t] *= alpha;
        w.lr[t] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 2 * DB; ++dt) {
          asm volatile("" : "+v"(w.o[t][dt]));
          w.o[t][dt] *= alpha;
          asm volatile("" : "+v"(w.o[t][dt]));
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
#pragma unroll
    for (int r = 0; r < 8; ++r) p[t][r] = fast_exp2(fmaf(sc[t][r >> 2][r & 3], c1, -w.ref[t]));
    w.l[t] += ((p[t][0] + p[t][1]) + (p[t][2] + p[t][3])) + ((p[t][4] + p[t][5]) + (p[t][6] + p[t][7]));
  }
}

// O^T += V^T P^T, and the row sums (an all-ones operand), with the step's values in `lv` as [key][d] bf16.  Lane (s, kg) of
// a 16-lane group addresses 8 bytes of key 16 h + 4 kg + s / 4 at d = 16 dt + 4 (s % 4); the transposing read hands lane j the
// four keys 16 h + 4 kg + 0 .. 3 at d = 16 dt + j, the order that the score accumulators have.
template <int TPW, int DB>
__device__ __forceinline__ void accumulate(Rows<TPW, DB> &w, const unsigned char *lv, int j, int kg, const bf16x8 (&pb)[TPW]) {
  constexpr int kRow = 64 * DB;  // bytes of a key's row
  // (no vector additions, and no sum over the lane groups: every row of the product is the sum)
  const bf16x8 ones = {(__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    w.lr[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[t], w.lr[t], 0, 0, 0);
    asm volatile("" : "+v"(w.lr[t]));
  }
  const int key = 4 * kg + (j >> 2);
  const int piece = (j >> 1) & 1, half = 8 * (j & 1), x = v_swz(key) & (4 * DB - 1);
  bf16x8 av[2 * DB];
#pragma unroll
  for (int dt = 0; dt < 2 * DB; ++dt) {
    const unsigned char *p = lv + key * kRow + (((2 * dt + piece) ^ x) * 16) + half;
    bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p));
    bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p + 16 * kRow));
    av[dt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
#pragma unroll
  for (int dt = 0; dt < 2 * DB; ++dt)
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      w.o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], pb[t], w.o[t][dt], 0, 0, 0);
      asm volatile("" : "+v"(w.o[t][dt]));
    }
}

// ... the weights rounded to bf16; `fine`: and what the rounding lost, as a second product.  Over many keys the roundings of
// 2^-9 average out; a row of few keys, the nodes' own and a short prefix, would show them.
template <int TPW, int DB>
__device__ __forceinline__ void weigh_values(Rows<TPW, DB> &w, const unsigned char *lv, int j, int kg, const f32x8 (&p)[TPW], bool fine) {
  bf16x8 pb[TPW];
#pragma unroll
  for (int t = 0; t < TPW; ++t) pb[t] = __builtin_convertvector(p[t], bf16x8);
  if (fine) {
    bf16x8 rest[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) rest[t] = __builtin_convertvector(p[t] - __builtin_convertvector(pb[t], f32x8), bf16x8);
    accumulate<TPW, DB>(w, lv, j, kg, rest);
  }
  accumulate<TPW, DB>(w, lv, j, kg, pb);
}

// A key's block of 32 values, widened, into its row in LDS
template <int DB>
__device__ __forceinline__ void put_values(unsigned char *lv, int key, int kg, const u32x4 &codes, uint32_t scale) {
  constexpr int kRow = 64 * DB;
  const float s = __uint_as_float(scale << 23);
  const int x = v_swz(key) & (4 * DB - 1);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x4 y;
    y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 0));
    y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 1));
    y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 2));
    y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 3));
    *(u32x4 *)(lv + key * kRow + (((4 * kg + i) ^ x) * 16)) = y;
  }
}

template <int TPW, int DB, int W>
__global__ __launch_bounds__(64 * W, 2) void kv4_attn_kernel(Kv4AttnArgs a, Kv4Plan plan,
                                                                       const int32_t *__restrict__ block_table) {
  constexpr int D = 32 * DB, kRow = 64 * DB;
  const hb_attn_desc &d = a.d;
  // values: 32 keys to a wavefront; at the end a tile's sums of all wavefronts; then references and sums
  __shared__ __attribute__((aligned(16))) unsigned char smem[W * (kStep * kRow > 64 * 16 * 2 * DB ? kStep * kRow : 64 * 16 * 2 * DB)];
  __shared__ float s_m[W][TPW * 16], s_l[W][TPW * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, kg = lane >> 4;
  // row groups of a chunk are neighbours on one XCD (workgroup ids go round the eight): they read the same keys
  const int id = blockIdx.x, slot = id >> 3;
  const int rg = slot % plan.row_groups, unit = (slot / plan.row_groups) * 8 + (id & 7);
  const int g = unit % d.num_kv_heads, G = d.num_q_heads / d.num_kv_heads;
  Chunk ch;
  if (!find_chunk(a, plan, unit / d.num_kv_heads, ch)) return;
  const int n0 = ch.n0, n = ch.n;
  const int R = n * G, tile0 = rg * TPW;
  if (tile0 * 16 >= R) return;
  const size_t row_base = (size_t)n0 * d.num_q_heads + (size_t)g * G;
  auto row_at = [&](int row) {  // of a row of this head, among all rows
    const int node = small_div(row, G);
    return row_base + (size_t)node * d.num_q_heads + (row - node * G);
  };

  // The prefix: the codes of a step, and the pages of the step behind the one that was asked for last.  Steps past the chunk's
  // end ask for its last keys again.
  const int steps = ch.end > ch.begin ? (ch.end - ch.begin + kStep - 1) / kStep : 0;
  // (a parameter of its own, which nothing that is written can be: then its entries come by scalar loads.  By vector loads
  // each wait for one is a wait for all codes on their way)
  const int32_t *table = block_table + (size_t)ch.b * d.max_blocks_per_seq;
  const int first16 = ch.begin >> 4, last16 = (ch.end - 1) >> 4;
  size_t next[2];  // rows of a pool: where the step's two halves begin
  auto find = [&](int step) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at16 = min(first16 + 2 * step + h, last16);  // 16 keys lie in one page
      const int page = plan.page_magic ? (int)__umulhi((uint32_t)at16, plan.page_magic) : at16;
      int blk = table[page];
      blk = blk < 0 ? 0 : (blk >= d.num_blocks ? d.num_blocks - 1 : blk);
      next[h] = ((size_t)blk * d.num_kv_heads + g) * d.page_size + (at16 * 16 - page * d.page_size);
    }
  };
  auto load = [&](int step, Tile &x) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const size_t codes = next[h] * (D / 2), scales = next[h] * DB;
      if (DB == 4 || kg < DB) {
        x.k[h] = *(const u32x4 *)(a.kp.codes + codes + j * (D / 2) + kg * 16);
        x.v[h] = *(const u32x4 *)(a.vp.codes + codes + j * (D / 2) + kg * 16);
        x.ks[h] = *(a.kp.scales + scales + j * DB + kg);
        x.vs[h] = *(a.vp.scales + scales + j * DB + kg);
      }
    }
    find(step + W);
  };
  Tile x, y;
  if (DB < 4) {  // lanes without a block
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x.k[h] = y.k[h] = x.v[h] = y.v[h] = (u32x4){0u, 0u, 0u, 0u};
      x.ks[h] = y.ks[h] = x.vs[h] = y.vs[h] = 127;
    }
  }
  if (wave < steps) {
    find(wave);
    load(wave, x);
    load(wave + W, y);
  }

  Rows<TPW, DB> w;
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int row = (tile0 + t) * 16 + j;
    u32x4 x[4] = {};
    if (row < R) {
      const u32x4 *src = (const u32x4 *)a.q + row_at(row) * (D / 8);
      x[0] = src[2 * kg], x[1] = src[2 * kg + 1];
      if (DB == 4) x[2] = src[8 + 2 * kg], x[3] = src[8 + 2 * kg + 1];
    }
    split_rows<DB>(x, w.q[t]);
    w.m[t] = w.limit[t] = kNegInf;
    w.ref[t] = 0.f;
    w.l[t] = 0.f;
    w.lr[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < 2 * DB; ++dt) {
      w.o[t][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
      asm volatile("" : "+v"(w.o[t][dt]));
    }
  }
  const float c1 = d.softmax_scale * kLog2e;
  unsigned char *lv = smem + wave * kStep * kRow;

  // ---- the nodes' own keys: 32 to a wavefront, chunk 0 only ------------------------------------------
  if (ch.c == 0 && wave < (n + 31) / 32) {
    const int first = 32 * wave;
    // node `first + i` is seen by the rows whose path it lies on; lane i holds node i's
    const unsigned long long path = path_of(lane < n ? a.parent[n0 + lane] : -1, lane, n);
    const uint32_t mine = (uint32_t)(path >> first);
    f32x4 sc[TPW][2];
    bf16x8 ak[2][DB];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int node = min(first + 16 * h + j, n - 1);
      const u32x4 *src = (const u32x4 *)a.k_tree + ((size_t)(n0 + node) * d.num_kv_heads + g) * (D / 8);
#pragma unroll
      for (int ks = 0; ks < DB; ++ks) ak[h][ks] = __builtin_bit_cast(bf16x8, src[4 * ks + kg]);
    }
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      const int row = (tile0 + t) * 16 + j;
      const u32x4 *src = (const u32x4 *)a.q + row_at(min(row, R - 1)) * (D / 8);
      sc[t][0] = sc[t][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < DB; ++ks) {
        const bf16x8 qf = __builtin_bit_cast(bf16x8, src[4 * ks + kg]);
#pragma unroll
        for (int h = 0; h < 2; ++h) sc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ak[h][ks], qf, sc[t][h], 0, 0, 0);
      }
      const uint32_t allow = (uint32_t)__shfl((int)mine, row < R ? small_div(row, G) : 0, 64) >> (4 * kg);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[t][h][r] = ((allow >> (16 * h + r)) & 1u) ? sc[t][h][r] : kNegInf;
    }
    // values: a node off a row's path weighs 0, and must not make that 0 * NaN
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = 16 * h + j, node = first + key;
      const u32x4 *src = (const u32x4 *)a.v_tree + ((size_t)(n0 + min(node, n - 1)) * d.num_kv_heads + g) * (D / 8);
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        u32x4 x = src[DB * kg + i];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = node < n ? finite_or_zero_bf16x2(x[e]) : 0u;
        *(u32x4 *)(lv + key * kRow + (((DB * kg + i) ^ (v_swz(key) & (4 * DB - 1))) * 16)) = x;
      }
    }
    f32x8 p[TPW];
    weigh<TPW, DB>(w, sc, c1, p);
    weigh_values<TPW, DB>(w, lv, j, kg, p, true);
  }

  // ---- the prefix -------------------------------------------------------------------------------------
  // left: keys of the step, 32 of them unless it is the sequence's last
  auto attend = [&](auto tail, int step, Tile &x, int left) {
    constexpr bool kTail = decltype(tail)::value;
    f32x4 sc[TPW][2];
#pragma unroll
    for (int t = 0; t < TPW; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const i32x8 ak = {(int)x.k[h][0], (int)x.k[h][1], (int)x.k[h][2], (int)x.k[h][3], 0, 0, 0, 0};
        sc[t][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ak, w.q[t].lo, (f32x4){0.f, 0.f, 0.f, 0.f}, 4, 0, 0, (int)x.ks[h], 0, w.q[t].lo_scale);
        sc[t][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ak, w.q[t].hi, sc[t][h], 4, 0, 0, (int)x.ks[h], 0, w.q[t].hi_scale);
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 c = x.v[h];
      uint32_t s = x.vs[h];
      if (kTail) {  // whatever lies behind the end: its weight is 0, and must not make that 0 * NaN
        const bool there = 16 * h + j < left;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = there ? c[e] : 0u;
        s = there ? s : 127u;
      }
      if (DB == 4 || kg < DB) put_values<DB>(lv, 16 * h + j, kg, c, s);
    }
    if (kTail) {
#pragma unroll
      for (int t = 0; t < TPW; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[t][h][r] = 16 * h + 4 * kg + r < left ? sc[t][h][r] : kNegInf;
    } else {
      load(step + 2 * W, x);
    }
    f32x8 p[TPW];
    weigh<TPW, DB>(w, sc, c1, p);
    weigh_values<TPW, DB>(w, lv, j, kg, p, kTail);
  };
  if (wave < steps) {
    const int whole = (ch.end - ch.begin) / kStep;
    int step = wave;
    for (; step + W < whole; step += 2 * W) {
      attend(std::false_type(), step, x, kStep);
      attend(std::false_type(), step + W, y, kStep);
    }
    if (step < whole) {
      attend(std::false_type(), step, x, kStep);
      step += W;
      x = y;
    }
    if (step < steps) attend(std::true_type(), step, x, ch.end - ch.begin - step * kStep);
  }

  // ---- join the wavefronts' results --------------------------------------------------------------------
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const float l = group_sum(w.l[t]);
    w.l[t] = w.lr[t][0] > 0.f ? l / w.lr[t][0] : 1.f;  // values weighed as the sum that they are divided by
    if (kg == 0) {
      s_m[wave][16 * t + j] = w.m[t];
      s_l[wave][16 * t + j] = l;
    }
  }
  __syncthreads();  // also: everybody is done with the values in LDS
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmaxf(m, s_m[i][16 * t + j]);
    const float ref = m == kNegInf ? 0.f : m;
#pragma unroll
    for (int i = 0; i < W; ++i) l += s_l[i][16 * t + j] * fast_exp2(s_m[i][16 * t + j] - ref);
    const float mine = fast_exp2(w.m[t] - ref) * w.l[t];
    f32x4 *all = (f32x4 *)smem;  // [dt][wave][lane]
#pragma unroll
    for (int dt = 0; dt < 2 * DB; ++dt) all[(dt * W + wave) * 64 + lane] = w.o[t][dt] * mine;
    __syncthreads();
    const int row = (tile0 + t) * 16 + j;
    const size_t rr = row < R ? row_at(row) : 0;
    for (int dt = wave; dt < 2 * DB; dt += W) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < W; ++i) o += all[(dt * W + i) * 64 + lane];
      if (row < R) {
        if (ch.chunks == 1) {
          const float inv = 1.f / l;
          *(u32x2 *)((bf16_t *)a.out + rr * D + 16 * dt + 4 * kg) = (u32x2){pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
        } else {
          *(f32x4 *)(a.part_o + (rr * plan.splits + ch.c) * D + 16 * dt + 4 * kg) = o;
        }
      }
    }
    if (wave == 0 && kg == 0 && row < R) {
      if (ch.chunks > 1) {
        *(kv4_f32x2 *)(a.part_ml + (rr * plan.splits + ch.c) * 2) = (kv4_f32x2){m, l};
      } else if (a.lse) {
        a.lse[rr] = (m + log2f(l)) * kLn2;
      }
    }
    if (t + 1 < TPW) __syncthreads();
  }
}

// Rows of sequences that were cut: the chunks' results joined (log2 units).  A row's threads hold four elements each; results
// are asked for eight chunks at a time.
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4AttnArgs a, Kv4Plan plan) {
  const int D = a.d.head_dim, tpr = D / 4;
  const int len = chunk_length(a.d, a.prefix_len, plan);
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(gid / tpr), piece = (int)(gid - (long)row * tpr);
  if (row >= a.d.total_nodes * a.d.num_q_heads) return;
  const int node = row / a.d.num_q_heads, b = kv4_sequence(a.node_offset, a.d.batch, node);
  const int first = a.node_offset[b], n = min(a.node_offset[b + 1] - first, a.d.max_nodes_per_tree);
  if (node < first || node >= first + n || first + n > a.d.total_nodes) return;
  const int chunks = kv4_chunks(kv4_length(a.d, a.prefix_len, b), len);
  if (chunks == 1) return;
  const kv4_f32x2 *ml = (const kv4_f32x2 *)a.part_ml + (size_t)row * plan.splits;
  const f32x4 *po = (const f32x4 *)a.part_o + (size_t)row * plan.splits * tpr + piece;
  float m = kNegInf, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int c0 = 0; c0 < chunks; c0 += 8) {
    kv4_f32x2 x[8];
    f32x4 y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = min(c0 + i, chunks - 1);
      x[i] = ml[c];
      y[i] = po[(size_t)c * tpr];
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i][0]);
    const float ref = top == kNegInf ? 0.f : top, corr = fast_exp2(m - ref);
    m = top;
    l *= corr;
    o *= corr;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (c0 + i < chunks) {
        const float w = fast_exp2(x[i][0] - ref);
        l = fmaf(x[i][1], w, l);
        o += y[i] * w;
      }
    }
  }
  const float inv = 1.f / l;
  *(u32x2 *)((bf16_t *)a.out + (size_t)row * D + piece * 4) = (u32x2){pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  if (a.lse && piece == 0) a.lse[row] = (m + log2f(l)) * kLn2;
}

template <int TPW, int DB, int W>
hipError_t launch(const Kv4AttnArgs &a, const Kv4Plan &plan, hipStream_t s) {
  const long units = ((long)plan.target + a.d.batch) * a.d.num_kv_heads;  // chunks on the line, at most
  kv4_attn_kernel<TPW, DB, W><<<(unsigned)((units + 7) / 8 * 8 * plan.row_groups), 64 * W, 0, s>>>(a, plan, a.block_table);
  return hipGetLastError();
}

}  // namespace

bool kv4_attn_supports(const hb_attn_desc &d) {
  return d.dtype == HB_BF16 && (d.head_dim == 64 || d.head_dim == 128) && d.page_size % 16 == 0 && d.page_size <= 1024 &&
         d.softmax_scale > 0.f && d.softmax_scale < 1e30f && d.num_q_heads / d.num_kv_heads <= 512;
}

static int tiles_of(const hb_attn_desc &d) { return (d.num_q_heads / d.num_kv_heads * d.max_nodes_per_tree + 15) / 16; }

// Chunks are planned for some 512 workgroups
void kv4_attn_plan(const hb_attn_desc &d, int64_t span, Kv4Plan *plan) {
  const int tiles = tiles_of(d), tpw = tiles > 1 ? 2 : 1;
  plan->row_groups = (tiles + tpw - 1) / tpw;
  plan->grain = kWaves * kStep;
  int64_t target = 512 / ((int64_t)d.num_kv_heads * plan->row_groups);
  target = target < 1 ? 1 : target;
  int64_t splits = d.num_splits ? d.num_splits : target;
  const int64_t most = (span + plan->grain - 1) / plan->grain;
  splits = splits > most ? most : splits;
  splits = splits < 1 ? 1 : splits > 1024 ? 1024 : splits;
  plan->target = (int32_t)(d.num_splits ? (int64_t)d.num_splits * d.batch > 1 << 16 ? 1 << 16 : d.num_splits * d.batch : target);
  plan->target = plan->target < 1 ? 1 : plan->target;
  plan->over = !d.num_splits && plan->target > 2 * d.batch ? d.batch : 0;
  plan->splits = (int32_t)splits;
  const int page16 = d.page_size / 16;
  plan->page_magic = page16 == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + page16 - 1) / page16);
}

hipError_t launch_kv4_attn(const Kv4AttnArgs &a, const Kv4Plan &plan, hipStream_t s) {
  const bool wide = tiles_of(a.d) > 1;
  hipError_t e;
  if (a.d.head_dim == 128) e = wide ? launch<2, 4, kWaves>(a, plan, s) : launch<1, 4, kWaves>(a, plan, s);
  else e = wide ? launch<2, 2, kWaves>(a, plan, s) : launch<1, 2, kWaves>(a, plan, s);
  if (e != hipSuccess || plan.splits == 1) return e;
  const long threads = (long)a.d.total_nodes * a.d.num_q_heads * (a.d.head_dim / 4);
  kv4_join_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a, plan);
  return hipGetLastError();
}

}  // namespace hb
