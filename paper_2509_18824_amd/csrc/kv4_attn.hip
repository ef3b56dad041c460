// Attention over the 4-bit cache on the matrix cores of gfx950 (heads of 64 and 128, pages of a multiple of 16).
//
// Formulation (transposed, so that no score crosses lanes on its way into the second product):
//   S^T = K Q^T     v_mfma_f32_16x16x32_bf16: A = 16 cached keys (16 keys x 32 d), B = 16 query rows
//   O^T = V^T P^T   the same: A = V^T (16 d x 32 keys), B = P^T
// A block of 32 cached numbers is widened to bf16 by one instruction for two of them, scale included, and exactly: scores are
// those of a bf16 cache.  (The matrix cores also take the codes as they are, against 8-bit pieces of the queries: two pieces
// of a 128-long product cost the same 64 clocks as the four bf16 products, and what the hardware drops of such a sum, 5e-6
// of a score's spread, shows in the log-sum-exp.)
// Probabilities are rounded to bf16 for the second product, sums are kept in 32 bits.
//
// A wavefront takes 32 keys at a time of its own and TPW tiles of 16 query rows (row = node * G + head of the group); the
// wavefronts of a workgroup take turns on the steps of a chunk of the prefix and join their results in LDS at its end.  Nobody
// waits for anybody in between: a step's codes go from memory to registers two steps ahead, keys from there to the matrix core,
// values through 8 KB of LDS of the wavefront's own, where a transposing read turns them.
//
// Chunks are cut on the device from the lengths (find_piece below), so that about as many workgroups start as the host planned
// for, whatever the lengths are: one to a CU, of eight wavefronts of up to 256 registers each.
//
// What bounds it, single tokens: memory.  16 of them over 16384 to 32768 positions, 28/4 heads of 128, 214 MB: 50 us, the join
// with 5 of them included, 4.3 TB/s (a large copy runs at 5.1); one over 2048, 1.1 MB: 12 us, the join with 3.5 of them included, the round trips to lengths,
// pages, codes and back and the start of two launches.  16 chains of 8 nodes (56 rows) over 1024 to 4096: 24 us, join 5, a
// few steps to a wavefront between the same round trips.  Two workgroups of four wavefronts to a CU: 53, 12.6 and 25.4 us.
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
typedef unsigned int swap2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;  // keys
constexpr int kWaves = 8;    // of a workgroup, one on a CU
constexpr int kSharing = 4;  // of one whose wavefronts share keys, two on a CU
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kMostSum = 4096.f;  // of eight weights against their row's reference
constexpr float kSlack = 8.f;       // log2 units: a largest score that is no further above the reference leaves it where it is
constexpr float kFar = 0x1p27f;     // log2 units: half a unit in the last place of a larger score is more than eight
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

// A row as operand of the scores' products: lane (j, kg) of the i-th holds d = 32 kg + 8 i + 0 .. 7 of row j, which is how a cached
// key's block kg lies.  (Heads of 64: lanes without a block hold zeros.)
template <int DB>
__device__ __forceinline__ void row_operand(const u32x4 *row, bool there, int kg, bf16x8 (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x4 y = {0u, 0u, 0u, 0u};
    if (there && (DB == 4 || kg < DB)) y = row[4 * kg + i];
    x[i] = __builtin_bit_cast(bf16x8, y);
  }
}

// a block of 32 codes as the same operand
__device__ __forceinline__ u32x4 widen8(uint32_t codes, float scale) {
  u32x4 y;
  y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return y;
}
__device__ __forceinline__ void widen_key(const u32x4 &codes, uint32_t scale, bf16x8 (&k)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) k[i] = __builtin_bit_cast(bf16x8, widen8(codes[i], __uint_as_float(scale << 23)));
}

// What a wavefront holds of 32 keys: lane (j, kg) the block kg of keys j and 16 + j
struct Tile {
  u32x4 k[2], v[2];
  uint32_t ks[2], vs[2];
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((kv4_f32x2){a, b}, bf16x2));
}

__device__ __forceinline__ void store4(bf16_t *p, f32x4 v) { *(u32x2 *)p = (u32x2){pack2(v[0], v[1]), pack2(v[2], v[3])}; }
__device__ __forceinline__ void store4(float *p, f32x4 v) { *(f32x4 *)p = v; }
// sum / weight of a row, a mean of values: where rounding takes it past the largest number of float32 it is that number.  (bf16's
// largest is further from there than roundings go.)
__device__ __forceinline__ f32x4 mean_of(bf16_t, f32x4 sum, float weight) { return sum * (1.f / weight); }
__device__ __forceinline__ f32x4 mean_of(float, f32x4 sum, float weight) {
  f32x4 v = sum * (1.f / weight);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (fabsf(v[e]) == -kNegInf && fabsf(sum[e]) != -kNegInf) v[e] = copysignf(__FLT_MAX__, v[e]);
  return v;
}

// Pages of a chunk's keys, 64 times 16 keys to the registers of a wavefront (lane l: the l-th 16) and the next 64 on their way.
// Asked for one by one, by scalar loads, they would be waited for with the LDS reads of every step.
struct Pages {
  const int32_t *table;
  int blocks, last16, first16, now, ahead;
  uint32_t magic;

  __device__ __forceinline__ int ask(int from) const {
    const int at16 = min(from + (int)(threadIdx.x & 63), last16);
    return table[magic ? (int)__umulhi((uint32_t)at16, magic) : at16];
  }
  __device__ __forceinline__ void begin(const hb_attn_desc &d, const int32_t *row, int at16, int last, uint32_t page_magic) {
    table = row;
    blocks = d.num_blocks;
    last16 = last;
    first16 = at16;
    magic = page_magic;
    now = ask(at16);
    ahead = ask(at16 + 64);
    asm volatile("" : "+v"(now));  // waited for here: where it is used next would be a wait for the codes asked for in between
  }
  // where in a pool the rows of the keys 16 at16 .. 16 at16 + 15 of head g begin; at16 never goes back by more than it has come
  // on since the last 64 were left (a chunk's last keys, asked for again, are in the 64 that are there)
  __device__ __forceinline__ size_t row(const hb_attn_desc &d, int at16, int g) {
    at16 = min(at16, last16);
    if (at16 - first16 >= 64) {  // uniform
      first16 += 64;
      now = ahead;
      asm volatile("" : "+v"(now));
      ahead = ask(first16 + 64);
    }
    int blk = __builtin_amdgcn_readlane(now, at16 - first16);
    blk = blk < 0 ? 0 : (blk >= blocks ? blocks - 1 : blk);
    const int page = magic ? (int)__umulhi((uint32_t)at16, magic) : at16;
    return ((size_t)blk * d.num_kv_heads + g) * d.page_size + (at16 * 16 - page * d.page_size);
  }
};

// What a workgroup works on: row group rg of the keys [begin, end) of head g of sequence b (chunk c of `chunks`), and the
// sequence's nodes
struct Piece {
  int b, c, chunks, g, rg, groups, L, begin, end, n0, n;
};

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }
// chunks of a sequence of `grains` grains, len grains long
__device__ __forceinline__ int chunks_of(int grains, int len) { return grains > 0 ? div_up(grains, len) : 1; }
__device__ __forceinline__ int grains_of(int L, const Kv4Plan &plan) { return (L + (1 << plan.grain_shift) - 1) >> plan.grain_shift; }
__device__ __forceinline__ int nodes_of(const hb_attn_desc &d, int n0, int n1) {
  const int n = n1 - n0 < 0 ? 0 : n1 - n0 > d.max_nodes_per_tree ? d.max_nodes_per_tree : n1 - n0;
  return n0 < 0 || n0 + n > d.total_nodes ? 0 : n;  // malformed offsets: touch nothing
}
// row groups of a sequence with n nodes
__device__ __forceinline__ int groups_of(int n, const Kv4Plan &plan) {
  return (n * plan.heads + (1 << plan.group_shift) - 1) >> plan.group_shift;
}

// The workgroups' pieces.  Every sequence is cut into chunks of one length, a multiple of a grain, the shortest with which
// about `target` workgroups a kv head (a chunk has one for each of the sequence's row groups) and no sequence in more than
// `splits` chunks come out; a sequence without a prefix has one chunk, for its tree.  Every workgroup finds this out from the
// lengths, a sequence to a lane, and then which piece is its own.  Row groups of a chunk are neighbours, so are the heads,
// and neighbours are on one XCD (workgroup ids go round the eight): they read the same keys, or the same lines of scales.
// What is left over without a piece are the last ids: holes in between would leave the CUs of one shader engine idle.
__device__ __forceinline__ bool find_piece(const Kv4AttnArgs &a, const Kv4Plan &plan, Piece &c) {
  const hb_attn_desc &d = a.d;
  const int lane = threadIdx.x & 63;
  int L = 0, n0 = 0, n1 = 0;  // of sequence b0 + lane
  auto ask = [&](int b) {
    const bool there = b < d.batch;
    L = there ? kv4_length(d, a.prefix_len, b) : 0;
    n0 = there ? a.node_offset[b] : 0;
    n1 = there ? a.node_offset[b + 1] : 0;
  };
  int work = 0, longest = 0;  // grains, as often as there are row groups; of a sequence
  for (int b0 = 0; b0 < d.batch; b0 += 64) {
    ask(b0 + lane);
    const int n = grains_of(L, plan);
    work += sum_lanes(n * groups_of(nodes_of(d, n0, n1), plan));
    longest = max(longest, max_lanes(n));
  }
  int len = max(max(div_up(work, plan.target), div_up(longest, plan.splits)), 1);  // in grains
  int total = 0;  // workgroups of a kv head
  for (;;) {
    total = 0;
    for (int b0 = 0; b0 < d.batch; b0 += 64) {
      if (d.batch > 64) ask(b0 + lane);
      total += sum_lanes(chunks_of(grains_of(L, plan), len) * groups_of(nodes_of(d, n0, n1), plan));
    }
    // short last chunks make more of them than were asked for: longer ones, unless there are too many sequences for that
    if (total <= plan.target || len >= longest || !plan.fit) break;
    len += (len + 15) / 16;
  }
  const int each = (total * d.num_kv_heads + 7) / 8;  // of an XCD
  const int id = blockIdx.x, slot = id >> 3, index = (id & 7) * each + slot;
  if (a.cut && id == 0 && threadIdx.x == 0) *a.cut = len;  // for the launch that joins the chunks
  if (slot >= each || index >= total * d.num_kv_heads) return false;
  int before = 0;
  const int at = index / d.num_kv_heads;
  for (int b0 = 0; b0 < d.batch; b0 += 64) {
    if (d.batch > 64) ask(b0 + lane);
    const int chunks = chunks_of(grains_of(L, plan), len), groups = groups_of(nodes_of(d, n0, n1), plan);
    const int up = scan_lanes(chunks * groups);
    const unsigned long long behind = __ballot(before + up > at);
    if (behind) {
      const int who = __builtin_ctzll(behind);
      c.b = b0 + who;
      c.L = __builtin_amdgcn_readlane(L, who);
      c.chunks = __builtin_amdgcn_readlane(chunks, who);
      c.groups = __builtin_amdgcn_readlane(groups, who);
      int rest = index - (before + __builtin_amdgcn_readlane(up - chunks * groups, who)) * d.num_kv_heads;
      c.rg = rest % c.groups;
      rest /= c.groups;
      c.g = rest % d.num_kv_heads;
      c.c = rest / d.num_kv_heads;
      c.begin = (c.c * len) << plan.grain_shift;
      c.end = min(c.L, c.begin + (len << plan.grain_shift));
      c.n0 = __builtin_amdgcn_readlane(n0, who);
      c.n = nodes_of(d, c.n0, __builtin_amdgcn_readlane(n1, who));
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

// Values of nodes that are not finite count as 0 in the products, where they would reach every row.  Those that see them get them
// here, in what this lane has written: the elements d .. d + 3 of a row, `seen` its path; v: the first node's values.
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
template <typename T, typename O>
__device__ __forceinline__ void add_not_finite(const T *v, size_t stride, unsigned long long seen, int d, O *out) {
#pragma nounroll
  for (; seen; seen &= seen - 1) {
    const T *x = v + __builtin_ctzll(seen) * stride + d;
#pragma nounroll
    for (int e = 0; e < 4; ++e)
      if (const float y = load_f32(x + e); not_finite(y)) store_f32(out + e, load_f32(out + e) + y);
  }
}
// the path of node `node`, asked for by every lane
__device__ __forceinline__ unsigned long long path_at(unsigned long long path, int node) {
  return ((unsigned long long)(uint32_t)__shfl((int)(path >> 32), node, 64) << 32) | (uint32_t)__shfl((int)path, node, 64);
}

template <int TPW, int DB>
struct Rows {
  bf16x8 q[TPW][4];
  f32x4 o[TPW][2 * DB];  // O^T: lane (j, kg) holds d = 16 dt + 4 kg + r of row j
  f32x4 lr[TPW];         // row sums of the rounded weights (every element), which is what the values are weighed with
  float l[TPW];          // of the weights as they are, the lane's own keys: a log-sum-exp of few keys would show their rounding
  float m[TPW], ref[TPW], limit[TPW];  // reference exponent (log2 units), the same or 0 where there is none yet, largest sum of weights that keeps it
};

// ---- float32 ----------------------------------------------------------------------------------------
// Queries, weights and the nodes' own keys and values are taken as three bf16 pieces; cached keys are widened to bf16, which is
// exact.  A product of two such numbers keeps the six products of pieces that matter to 2^-23, the smallest first.
__device__ __forceinline__ f32x8 load_f32x8(const float *at) {
  const f32x4 a = *(const f32x4 *)at, b = *(const f32x4 *)(at + 4);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x8 within(f32x8 x, float most) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e], -most, most);
  return x;
}
// the first piece of a number up to the largest
__device__ __forceinline__ bf16x8 cut_of(const f32x8 &x) {
  u32x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = kv4_pack_cut(x[2 * e], x[2 * e + 1]);
  return __builtin_bit_cast(bf16x8, y);
}
__device__ __forceinline__ f32x8 rest_of(f32x8 x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] -= kv4_cut(x[e]);
  return x;
}
// of a softmax weight, which is far from the largest number: the first is rounded too
__device__ __forceinline__ void pieces_of(f32x8 x, bf16x8 (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = __builtin_convertvector(x, bf16x8);
    x -= __builtin_convertvector(p[i], f32x8);
  }
}
// Lane (j, kg) of the i-th operand of a row: d = 32 kg + 8 i + 0 .. 7, as a cached key's block lies.  An infinity gives NaN in its
// products.  INF: its first two pieces are finite, and the third, an infinity, meets the other factor's first piece alone.
template <int DB, bool INF = false>
__device__ __forceinline__ void row_pieces(const float *row, bool there, int kg, bf16x8 (&p)[3][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x8 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (there && (DB == 4 || kg < DB)) x = load_f32x8(row + 32 * kg + 8 * i);
    p[0][i] = cut_of(INF ? within(x, __FLT_MAX__) : x);
    x -= __builtin_convertvector(p[0][i], f32x8);
    p[1][i] = __builtin_convertvector(INF ? within(x, 0x1p120f) : x, bf16x8);
    x -= __builtin_convertvector(p[1][i], f32x8);
    p[2][i] = __builtin_convertvector(x, bf16x8);
  }
}
// Scores of 16 keys
template <int TPW>
__device__ __forceinline__ void score_tiles(const bf16x8 (&k)[4], const bf16x8 (&q)[TPW][4], int h, f32x4 (&sc)[TPW][2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int t = 0; t < TPW; ++t)
      sc[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i], q[t][i], i ? sc[t][h] : (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
}

// Softmax weights of a step's scores.  A row's reference is the largest score of the first step it sees, and moves when the
// weights of a lane's eight keys against it sum to more than 2^12 (or to no number): then one of them is 2^9 or more, and
// the reference becomes the row's largest score of the step.  Their sum is needed anyway, so that the common case takes no
// maximum at all.  F32: it lies a factor of two above that score, so that the nodes' weights, rounded as they are, stay below one and
// the largest of float32 among the nodes' values does not overflow.  NODES: their second 32 as well, so it moves for any larger score.
template <bool F32, bool NODES = false, int TPW, int DB>
__device__ __forceinline__ void weigh(Rows<TPW, DB> &w, f32x4 (&sc)[TPW][2], float c1, f32x8 (&p)[TPW]) {
#pragma clang fp contract(off)
  float sum[TPW];
  auto weights = [&](int t, float scale) {
#pragma unroll
    for (int r = 0; r < 8; ++r) p[t][r] = fast_exp2(fmaf(sc[t][r >> 2][r & 3], scale, -w.ref[t]));
    sum[t] = ((p[t][0] + p[t][1]) + (p[t][2] + p[t][3])) + ((p[t][4] + p[t][5]) + (p[t][6] + p[t][7]));
  };
#pragma unroll
  for (int t = 0; t < TPW; ++t) weights(t, c1);
  bool need = NODES;
#pragma unroll
  for (int t = 0; t < TPW; ++t) need |= !(sum[t] <= w.limit[t]);
  if (__any(need)) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      const float lm = fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(sc[t][0][0], sc[t][0][1]), sc[t][0][2]), sc[t][0][3]), sc[t][1][0]), sc[t][1][1]), sc[t][1][2]), sc[t][1][3]);
      const float mx = group_max(lm) * c1 + (F32 ? 1.f : 0.f);  // c1 > 0
      const float old = w.m[t] == kNegInf ? mx : w.m[t];
      const bool grow = mx > old + (NODES ? 0.f : kSlack);
      w.m[t] = grow ? mx : old;
      w.ref[t] = w.m[t] == kNegInf ? 0.f : w.m[t];
      const bool far = fabsf(w.ref[t]) > kFar;
      w.limit[t] = w.m[t] == kNegInf || far ? -1.f : kMostSum;
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
      if (__any(far)) {
#pragma unroll
        for (int r = 0; r < 8; ++r) sc[t][r >> 2][r & 3] *= far ? c1 : 1.f;
      }
      weights(t, far ? 1.f : c1);
    }
  }
#pragma unroll
  for (int t = 0; t < TPW; ++t) w.l[t] += sum[t];
}

// V^T of a step, from its values in LDS as [key][d] bf16.  Lane (s, kg) of a 16-lane group addresses 8 bytes of key
// 16 h + 4 kg + s / 4 at d = 16 dt + 4 (s % 4); the transposing read hands lane j the four keys 16 h + 4 kg + 0 .. 3 at
// d = 16 dt + j, the order that the score accumulators have.
template <int DB>
__device__ __forceinline__ void read_values(const unsigned char *lv, int j, int kg, bf16x8 (&av)[2 * DB]) {
  constexpr int kRow = 64 * DB;  // bytes of a key's row
  const int key = 4 * kg + (j >> 2);
  const int piece = (j >> 1) & 1, half = 8 * (j & 1), x = v_swz(key) & (4 * DB - 1);
#pragma unroll
  for (int dt = 0; dt < 2 * DB; ++dt) {
    const unsigned char *p = lv + key * kRow + (((2 * dt + piece) ^ x) * 16) + half;
    bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p));
    bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(p + 16 * kRow));
    av[dt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// O^T += V^T P^T, and the row sums (an all-ones operand: no vector additions, and no sum over the lane groups)
template <int TPW, int DB>
__device__ __forceinline__ void accumulate(Rows<TPW, DB> &w, const bf16x8 (&av)[2 * DB], const bf16x8 (&pb)[TPW]) {
  const bf16x8 ones = {(__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    w.lr[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[t], w.lr[t], 0, 0, 0);
    asm volatile("" : "+v"(w.lr[t]));
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
  bf16x8 pb[TPW], av[2 * DB];
#pragma unroll
  for (int t = 0; t < TPW; ++t) pb[t] = __builtin_convertvector(p[t], bf16x8);
  read_values<DB>(lv, j, kg, av);
  if (fine) {
    bf16x8 rest[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) rest[t] = __builtin_convertvector(p[t] - __builtin_convertvector(pb[t], f32x8), bf16x8);
    accumulate<TPW, DB>(w, av, rest);
  }
  accumulate<TPW, DB>(w, av, pb);
}

// A key's block of 32 numbers, widened, into its row in LDS
template <int DB>
__device__ __forceinline__ void put_block(unsigned char *lv, int key, int kg, const u32x4 &codes, uint32_t scale) {
  constexpr int kRow = 64 * DB;
  const int x = v_swz(key) & (4 * DB - 1);
#pragma unroll
  for (int i = 0; i < 4; ++i) *(u32x4 *)(lv + key * kRow + (((4 * kg + i) ^ x) * 16)) = widen8(codes[i], __uint_as_float(scale << 23));
}

template <typename T, int TPW, int DB, int W>
__global__ __launch_bounds__(64 * W, 2) void kv4_attn_kernel(Kv4AttnArgs a, Kv4Plan plan) {
  constexpr int D = 32 * DB, kRow = 64 * DB;
  constexpr bool F32 = sizeof(T) == 4;
  static_assert(!F32 || TPW == 1, "float32: one tile of rows");
  const hb_attn_desc &d = a.d;
  // values: 32 keys to a wavefront; at the end a tile's sums of all wavefronts; then references and sums
  __shared__ __attribute__((aligned(16))) unsigned char smem[W * (kStep * kRow > 64 * 16 * 2 * DB ? kStep * kRow : 64 * 16 * 2 * DB)];
  __shared__ float s_m[W][TPW * 16], s_l[W][TPW * 16];
  __shared__ int s_odd[W];  // whether a wavefront's nodes have values that are not finite
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, kg = lane >> 4;
  Piece ch;
  if (!find_piece(a, plan, ch)) return;
  const int g = ch.g, G = plan.heads, n0 = ch.n0, n = ch.n, R = n * G, tile0 = ch.rg * TPW;
  const size_t row_base = (size_t)n0 * d.num_q_heads + (size_t)g * G;
  auto row_at = [&](int row) {  // of a row of this head, among all rows
    const int node = small_div(row, G);
    return row_base + (size_t)node * d.num_q_heads + (row - node * G);
  };

  // The prefix: the codes of a step, and the pages of the step behind the one that was asked for last.  Steps past the chunk's
  // end ask for its last keys again.
  const int steps = ch.end > ch.begin ? (ch.end - ch.begin + kStep - 1) / kStep : 0;
  const int first16 = ch.begin >> 4, last16 = (ch.end - 1) >> 4;
  Pages pages;
  size_t next[2];  // where the step's two halves begin
  auto find = [&](int step) {
#pragma unroll
    for (int h = 0; h < 2; ++h) next[h] = pages.row(d, first16 + 2 * step + h, g);
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
    pages.begin(d, a.block_table + (size_t)ch.b * d.max_blocks_per_seq, first16, last16, plan.page_magic);
    find(wave);
    load(wave, x);
    load(wave + W, y);
  }

  Rows<TPW, DB> w;
  bf16x8 q32[3][4];  // float32: the rows' pieces
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int row = (tile0 + t) * 16 + j;
    if constexpr (F32) {
      row_pieces<DB>((const float *)a.q + row_at(min(row, R - 1)) * D, row < R, kg, q32);
    } else {
      row_operand<DB>((const u32x4 *)a.q + row_at(min(row, R - 1)) * (D / 8), row < R, kg, w.q[t]);
    }
    w.m[t] = kNegInf;
    w.ref[t] = 0.f;
    w.limit[t] = -1.f;
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
  if (lane == 0) s_odd[wave] = 0;

  // ---- the nodes' own keys: 32 to a wavefront, chunk 0 only ------------------------------------------
  if (ch.c == 0 && wave < (n + 31) / 32) {
    const int first = 32 * wave;
    bool odd = false;
    // node `first + i` is seen by the rows whose path it lies on; lane i holds node i's
    const unsigned long long path = path_of(lane < n ? a.parent[n0 + lane] : -1, lane, n);
    const uint32_t mine = (uint32_t)(path >> first);
    f32x4 sc[TPW][2];
    auto mask = [&](int t) {
      const int row = (tile0 + t) * 16 + j;
      const uint32_t allow = (uint32_t)__shfl((int)mine, row < R ? small_div(row, G) : 0, 64) >> (4 * kg);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[t][h][r] = ((allow >> (16 * h + r)) & 1u) ? sc[t][h][r] : kNegInf;
    };
    auto piece_at = [&](int key, int piece) { return (u32x4 *)(lv + key * kRow + ((piece ^ (v_swz(key) & (4 * DB - 1))) * 16)); };
    f32x8 p[TPW];
    if constexpr (F32) {
      auto scores = [&](auto inf) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 k[3][4];
          row_pieces<DB, decltype(inf)::value>((const float *)a.k_tree + ((size_t)(n0 + min(first + 16 * h + j, n - 1)) * d.num_kv_heads + g) * D, true, kg, k);
          sc[0][h] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int sum = 2; sum >= 0; --sum)
#pragma unroll
            for (int b = 0; b <= sum; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) sc[0][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[b][i], q32[sum - b][i], sc[0][h], 0, 0, 0);
        }
        mask(0);
      };
      scores(std::false_type());
      const f32x4 both = sc[0][0] + sc[0][1];
      if (const float sum = (both[0] + both[1]) + (both[2] + both[3]); __any(sum != sum)) scores(std::true_type());  // an infinity in a key, or NaN
      weigh<F32>(w, sc, c1, p);
      bf16x8 weight[3];
      pieces_of(p[0], weight);
      f32x8 x[2][DB];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int node = first + 16 * h + j;
        const float *row = (const float *)a.v_tree + ((size_t)(n0 + min(node, n - 1)) * d.num_kv_heads + g) * D;
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          x[h][i] = load_f32x8(row + (DB * kg + i) * 8);
          // a node off a row's path weighs 0, and must not make that 0 * NaN
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float y = x[h][i][e];
            odd |= not_finite(y);
            x[h][i][e] = node < n && !not_finite(y) ? y : 0.f;
          }
        }
      }
      // the values a piece at a time, by a loop: it is done once, and what costs then is to bring its instructions
#pragma nounroll
      for (int b = 0; b < 3; ++b) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < DB; ++i) {
            *piece_at(16 * h + j, DB * kg + i) = __builtin_bit_cast(u32x4, cut_of(x[h][i]));  // (all three: 24 bits)
            x[h][i] = rest_of(x[h][i]);
          }
        bf16x8 av[2 * DB];
        read_values<DB>(lv, j, kg, av);
        // (the sums of the weights are those that the largest pieces of the values are weighed with)
        const f32x4 lr = w.lr[0];
#pragma unroll
        for (int e = 2; e >= 0; --e) {
          if (e > 2 - b) continue;  // uniform
          const bf16x8 one[1] = {weight[e]};
          accumulate<TPW, DB>(w, av, one);
        }
        if (b) w.lr[0] = lr;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 k[4];
        row_operand<DB>((const u32x4 *)a.k_tree + ((size_t)(n0 + min(first + 16 * h + j, n - 1)) * d.num_kv_heads + g) * (D / 8), true, kg, k);
        score_tiles<TPW>(k, w.q, h, sc);
      }
#pragma unroll
      for (int t = 0; t < TPW; ++t) mask(t);
      // values: a node off a row's path weighs 0, and must not make that 0 * NaN
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = 16 * h + j, node = first + key;
        const u32x4 *src = (const u32x4 *)a.v_tree + ((size_t)(n0 + min(node, n - 1)) * d.num_kv_heads + g) * (D / 8);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          u32x4 x = src[DB * kg + i];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = finite_or_zero_bf16x2(x[e]);
            odd |= y != x[e];
            x[e] = node < n ? y : 0u;
          }
          *piece_at(key, DB * kg + i) = x;
        }
      }
      weigh<F32>(w, sc, c1, p);
      weigh_values<TPW, DB>(w, lv, j, kg, p, true);
    }
    if (odd) s_odd[wave] = 1;
  }

  // ---- the prefix -------------------------------------------------------------------------------------
  // left: keys of the step, 32 of them unless it is the sequence's last
  auto attend = [&](auto tail, int step, Tile &x, int left) {
    constexpr bool kTail = decltype(tail)::value;
    f32x4 sc[TPW][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 k[4];
      widen_key(x.k[h], x.ks[h], k);
      if constexpr (F32) {
        sc[0][h] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 2; b >= 0; --b)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[0][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i], q32[b][i], sc[0][h], 0, 0, 0);
      } else {
        score_tiles<TPW>(k, w.q, h, sc);
      }
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
      if (DB == 4 || kg < DB) put_block<DB>(lv, 16 * h + j, kg, c, s);
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
    weigh<F32>(w, sc, c1, p);
    if constexpr (F32) {
      bf16x8 weight[3], av[2 * DB];
      pieces_of(p[0], weight);
      read_values<DB>(lv, j, kg, av);
#pragma unroll
      for (int b = 2; b >= 0; --b) {
        const bf16x8 one[1] = {weight[b]};
        accumulate<TPW, DB>(w, av, one);
      }
    } else {
      weigh_values<TPW, DB>(w, lv, j, kg, p, kTail);
    }
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
          store4((T *)a.out + rr * D + 16 * dt + 4 * kg, mean_of(T(), o, l));
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
  if (__builtin_expect(s_odd[0] | s_odd[1], 0)) {  // chunk 0 alone has nodes, and two wavefronts
    const unsigned long long path = path_of(lane < n ? a.parent[n0 + lane] : -1, lane, n);
    const T *v = (const T *)a.v_tree + ((size_t)n0 * d.num_kv_heads + g) * D;
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      const int row = (tile0 + t) * 16 + j;
      const unsigned long long seen = path_at(path, row < R ? small_div(row, G) : 0);
      const size_t rr = row < R ? row_at(row) : 0;
      for (int at = 16 * wave + 4 * kg; at < D && row < R; at += 16 * W) {
        if (!F32 && ch.chunks == 1) add_not_finite(v, (size_t)d.num_kv_heads * D, seen, at, (T *)a.out + rr * D + at);
        else add_not_finite(v, (size_t)d.num_kv_heads * D, seen, at, (ch.chunks == 1 ? (float *)a.out + rr * D : a.part_o + rr * plan.splits * D) + at);
      }
    }
  }
}

// ---- many rows ------------------------------------------------------------------------------------------
// The same products where a (sequence, kv head) has many query rows (60 nodes of 7 heads: 27 tiles): the W wavefronts of a
// workgroup have up to two tiles of rows each and share 64 keys at a time, which are widened into LDS once for all.
// What bounds it is the issue of vector instructions and MFMAs by the two wavefronts of a SIMD: some 140 of them, 16 exponentials
// of four slots among them, are 750 clocks for 32 keys and 32 rows, 544 of them the matrix core's; it takes 900.  Two trees of 52
// and 55 nodes, 28/4 heads, over 32768 positions: 84 us and 8 for the join, 50 GFLOP; 16 of 30 to 60 nodes over 1024 to
// 8192: 86 and 10.  Eight wavefronts to a workgroup, which share the keys among twice the rows: 93 and 114 us for the calls
// that take 89 and 95, since a barrier then holds up all of a CU.
// The loop over 32-key blocks is skewed by one: the matrix core gets a block's V^T P^T and the next one's scores in one go, and
// the vector work that follows has its scores already.  A thread asks for its share of a tile (16 bytes of keys and of
// values, two scales) two tiles ahead and puts it in LDS one tile ahead, while the matrix core has that work.  Two stages of
// LDS: what a barrier lets in has been written by everybody, and what it lets be overwritten has been read.
template <int DB, int W>
__global__ __launch_bounds__(64 * W, 2) void kv4_rows_kernel(Kv4AttnArgs a, Kv4Plan plan) {
  constexpr int D = 32 * DB, kRow = 64 * DB, TPW = 2, kTile = 64, kThreads = 64 * W;
  constexpr int kPieces = kTile * DB, kShare = (kPieces + kThreads - 1) / kThreads;  // 16-byte pieces of a tile; of a thread
  constexpr int kStage = 2 * kTile * kRow;
  const hb_attn_desc &d = a.d;
  __shared__ __attribute__((aligned(16))) unsigned char smem[2 * kStage];  // [values 64 x kRow | keys 64 x kRow]
  __shared__ int s_odd[W];  // whether a wavefront brought values of nodes that are not finite
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, kg = lane >> 4;
  Piece ch;
  if (!find_piece(a, plan, ch)) return;
  const int g = ch.g, G = plan.heads, n0 = ch.n0, n = ch.n, R = n * G;
  // full groups and a last one that is not: wavefronts without rows only help to bring the keys, which leaves the CU to others
  const int tiles = (R + 15) >> 4, tile_lo = ch.rg * TPW * W, tile_hi = min(tiles, tile_lo + TPW * W);
  const size_t row_base = (size_t)n0 * d.num_q_heads + (size_t)g * G;
  auto row_at = [&](int row) {
    const int node = small_div(row, G);
    return row_base + (size_t)node * d.num_q_heads + (row - node * G);
  };
  // tile t of this wavefront, and the rows of it that there are
  auto tile_of = [&](int t) { return tile_lo + TPW * wave + t; };
  const bool busy = tile_of(0) < tile_hi;
  auto row_of = [&](int t) { return tile_of(t) < tile_hi ? tile_of(t) * 16 + j : R; };

  // ---- a thread's share of a tile: piece i of 64 keys x DB blocks -----------------------------------
  struct Share {
    u32x4 k[kShare], v[kShare];
    uint32_t ks[kShare], vs[kShare];
  };
  const int keys = ch.end > ch.begin ? ch.end - ch.begin : 0, n_tiles = (keys + kTile - 1) / kTile;
  const int first16 = ch.begin >> 4, last16 = (ch.end - 1) >> 4;
  constexpr int kWave16 = 64 / DB / 16;  // 16s of keys in a wavefront's pieces
  static_assert(kWave16 == 1 || kWave16 == 2, "a wavefront takes 16 or 32 keys");
  Pages pages;
  size_t next[kShare][kWave16];
  auto find = [&](int tile) {
#pragma unroll
    for (int i = 0; i < kShare; ++i)
#pragma unroll
      for (int q = 0; q < kWave16; ++q) next[i][q] = pages.row(d, first16 + tile * 4 + (wave + i * W) * kWave16 + q, g);
  };
  auto load = [&](int tile, Share &x) {
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      if (kShare * kThreads > kPieces && i * kThreads + tid >= kPieces) continue;
      const int key = lane / DB;
      const size_t row = (kWave16 == 2 && key >= 16 ? next[i][kWave16 - 1] : next[i][0]) + (key & 15);
      x.k[i] = *(const u32x4 *)(a.kp.codes + row * (D / 2) + lane % DB * 16);
      x.v[i] = *(const u32x4 *)(a.vp.codes + row * (D / 2) + lane % DB * 16);
      x.ks[i] = a.kp.scales[row * DB + lane % DB];
      x.vs[i] = a.vp.scales[row * DB + lane % DB];
    }
    find(tile + 1);
  };
  auto put = [&](int tile, auto stage, const Share &x) {  // stage: tile & 1, known to the compiler
    unsigned char *st = smem + decltype(stage)::value * kStage;
    const int left = keys - tile * kTile;
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const int piece = i * kThreads + tid, key = piece / DB, blk = piece % DB;
      if (kShare * kThreads > kPieces && piece >= kPieces) continue;
      u32x4 c = x.v[i];
      uint32_t s = x.vs[i];
      if (left < kTile) {  // uniform: past the end, whatever it is, its weight is 0 and must not make that 0 * NaN
        asm volatile("" ::: "memory");
        const bool there = key < left;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = there ? c[e] : 0u;
        s = there ? s : 127u;
      }
      put_block<DB>(st, key, blk, c, s);
      put_block<DB>(st + kTile * kRow, key, blk, x.k[i], x.ks[i]);
    }
  };

  Share x, y;
  if (n_tiles > 0) {
    pages.begin(d, a.block_table + (size_t)ch.b * d.max_blocks_per_seq, first16, last16, plan.page_magic);
    find(0);
    load(0, x);
    load(1, y);
  }

  Rows<TPW, DB> w;
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int row = row_of(t);
    row_operand<DB>((const u32x4 *)a.q + row_at(min(row, R - 1)) * (D / 8), row < R, kg, w.q[t]);
    w.m[t] = kNegInf;
    w.ref[t] = 0.f;
    w.limit[t] = -1.f;
    w.l[t] = 0.f;
    w.lr[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < 2 * DB; ++dt) {
      w.o[t][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
      asm volatile("" : "+v"(w.o[t][dt]));
    }
  }
  const float c1 = d.softmax_scale * kLog2e;

  // ---- the nodes' own keys, chunk 0 only: values in the second stage, keys straight from memory -----
  if (ch.c == 0) {
    unsigned char *lv = smem + kStage;
    bool odd = false;
    for (int i = tid; i < kTile * 2 * DB * 2; i += kThreads) {
      const int key = i / (4 * DB), piece = i % (4 * DB);
      u32x4 v = {0u, 0u, 0u, 0u};
      if (key < n) {
        v = ((const u32x4 *)a.v_tree)[((size_t)(n0 + key) * d.num_kv_heads + g) * (D / 8) + piece];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t y = finite_or_zero_bf16x2(v[e]);
          odd |= y != v[e];
          v[e] = y;
        }
      }
      *(u32x4 *)(lv + key * kRow + ((piece ^ (v_swz(key) & (4 * DB - 1))) * 16)) = v;
    }
    if (const bool any = __any(odd); lane == 0) s_odd[wave] = any;
    const unsigned long long path = path_of(lane < n ? a.parent[n0 + lane] : -1, lane, n);
    __syncthreads();
    for (int blk = 0; blk < 2; ++blk) {
      if (32 * blk >= n || !busy) break;
      const uint32_t mine = (uint32_t)(path >> (32 * blk));
      f32x4 sc[TPW][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 k[4];
        row_operand<DB>((const u32x4 *)a.k_tree + ((size_t)(n0 + min(32 * blk + 16 * h + j, n - 1)) * d.num_kv_heads + g) * (D / 8), true, kg, k);
        score_tiles<TPW>(k, w.q, h, sc);
      }
#pragma unroll
      for (int t = 0; t < TPW; ++t) {
        const int row = row_of(t);
        const uint32_t allow = (uint32_t)__shfl((int)mine, row < R ? small_div(row, G) : 0, 64) >> (4 * kg);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[t][h][r] = ((allow >> (16 * h + r)) & 1u) ? sc[t][h][r] : kNegInf;
      }
      f32x8 p[TPW];
      weigh<false, true>(w, sc, c1, p);
      weigh_values<TPW, DB>(w, lv + 32 * blk * kRow, j, kg, p, true);
    }
  }

  // ---- the prefix --------------------------------------------------------------------------------------
  if (n_tiles > 0) {
    f32x4 sc[TPW][2];
    bf16x8 av[2 * DB];
    bf16x8 ak[2][4];  // a block's keys
    auto read_keys = [&](auto stage, int blk) {
      const unsigned char *at = smem + decltype(stage)::value * kStage + kTile * kRow;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = 32 * blk + 16 * h + j;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ak[h][i] = __builtin_bit_cast(bf16x8, (u32x4){0u, 0u, 0u, 0u});
          if (DB == 4 || kg < DB) ak[h][i] = *(const bf16x8 *)(at + key * kRow + (((4 * kg + i) ^ (v_swz(key) & (4 * DB - 1))) * 16));
        }
      }
    };
    auto scores = [&] {
      score_tiles<TPW>(ak[0], w.q, 0, sc);
      score_tiles<TPW>(ak[1], w.q, 1, sc);
    };
    // softmax of the scores that there are; the values of their block are asked for first
    auto vector_work = [&](int tile, auto stage, int blk, f32x8 (&p)[TPW]) {
      read_values<DB>(smem + decltype(stage)::value * kStage + 32 * blk * kRow, j, kg, av);
      const int left = keys - tile * kTile - 32 * blk;
      if (left < 32) {  // uniform
        asm volatile("" ::: "memory");  // a branch, not selects in every pass
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) sc[t][h][r] = 16 * h + 4 * kg + r < left ? sc[t][h][r] : kNegInf;
      }
      weigh<false>(w, sc, c1, p);
      if (left < 32) {  // few keys or many, a sequence's last ones may be all that it has: see weigh_values
        bf16x8 rest[TPW];
#pragma unroll
        for (int t = 0; t < TPW; ++t) rest[t] = __builtin_convertvector(p[t] - __builtin_convertvector(__builtin_convertvector(p[t], bf16x8), f32x8), bf16x8);
        accumulate<TPW, DB>(w, av, rest);
      }
    };
    auto values = [&](const f32x8 (&p)[TPW]) {
      bf16x8 pb[TPW];
#pragma unroll
      for (int t = 0; t < TPW; ++t) pb[t] = __builtin_convertvector(p[t], bf16x8);
      accumulate<TPW, DB>(w, av, pb);
    };
    // Barrier without the fence of __syncthreads(), which would wait for every load in flight: what has to be done in front of
    // it are reads and writes of LDS, and the wait for them is one statement with it
    auto barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    put(0, even, x);
    load(2, x);
    barrier();  // tile 0 is there, and the nodes' values have been read
    if (busy) {
      read_keys(even, 0);
      scores();
    }
    auto one_tile = [&](int i, auto stage, auto other, Share &share) {
      f32x8 p[TPW];
      put(i + 1, other, share);  // (behind the last tile: its keys once more, which nobody reads)
      load(i + 3, share);
      if (busy) {
        vector_work(i, stage, 0, p);
        read_keys(stage, 1);
        values(p);
        scores();
        vector_work(i, stage, 1, p);
      }
      barrier();
      if (busy) {
        read_keys(other, 0);
        values(p);
        scores();
      }
    };
    for (int i = 0; i < n_tiles; i += 2) {
      one_tile(i, even, odd, y);
      if (i + 1 < n_tiles) one_tile(i + 1, odd, even, x);
    }
  }

  // ---- write out: lane (j, kg) holds O[row j][16 dt + 4 kg + r] ----------------------------------------
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int row = row_of(t);
    const float l = group_sum(w.l[t]);
    if (row >= R) continue;
    const size_t rr = row_at(row);
    const float scale = w.lr[t][0] > 0.f ? l / w.lr[t][0] : 1.f;  // values weighed as the sum that they are divided by
    if (ch.chunks == 1) {
      const float inv = scale / l;
#pragma unroll
      for (int dt = 0; dt < 2 * DB; ++dt)
        store4((bf16_t *)a.out + rr * D + 16 * dt + 4 * kg, w.o[t][dt] * inv);
      if (a.lse && kg == 0) a.lse[rr] = (w.m[t] + log2f(l)) * kLn2;
    } else {
      float *po = a.part_o + (rr * plan.splits + ch.c) * D;
#pragma unroll
      for (int dt = 0; dt < 2 * DB; ++dt) *(f32x4 *)(po + 16 * dt + 4 * kg) = w.o[t][dt] * scale;
      if (kg == 0) *(kv4_f32x2 *)(a.part_ml + (rr * plan.splits + ch.c) * 2) = (kv4_f32x2){w.m[t], l};
    }
  }
  if (ch.c == 0) {
    int odd = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) odd |= s_odd[i];
    if (__builtin_expect(!odd, 1)) return;
    const unsigned long long path = path_of(lane < n ? a.parent[n0 + lane] : -1, lane, n);
    const bf16_t *v = (const bf16_t *)a.v_tree + ((size_t)n0 * d.num_kv_heads + g) * D;
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      const int row = row_of(t);
      const unsigned long long seen = path_at(path, row < R ? small_div(row, G) : 0);
      const size_t rr = row < R ? row_at(row) : 0;
      for (int at = 4 * kg; at < D && row < R; at += 16) {
        if (ch.chunks == 1) add_not_finite(v, (size_t)d.num_kv_heads * D, seen, at, (bf16_t *)a.out + rr * D + at);
        else add_not_finite(v, (size_t)d.num_kv_heads * D, seen, at, a.part_o + rr * plan.splits * D + at);
      }
    }
  }
}

// Rows of sequences that were cut: the chunks' results joined (log2 units).  A row's threads hold four elements each; results
// are asked for eight chunks at a time.
template <typename T>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4AttnArgs a, Kv4Plan plan) {
  const int D = a.d.head_dim, tpr = D / 4;
  const int len = *a.cut, lane = threadIdx.x & 63;
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(gid / tpr), piece = (int)(gid - (long)row * tpr);
  const int node = row / a.d.num_q_heads;
  // the row's sequence: up to 64 of them by their offsets in the lanes, which is one round trip
  int b, n0, n1, L;
  if (a.d.batch <= 64) {
    const bool there = lane < a.d.batch;
    const int at = there ? a.node_offset[lane] : 0, behind = there ? a.node_offset[lane + 1] : 0;
    const int length = there ? kv4_length(a.d, a.prefix_len, lane) : 0;
    b = 0;
    for (int r = 0; r < 64; r += tpr) {  // the wavefront's rows
      const unsigned long long m = __ballot(there && at <= __builtin_amdgcn_readlane(node, r));
      b = lane >= r && m ? 63 - __builtin_clzll(m) : b;
    }
    n0 = __shfl(at, b, 64);
    n1 = __shfl(behind, b, 64);
    L = __shfl(length, b, 64);
  } else {
    b = kv4_sequence(a.node_offset, a.d.batch, node < a.d.total_nodes ? node : 0);
    n0 = a.node_offset[b];
    n1 = a.node_offset[b + 1];
    L = kv4_length(a.d, a.prefix_len, b);
  }
  const int chunks = chunks_of(grains_of(L, plan), len);
  if (row >= a.d.total_nodes * a.d.num_q_heads || node < n0 || node >= n0 + nodes_of(a.d, n0, n1) || chunks == 1) return;
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
  store4((T *)a.out + (size_t)row * D + piece * 4, mean_of(T(), o, l));
  if (a.lse && piece == 0) a.lse[row] = (m + log2f(l)) * kLn2;
}

template <typename T, int TPW, int DB>
hipError_t launch(const Kv4AttnArgs &a, const Kv4Plan &plan, hipStream_t s) {
  kv4_attn_kernel<T, TPW, DB, kWaves><<<(unsigned)plan.grid, 64 * kWaves, 0, s>>>(a, plan);
  return hipGetLastError();
}

template <int DB, int W>
hipError_t launch_rows(const Kv4AttnArgs &a, const Kv4Plan &plan, hipStream_t s) {
  kv4_rows_kernel<DB, W><<<(unsigned)plan.grid, 64 * W, 0, s>>>(a, plan);
  return hipGetLastError();
}

}  // namespace

// Rows of (sequence, kv head) from which on wavefronts share the keys: four tiles and less, each wavefront has keys of its own.
// Own and shared, us (28 / 4 heads of 128; of 64 the same within a tenth): one sequence over 4096 keys, 63 rows 16.9 and 18.5, 70 17.1 and 19.0,
// 259 19.1 and 27.6; 16 over 2048, 63 21.7 and 28.9, 70 21.1 and 30.0, 126 22.2 and 33.9, 133 37.9 and 40.9; 16 over 300, 161 24.4
// and 18.7; 16 over 8192, 161 98 and 89, 420 195 and 162; 24 over 4000, 63 34.4 and 44.5, 70 59 and 47; two over 32768, 63 26.7 and
// 37.4, 126 35 and 43, 259 72 and 75, 364 99 and 76; 64 over 1000, 63 32.3 and 32.8, 126 60 and 38; 64 over 300, 35 26.0 and 16.1, 63 26.5
// and 16.9.  So 64 is low where workgroups of 32 rows are a round of the CUs or less and prefixes are not the longest, and high
// for many short sequences: what decides is how full either kernel's last round is, which this bound does not ask.
static bool shares_keys(const hb_attn_desc &d) { return d.num_q_heads / d.num_kv_heads * d.max_nodes_per_tree > 64; }

static int tiles_of(const hb_attn_desc &d) { return (d.num_q_heads / d.num_kv_heads * d.max_nodes_per_tree + 15) / 16; }
constexpr int64_t kMostGroups = 1 << 22;  // workgroups

bool kv4_attn_supports(const hb_attn_desc &d) {
  // what the workgroups count with 32 bits: pieces, and grains times row groups
  const int64_t ends = (int64_t)d.batch * tiles_of(d);
  if (ends * d.num_kv_heads > kMostGroups || ends * (((int64_t)d.page_size * d.max_blocks_per_seq) / 128 + 1) > 1 << 30) return false;
  return (d.head_dim == 64 || d.head_dim == 128) && d.page_size % 16 == 0 && d.page_size <= 1024 &&
         d.softmax_scale > 0.f && d.softmax_scale < 1e30f && d.num_q_heads / d.num_kv_heads <= 512;
}

// Chunks are planned for a round of the CUs: one workgroup to each, or two that share keys
void kv4_attn_plan(const hb_attn_desc &d, int64_t span, Kv4Plan *plan) {
  const int tiles = tiles_of(d), group = d.dtype == HB_F32 ? 1 : shares_keys(d) ? 2 * kSharing : tiles > 1 ? 2 : 1;
  plan->row_groups = (tiles + group - 1) / group;  // at most
  plan->group_shift = group == 1 ? 4 : group == 2 ? 5 : 7;
  static_assert(2 * kSharing == 8, "128 rows to a workgroup whose wavefronts share keys");
  static_assert(kWaves * kStep == 256, "a step of every wavefront");
  const bool sharing = group == 2 * kSharing;
  plan->grain_shift = sharing ? 7 : 8;
  plan->heads = d.num_q_heads / d.num_kv_heads;
  int64_t target = (sharing ? 512 : 256) / d.num_kv_heads;  // workgroups of a kv head
  target = target < 1 ? 1 : target;
  const int64_t most = (span + (1 << plan->grain_shift) - 1) >> plan->grain_shift;
  int64_t splits = d.num_splits ? d.num_splits : target;
  // Whole sequences where they are short, longer ones the more workgroups there are without a cut: that saves the write and the
  // reading of partial results and a launch.  Cut and whole, us (28 / 4 heads of 128): one token of one sequence over 512 keys 11.2
  // and 9.6, over 1024 11.4 and 11.1, over 1536 11.4 and 12.6; 16 chains of 8 nodes over 512 17.1 and 13.9, over 1024 19.2 and
  // 15.8, over 2048 21.6 and 20.0, over 3000 23.7 and 24.8; 60-node trees, 4 over 256 20.7 and 19.2, over 768 23.4 and 31.7,
  // 16 over 256 34.0 and 19.9, over 1536 54.3 and 51.8, over 2048 62.3 and 63.1.  Beyond those lengths never, for ragged ones.
  // Heads of 64, 8 / 8, 32 / 8 and 16 / 2 heads, float32, 204 calls of one to 16 sequences over 512 to 3000: the rule's choice is
  // the better or within 9 % of it.
  const int64_t pieces = (int64_t)d.batch * d.num_kv_heads * plan->row_groups;
  const int64_t whole = sharing ? std::min<int64_t>(pieces / 20, 12) : std::min<int64_t>(3 + pieces / 32, 8);
  if (!d.num_splits && most <= whole) splits = 1;
  splits = splits > most ? most : splits;
  splits = splits < 1 ? 1 : splits > 1024 ? 1024 : splits;
  if (d.num_splits) target = (int64_t)d.num_splits * d.batch * plan->row_groups;
  const int64_t room = kMostGroups / d.num_kv_heads;
  plan->target = (int32_t)(target < 1 ? 1 : target > room ? room : target);
  // each sequence's last chunk may be one more than its share of the target
  const int64_t ends = (int64_t)d.batch * plan->row_groups, most_wg = (plan->target + ends) * d.num_kv_heads;
  plan->fit = d.num_splits == 0 && d.batch <= 64 && ends < plan->target;
  plan->grid = (int32_t)((most_wg + 7) / 8 * 8);
  plan->splits = (int32_t)splits;
  const int page16 = d.page_size / 16;
  plan->page_magic = page16 == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + page16 - 1) / page16);
}

hipError_t launch_kv4_attn(const Kv4AttnArgs &a, const Kv4Plan &plan, hipStream_t s) {
  const bool f32 = a.d.dtype == HB_F32, wide = tiles_of(a.d) > 1, whole = a.d.head_dim == 128;
  hipError_t e;
  if (f32) e = whole ? launch<float, 1, 4>(a, plan, s) : launch<float, 1, 2>(a, plan, s);
  else if (shares_keys(a.d)) e = whole ? launch_rows<4, kSharing>(a, plan, s) : launch_rows<2, kSharing>(a, plan, s);
  else if (wide) e = whole ? launch<bf16_t, 2, 4>(a, plan, s) : launch<bf16_t, 2, 2>(a, plan, s);
  else e = whole ? launch<bf16_t, 1, 4>(a, plan, s) : launch<bf16_t, 1, 2>(a, plan, s);
  if (e != hipSuccess || plan.splits == 1) return e;
  const long threads = (long)a.d.total_nodes * a.d.num_q_heads * (a.d.head_dim / 4);
  const unsigned grid = (unsigned)((threads + 255) / 256);
  if (f32) kv4_join_kernel<float><<<grid, 256, 0, s>>>(a, plan);
  else kv4_join_kernel<bf16_t><<<grid, 256, 0, s>>>(a, plan);
  return hipGetLastError();
}

}  // namespace hb
