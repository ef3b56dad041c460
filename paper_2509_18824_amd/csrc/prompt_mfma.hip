// Attention of prompts on the bf16 matrix cores (hb_prompt_attn; head sizes 64 and 128, pages of a power of two).
//
// A workgroup has 256 rows, pairs (token, query head of the group) of one (sequence, kv head), and a part of their keys; each of
// its eight wavefronts has 32 rows, which all share the keys: tiles of 64, four stages of them in LDS.  Both products are
// transposed, with 32x32x16 instructions:
//   S^T = K Q^T     A = 32 keys x 16 of D from LDS, B = the rows' queries, which stay in registers
//   O^T = V^T P^T   A = 32 of D x 16 keys, by the transposing reads of LDS, B = the weights
// so that a lane's scores are all of one row (two lanes share it), a row's sum and reference are numbers of a lane, and the scores
// of the first product are, exponentiated and packed in place, the second one's operand.
//   softmax   in base 2, online.  A row's reference is the largest score of its first block of 32 keys, and moves only when a lane's
//             weights of a step sum to more than 256: float32 and bf16 have the room, and a step needs no maximum, no exchange between
//             lanes and no scaling of the result.  A weight is rounded to bf16; results are divided by the sum of the rounded ones
//             (errors of the two then cancel in part), the log-sum-exp is made of the others.
//   loads     global to LDS, 16 bytes a lane, each piece of a row at its place XOR a number of the row, so that neither product's
//             reads meet in a bank.  A tile is asked for three tiles ahead; its addresses are made once.
//   a step    is 16 matrix instructions of 32 clocks and, between each two, a sixteenth of the last block's softmax and of the
//             next reads from LDS, laid side by side by hand: left alone, the compiler puts them one behind the other
//             (8192 rows: 0.62 ms, so 0.50).
//
// What bounds it is how a SIMD's two wavefronts share it: over 8192 rows the matrix core is busy for 53 % of the cycles, vector
// instructions are issued in 43 (four and an exponential for each matrix instruction), LDS is busy for 27, without bank conflicts;
// a wavefront waits for a place to issue in 33 % of its time and for LDS and barriers in 29.  The clock is 1.8 GHz of 2.4 under this load.
// 28 query and 4 kv heads of 128:
//   one prompt of 8192 rows 479 us, 997 TFLOP/s; of 32768 1106 TFLOP/s (a large bf16 product: 1201 to 1510)
//   512 rows over 32 K cached 272 us, 878 TFLOP/s: 56 tiles in 4 parts on 256 compute units, and a join of 12 us
//   8 prompts of 1 to 2048 rows, some behind a cached beginning, 230 us, 830 TFLOP/s
// Not taken: 64 rows a wavefront, one a SIMD (500 us; 8 ragged prompts 295); tiles of 128 rows by four wavefronts (64 rows alone 9 us
// instead of 12, but 1024 43 to 52 instead of 36); 512 rows over 32 K in one to three parts (814, 440, 309 us).
#include <type_traits>

#include "prompt.h"

namespace hb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 *lds_bf16x4_ptr;
typedef __attribute__((address_space(1))) const void *gptr_t;
typedef __attribute__((address_space(3))) void *lptr_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(4))) int32_t *table_t;
typedef unsigned int swap2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
#define HB_NEG_INF (-__builtin_huge_valf())
constexpr float kMost = 256.f;  // sum of a lane's weights of a step, up to which their row's reference stays

__device__ __forceinline__ uint32_t finite_or_zero(uint32_t w) {  // of two bf16
  const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu, hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
  return lo | hi;
}
__device__ __forceinline__ float half_max(float x) {
  const swap2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const swap2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
// sum + both numbers of a pair
__device__ __forceinline__ float add2(uint32_t two, float sum) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
}
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float max16(const f32x16 &s) {
  return fmaxf(max3(max3(max3(s[0], s[1], s[2]), s[3], s[4]), max3(s[5], s[6], s[7]), max3(s[8], s[9], s[10])),
               max3(max3(s[11], s[12], s[13]), s[14], s[15]));
}

template <int D, int NW, int KT, int NS>
struct Shape {
  static constexpr int kRows = 32 * NW, kRowBytes = 2 * D, kPieces = D / 8, kKeysPerLoad = 64 / kPieces;
  static constexpr int kTileBytes = KT * kRowBytes, kStage = 2 * kTileBytes;
  static constexpr int kLoads = KT / kKeysPerLoad;     // of K, and as many of V, a tile
  static constexpr int kPer = kLoads / NW;             // of a wavefront
  static constexpr int kSteps = D / 16, kSlabs = D / 32, kBlocks = KT / 32;
  // tiles that have landed beside the one in work when its last block begins; tiles that may still be under way then
  static constexpr int kAhead = kBlocks == 1 ? 3 : 2, kLate = NS - 1 - kAhead;
  static constexpr size_t kLds = (size_t)NS * kStage + 4 * NW;  // and a word for each wavefront's rows
  static_assert(KT == 32 || KT == 64, "blocks of 32 keys, one or two a tile");
  static_assert(NW * kKeysPerLoad % 16 == 0, "a wavefront's loads lie sixteens apart");
  static_assert(kLoads % NW == 0 && kLate >= 0 && kLds <= 160 * 1024, "a tile's loads are dealt evenly");
  // XOR on a row's 16-byte pieces
  static __device__ __forceinline__ int k_swz(int key) { return D == 128 ? key & 15 : (key >> 1) & 7; }
  static __device__ __forceinline__ int v_swz(int key) { return D == 128 ? (key & 3) << 2 : ((key >> 1) & 1) << 2; }
};

struct Sums {  // of a step's weights
  float rounded, whole;
};

// the kernel's first argument, from where the launch has put it
typedef const __attribute__((address_space(4))) PromptArgs *args_t;
__device__ __forceinline__ args_t again() {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return (args_t)at;
}
template <typename T>
using global_t = __attribute__((address_space(1))) T *;

template <int D, int NW, int KT, int NS, bool LSE>
__global__ __launch_bounds__(64 * NW, 2) void prompt_mfma_kernel(PromptArgs a, int page_shift, const bf16_t *__restrict__ kr,
                                                                 const bf16_t *__restrict__ vr, const bf16_t *__restrict__ kp,
                                                                 const bf16_t *__restrict__ vp, const int32_t *__restrict__ block_table) {
  using S = Shape<D, NW, KT, NS>;
  constexpr int KS = S::kSteps, DT = S::kSlabs;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 31, hf = lane >> 5;
  const int Hkv = a.d.num_kv_heads, Hq = a.d.num_q_heads, G = Hq / Hkv;
  const int tile_id = blockIdx.x / (uint32_t)Hkv, h = blockIdx.x - tile_id * Hkv;
  const PromptTile w = prompt_tile<S::kRows, KT>(a, tile_id, blockIdx.y);
  prompt_head<S::kRows>(a, w, tile_id, h, blockIdx.y);
  if (w.t < 0) return;
  const int P = w.P, begin = w.begin, end = w.end, rows_all = w.n * G;

  // ---- rows: 32 of the wavefront's, one a lane (two lanes share it) -------------------------------------------------
  const int my_row0 = w.t * S::kRows + wave * 32;
  int sees;
  bf16x8 qf[KS];
  {
    const int row = my_row0 + j;
    const bool there = row < rows_all;
    const int token = there ? (int)((uint32_t)row / (uint32_t)G) : w.n - 1, head = there ? row - token * G : 0;
    sees = min(P + token, end - 1);
    const u32x4 *src = (const u32x4 *)a.q + ((size_t)(w.row0 + token) * Hq + (size_t)h * G + head) * (D / 8);
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, src[2 * s + hf]);  // a row that is not there: some row's, for nobody
  }
  const int first_sees = __builtin_amdgcn_readfirstlane(sees);
  // what the wavefront's last row sees: behind it there is nothing for it to do
  const int last_sees = __builtin_amdgcn_readlane(sees, 31);

  // ---- keys' way to LDS ---------------------------------------------------------------------------------------------
  const int n_tiles = (end - begin + KT - 1) / KT;
  const bool no_rows = my_row0 >= rows_all;
  const int my_tiles = no_rows || last_sees < begin ? 0 : (last_sees - begin) / KT + 1;
  // A load moves 64 pieces of 16 bytes: kKeysPerLoad keys, whose rows in memory are `row_bytes` (prompt) or kRowBytes (page)
  // apart.  The lane that fills piece p of a row in LDS takes piece p ^ swizzle(row) from memory; the swizzles repeat from one
  // of a wavefront's loads to the next, so that a lane's part of the address is one number for all.
  const int lkey = lane / S::kPieces, piece = lane % S::kPieces;
  const uint32_t row_bytes = (uint32_t)Hkv * S::kRowBytes;
  const int key_of_first = wave * S::kKeysPerLoad + lkey;
  const uint32_t k_piece = (piece ^ S::k_swz(key_of_first)) * 16, v_piece = (piece ^ S::v_swz(key_of_first)) * 16;
  const bool wide_pages = page_shift >= 4;
  const int page = 1 << page_shift;
  const int32_t *bt = block_table ? block_table + (size_t)w.b * a.d.max_blocks_per_seq : nullptr;
  auto page_at = [&](int idx) {
    int id = bt[idx];
    return id < 0 ? 0 : id >= a.d.num_blocks ? a.d.num_blocks - 1 : id;
  };
  int ids[S::kPer];
  auto fetch = [&](int i) {  // pages of the wavefront's loads of tile i, where it lies in the prefix as a whole
    int k0 = begin + i * KT, wv = wave;
    asm volatile("" : "+s"(k0), "+s"(wv));
    if (wide_pages && k0 + KT <= P && i < n_tiles)
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        // through the scalar cache: a vector load here would wait for every load of keys that is under way
        const int id = ((table_t)bt)[(k0 + (wv + NW * x) * S::kKeysPerLoad) >> page_shift];
        ids[x] = id < 0 ? 0 : id >= a.d.num_blocks ? a.d.num_blocks - 1 : id;
      }
  };
  uint64_t k_from[S::kPer], v_from[S::kPer];  // a lane's addresses
  auto place = [&](int i) {                    // ... of tile i
    int k0 = begin + i * KT, wv = wave;
    asm volatile("" : "+s"(k0), "+s"(wv));  // or a hundred numbers are made in front of the loop, and kept in lanes of registers
    if (wide_pages && k0 + KT <= P) {
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {  // a load's keys lie in one page
        const size_t from = (((size_t)ids[x] * Hkv + h) * page + ((k0 + (wv + NW * x) * S::kKeysPerLoad) & (page - 1))) * S::kRowBytes;
        k_from[x] = (uint64_t)kp + from + (lkey * S::kRowBytes + k_piece);
        v_from[x] = (uint64_t)vp + from + (lkey * S::kRowBytes + v_piece);
      }
    } else if (k0 >= P && k0 + KT <= end) {
      size_t from = ((size_t)(w.row0 + k0 - P + wv * S::kKeysPerLoad) * Hkv + h) * S::kRowBytes;
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        k_from[x] = (uint64_t)kr + from + (lkey * row_bytes + k_piece);
        v_from[x] = (uint64_t)vr + from + (lkey * row_bytes + v_piece);
        from += (size_t)(NW * S::kKeysPerLoad) * row_bytes;
      }
    } else {  // the end of the prefix, the end of the keys, narrow pages: every key for itself
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        int pos = k0 + (wv + NW * x) * S::kKeysPerLoad + lkey;
        pos = pos < end ? pos : end - 1;
        uint64_t row = (uint64_t)(w.row0 + pos - P) * Hkv + h, kb = (uint64_t)kr, vb = (uint64_t)vr;
        if (pos < P) {
          row = ((uint64_t)page_at(pos >> page_shift) * Hkv + h) * page + (pos & (page - 1));
          kb = (uint64_t)kp;
          vb = (uint64_t)vp;
        }
        asm volatile("" : "+v"(kb), "+v"(vb));  // values: no choice among their places in memory is made of this
        k_from[x] = kb + row * S::kRowBytes + k_piece;
        v_from[x] = vb + row * S::kRowBytes + v_piece;
      }
    }
  };
  auto load = [&](int i, int x) {  // one of tile i's loads of keys (x < kPer) and of values (behind)
    unsigned char *st = smem + (i % NS) * S::kStage + wave * 1024;
    if (x < S::kPer)
      __builtin_amdgcn_global_load_lds((gptr_t)k_from[x], (lptr_t)(st + NW * x * 1024), 16, 0, 0);
    else
      __builtin_amdgcn_global_load_lds((gptr_t)v_from[x - S::kPer], (lptr_t)(st + S::kTileBytes + NW * (x - S::kPer) * 1024), 16, 0, 0);
  };
  // the last key that all of the workgroup's rows see
  const int all_see = P + w.t * S::kRows / G;
  auto clean = [&](int i) {  // values of tile i, by the wavefront that loaded them
    if (i >= n_tiles || begin + i * KT + KT - 1 <= all_see) return;
#pragma unroll
    for (int x = 0; x < S::kPer; ++x) {
      const int n = wave + NW * x;
      if (begin + i * KT + n * S::kKeysPerLoad + lkey <= all_see) continue;
      u32x4 *p = (u32x4 *)(smem + (i % NS) * S::kStage + S::kTileBytes + n * 1024 + lane * 16);
      u32x4 y = *p;
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = finite_or_zero(y[q]);
      *p = y;
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): they are there
  };

  // ---- state ----------------------------------------------------------------------------------------------------------
  f32x16 o[DT], s;
  bf16x8 kf[KS], vf[DT][2], pb[2];
  // base-2 reference of a row's scores; sum of its weights as they are multiplied with values, in bf16, which results are
  // divided by; and as they are in float32, for the log-sum-exp
  float ref, l, le;
  const float c1 = a.d.softmax_scale * kLog2e;
  // A workgroup does its part up to three times, see below; in the third, rows whose bits are set here in a way of their own.  (In
  // registers, this and what it needs cost the loop some that it does not have.)
  uint32_t *const anew = (uint32_t *)(smem + (size_t)NS * S::kStage) + wave;
  int pass = 0;
#pragma unroll 1
  for (;; ++pass) {
  const bool careful = pass > 0;
  ref = 0.f;
  const float most = careful ? -1.f : kMost;  // careful: every step looks

  const int k_lane = j * S::kRowBytes, kx = hf ^ S::k_swz(j);
  auto k_at = [&](const unsigned char *st, int blk) { return st + blk * 32 * S::kRowBytes + k_lane; };
  auto one_k = [&](const unsigned char *p, int q) { return __builtin_bit_cast(bf16x8, *(const u32x4 *)(p + (((2 * q) ^ kx) << 4))); };
  const int s4 = lane & 15, e = (lane >> 4) & 1, vkey = 4 * hf + (s4 >> 2);
  const int v_lane = vkey * S::kRowBytes + 8 * (s4 & 1), vx = S::v_swz(vkey);
  auto v_at = [&](const unsigned char *st, int blk) { return st + S::kTileBytes + blk * 32 * S::kRowBytes + v_lane; };
  auto one_v = [&](const unsigned char *p, int dt, int c) {
    const unsigned char *pd = p + (((4 * dt + 2 * e + ((s4 >> 1) & 1)) ^ vx) << 4);
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(pd + 16 * c * S::kRowBytes));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_ptr)(pd + (16 * c + 8) * S::kRowBytes));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  // scores against the block of keys from k0: those of keys that a row does not see go
  auto mask = [&](int k0) {
    asm volatile("" : "+s"(k0));
    if (k0 + 31 > first_sees) {  // uniform: some row does not see some key
      const int lim = sees - k0 - 4 * hf;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) <= lim ? s[r] : HB_NEG_INF;
    }
  };
  auto weights = [&](const f32x16 &x, bf16x8 (&p)[2]) {  // of a block, plainly
    Sums part = {0.f, 0.f};
    uint32_t w[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float a0 = __builtin_amdgcn_exp2f(fmaf(x[2 * r], c1, -ref)), a1 = __builtin_amdgcn_exp2f(fmaf(x[2 * r + 1], c1, -ref));
      w[r] = pack2(a0, a1);
      part.rounded = add2(w[r], part.rounded);
      part.whole += a0 + a1;
    }
    p[0] = __builtin_bit_cast(bf16x8, (u32x4){w[0], w[1], w[2], w[3]});
    p[1] = __builtin_bit_cast(bf16x8, (u32x4){w[4], w[5], w[6], w[7]});
    return part;
  };
  // A block's weights, whose sum in this lane is `part`, are in pb in bf16; x: the scores.  A row's reference stays while
  // weights are small: all of a lane's are, if their sum is (they are not negative).  Else, and for the first block (a row sees
  // its first key, or nothing at all of this part), the reference becomes the row's largest score of the block and the weights
  // are made anew.
  auto settle = [&](const f32x16 &x, Sums part, bool first) {
    if (first || __any(!(part.rounded <= most))) {
      asm volatile("" ::: "memory");
      const float mx = half_max(max16(x)) * c1;  // c1 > 0
      // (a row's own weights decide, not those of the others in the wavefront)
      const bool mine = pass == 2 && (*anew >> j & 1);
      // a row of `anew`: 2^raise is more than twice the keys
      const float raise = (float)(33 - __builtin_clz(end - begin)), so_far = half_sum(l), heaviest = half_max(part.rounded), to = mine ? mx + raise : mx;
      // nothing: no score so far that was more than -infinity
      const bool nothing = first || (mine && so_far == 0.f);
      const bool grow = nothing ? mx > HB_NEG_INF : (mine || heaviest > kMost) && to > ref;
      const float alpha = grow && !nothing ? __builtin_amdgcn_exp2f(ref - to) : 1.f;
      ref = grow ? to : ref;
      if (first) {  // what the sums hold so far is nothing
        l = le = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = (f32x16)(0.f);
      } else if (__any(alpha != 1.f)) {
        l *= alpha;
        le *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
      }
      part = weights(x, pb);
    }
    l += part.rounded;
    if (LSE) le += part.whole;
  };

  // One step: a block's scores become weights, while the matrix core makes the next block's scores (first) and adds the last
  // block's weights' products.  None needs what another makes, so that they can be laid side by side by hand: an instruction
  // of the matrix core (32 clocks), then a sixteenth of the vector work and of the reads from LDS (the last block's values,
  // then the keys of the block behind the next), and a fence for the scheduler, which would put them one behind the other.
  auto step = [&](const unsigned char *pv, const unsigned char *pk, bool first, auto middle) {
    constexpr int kAll = KS + 2 * DT, kEach = 16 / kAll;
    f32x16 sn;
    float p[2];
    Sums part = {0.f, 0.f};
    uint32_t w[8];
    auto pair = [&](int q) {
      w[q] = pack2(p[0], p[1]);
      part.rounded = add2(w[q], part.rounded);
      asm volatile("" : "+v"(w[q]), "+v"(part.rounded));
      if (LSE) {
        part.whole += p[0] + p[1];
        asm volatile("" : "+v"(part.whole));
      }
    };
#pragma unroll
    for (int x = 0; x < kAll; ++x) {
      if (x == KS) middle();
      __builtin_amdgcn_sched_barrier(0);
      if (x < KS) {
        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x], qf[x], x ? sn : (f32x16)(0.f), 0, 0, 0);
        vf[x % DT][x / DT] = one_v(pv, x % DT, x / DT);
      } else {
        const int y = x - KS;
        o[y % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[y % DT][y / DT], pb[y / DT], o[y % DT], 0, 0, 0);
        kf[y] = one_k(pk, y);
      }
#pragma unroll
      for (int r = kEach * x; r < kEach * x + kEach; ++r) {
        float y = __builtin_amdgcn_exp2f(fmaf(s[r], c1, -ref));
        asm volatile("" : "+v"(y));
        if (r % 2 == 0 && r > 0) pair(r / 2 - 1);  // (an exponential's result has to wait an instruction)
        p[r % 2] = y;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    pair(7);
    pb[0] = __builtin_bit_cast(bf16x8, (u32x4){w[0], w[1], w[2], w[3]});
    pb[1] = __builtin_bit_cast(bf16x8, (u32x4){w[4], w[5], w[6], w[7]});
    settle(s, part, first);
    s = sn;
  };

  // ---- the loop -----------------------------------------------------------------------------------------------------
#define HB_BARRIER() asm volatile("s_barrier" ::: "memory")
#define HB_WAIT_LOADS(N_) __builtin_amdgcn_s_waitcnt(((N_) & 15) | (((N_) >> 4) << 14) | (7 << 4) | (15 << 8))  // vmcnt alone
  auto stage = [&](int i) { return smem + i % NS * S::kStage; };
  auto block_k = [&](int b) { return k_at(stage(b / S::kBlocks), b % S::kBlocks); };
  auto next_tile = [&](int i) {  // of those that are asked for one behind the other, fetch(i) before
    place(i);
#pragma unroll
    for (int x = 0; x < 2 * S::kPer; ++x) load(i, x);
    fetch(i + 1);
  };
  // In the middle of block kBlocks (i + 1), tile i + kAhead has to have landed, for everybody; and everybody is done with tile
  // i, whose stage takes tile i + NS.
  auto turn = [&](int i) {
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): reads of tile i have come back
    if (i + NS <= n_tiles)
      HB_WAIT_LOADS(2 * S::kPer * S::kLate);
    else
      HB_WAIT_LOADS(0);
    if (careful) clean(i + S::kAhead);
    HB_BARRIER();
    if (i + NS < n_tiles) next_tile(i + NS);
  };
  fetch(0);
#pragma unroll 1
  for (int i = 0; i < NS && i < n_tiles; ++i) next_tile(i);
  if (NS <= n_tiles)
    HB_WAIT_LOADS(2 * S::kPer * (NS - S::kAhead));
  else
    HB_WAIT_LOADS(0);
  if (careful)
    for (int i = 0; i < S::kAhead; ++i) clean(i);
  HB_BARRIER();

  if (my_tiles > 0) {
#pragma unroll
    for (int q = 0; q < KS; ++q) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one_k(block_k(0), q), qf[q], q ? s : (f32x16)(0.f), 0, 0, 0);
#pragma unroll
    for (int q = 0; q < KS; ++q) kf[q] = one_k(block_k(1), q);
    pb[0] = pb[1] = (bf16x8)((__bf16)0.f);
    mask(begin);
    // (the first step has no block behind it: it multiplies some values of the first tile's with no weights, and forgets it)
    step(v_at(stage(0), 0), block_k(2), true, [] {});
    mask(begin + 32);
#pragma unroll 1
    for (int i = 0; i < my_tiles; ++i) {
      const unsigned char *st = stage(i);
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) {
        const int blk = i * S::kBlocks + b + 1;
        step(v_at(st, b), k_at(stage(i + (b + 3) / S::kBlocks), (b + 3) % S::kBlocks), false, [&] {
          if (b == S::kBlocks - 1) turn(i);
        });
        mask(begin + 32 * (blk + 1));
      }
    }
  } else {
    l = le = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = (f32x16)(0.f);
  }
#pragma unroll 1
  for (int i = my_tiles; i < n_tiles; ++i) turn(i);

  // Keys that a row does not see have weight 0 in the products, and 0 times a value that is not finite is no number.  Where
  // that, or anything else, has made results that are not finite, or a row that sees keys has next to no weights (a row with a
  // reference has one of 1; its first block's scores were all -infinity, and those behind are below 0), the workgroup does its part once
  // more, `careful`: such values of keys that some row does not see are zeros in LDS.  What is so now is so by what a row sees.  Where
  // there are such rows still (weights of up to 256, or many, times values near float32's largest; no reference; a value that is not
  // finite), it does its part a third time, in which a row that was such has its reference when it has a score, and `raise`
  // above its largest score: its weights' sum is at most one, and a sum of them times finite values finite.  All others get the bits
  // that they had each time.
  if (pass == 2) break;
  // (a lane's; 0, or no number)
  float none = !(half_sum(l) >= 0.5f) && sees >= begin ? __builtin_nanf("") : 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) none = fmaf(o[dt][r], 0.f, none);
  // (everybody is behind the last reads of the stages)
  __syncthreads();
  if (tid == 0) *(int *)smem = 0;
  __syncthreads();
  if (!no_rows && my_tiles > 0 && none != none) *(int *)smem = 1;
  __syncthreads();
  if (*(int *)smem == 0) break;
  if (careful) {
    const unsigned long long lanes = __ballot(none != none);
    *anew = (uint32_t)lanes | (uint32_t)(lanes >> 32);  // two lanes share a row
  }
  __syncthreads();
  }
  if (pass > 0)  // values that were left out, to the rows that see them
    for (int kk = max(begin, all_see + 1); kk < end; ++kk) {  // a row of the prompt: the prefix is seen by all
      const bf16_t *vs = vr + ((size_t)(w.row0 + kk - P) * Hkv + h) * D;
      if (kk <= sees)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float y = bf16_to_f32(vs[32 * dt + 8 * (r >> 2) + 4 * hf + (r & 3)]);
            if (!(fabsf(y) < __builtin_huge_valf())) o[dt][r] += y;
          }
    }

  // ---- results ------------------------------------------------------------------------------------------------------
  // (the arguments are read again, so that the loop need not keep them in its registers)
  const args_t z = again();
  const int zHq = z->d.num_q_heads, zHkv = z->d.num_kv_heads, zG = zHq / zHkv;
  const float sum = half_sum(l), whole = half_sum(le);
  const int r0 = wave * 32 + j, row = w.t * S::kRows + r0;
  if (row >= w.n * zG) return;
  if (w.parts == 1) {
    const int token = (int)((uint32_t)row / (uint32_t)zG);
    const size_t at = (size_t)(w.row0 + token) * zHq + (size_t)h * zG + (row - token * zG);
    const float inv = 1.f / sum;
    const global_t<bf16_t> out = (global_t<bf16_t>)z->out;
    const global_t<float> lse = (global_t<float>)z->lse;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        u32x2 x;
        x[0] = pack2(o[dt][4 * g] * inv, o[dt][4 * g + 1] * inv);
        x[1] = pack2(o[dt][4 * g + 2] * inv, o[dt][4 * g + 3] * inv);
        *(global_t<u32x2>)(out + at * D + 32 * dt + 8 * g + 4 * hf) = x;
      }
    if (LSE && hf == 0) lse[at] = (ref + log2f(whole)) * kLn2;
  } else {
    const size_t slot = (((size_t)(blockIdx.x / zHkv) * zHkv + h) * z->parts + blockIdx.y) * S::kRows + r0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = o[dt][4 * g + r];
        *(global_t<f32x4>)((global_t<float>)z->part_o + slot * D + 32 * dt + 8 * g + 4 * hf) = x;
      }
    if (hf == 0) *(global_t<f32x4>)((global_t<float>)z->part_ml + slot * 4) = (f32x4){sum == 0.f ? HB_NEG_INF : ref, sum, whole, 0.f};
  }
#undef HB_BARRIER
#undef HB_WAIT_LOADS
}

template <int D, int NW, int KT, int NS>
hipError_t launch(const PromptArgs &a, hipStream_t s) {
  using S = Shape<D, NW, KT, NS>;
  auto kern = a.lse ? prompt_mfma_kernel<D, NW, KT, NS, true> : prompt_mfma_kernel<D, NW, KT, NS, false>;
  hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kLds);
  if (e != hipSuccess) return e;
  kern<<<dim3(a.tiles * a.d.num_kv_heads, a.parts), 64 * NW, S::kLds, s>>>(
      a, __builtin_ctz(a.d.page_size), (const bf16_t *)a.k, (const bf16_t *)a.v, (const bf16_t *)a.k_pool, (const bf16_t *)a.v_pool,
      a.block_table);
  e = hipGetLastError();
  if (e == hipSuccess && a.parts > 1) e = launch_prompt_join(a, S::kRows, s);
  return e;
}

}  // namespace

bool prompt_mfma_supports(const hb_attn_desc &d) {
  return d.dtype == HB_BF16 && (d.head_dim == 64 || d.head_dim == 128) && (d.page_size & (d.page_size - 1)) == 0 &&
         d.softmax_scale > 0.f && d.softmax_scale < 1e30f;
}

int32_t prompt_mfma_rows(const hb_attn_desc &) { return 256; }

hipError_t launch_prompt_mfma(const PromptArgs &a, hipStream_t s) {
  return a.d.head_dim == 128 ? launch<128, 8, 64, 4>(a, s) : launch<64, 8, 64, 4>(a, s);
}

}  // namespace hb
