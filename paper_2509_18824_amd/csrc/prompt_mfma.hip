// Attention of prompts on the bf16 matrix cores (hb_prompt_attn; head sizes 64 and 128, pages of a power of two).
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
constexpr float kSlack = 8.f;  // log2 units that a score may exceed its row's reference by

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
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ float max16(const f32x16 &s) {
  return fmaxf(max3(max3(max3(s[0], s[1], s[2]), s[3], s[4]), max3(s[5], s[6], s[7]), max3(s[8], s[9], s[10])),
               max3(max3(s[11], s[12], s[13]), s[14], s[15]));
}

template <int D, int NW, int KT, int NS>
struct Shape {
  static constexpr int kRows = 64 * NW, kRowBytes = 2 * D, kPieces = D / 8, kKeysPerLoad = 64 / kPieces;
  static constexpr int kTileBytes = KT * kRowBytes, kStage = 2 * kTileBytes;
  static constexpr int kLoads = KT / kKeysPerLoad;     // of K, and as many of V, a tile
  static constexpr int kPer = kLoads / NW;             // of a wavefront
  static constexpr int kSteps = D / 16, kSlabs = D / 32, kBlocks = KT / 32;
  static constexpr size_t kLds = (size_t)NS * kStage;
  static_assert(KT == 64, "an even and an odd block a tile");
  static_assert(NW * kKeysPerLoad % 16 == 0, "a wavefront's loads lie sixteens apart");
  static_assert(kLoads % NW == 0 && kLds <= 160 * 1024, "a tile's loads are dealt evenly");
  // XOR on a row's 16-byte pieces
  static __device__ __forceinline__ int k_swz(int key) { return D == 128 ? key & 15 : (key >> 1) & 7; }
  static __device__ __forceinline__ int v_swz(int key) { return D == 128 ? (key & 3) << 2 : ((key >> 1) & 1) << 2; }
};

// the kernel's first argument, from where the launch has put it
__device__ __forceinline__ const PromptArgs &again(const PromptArgs &a) {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const PromptArgs *)at;
}

template <int D, int NW, int KT, int NS>
__global__ __launch_bounds__(64 * NW, 1) void prompt_mfma_kernel(PromptArgs a, int page_shift, const bf16_t *__restrict__ kr,
                                                                 const bf16_t *__restrict__ vr, const bf16_t *__restrict__ kp,
                                                                 const bf16_t *__restrict__ vp, const int32_t *__restrict__ block_table) {
  using S = Shape<D, NW, KT, NS>;
  constexpr int KS = S::kSteps, DT = S::kSlabs;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 31, hf = lane >> 5;
  const int Hkv = a.d.num_kv_heads, Hq = a.d.num_q_heads, G = Hq / Hkv;
  const int h = blockIdx.x % Hkv, tile_id = blockIdx.x / Hkv;
  const PromptTile w = prompt_tile<S::kRows, KT>(a, tile_id, blockIdx.y);
  if (w.t < 0) return;
  const int P = w.P, begin = w.begin, end = w.end, rows_all = w.n * G;

  // ---- rows: 32 of each of the wavefront's two tiles, one a lane (two lanes share it) ------------------------------
  int sees[2], first_sees[2];
  bf16x8 qf[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = w.t * S::kRows + wave * 64 + 32 * t + j;
    const bool there = row < rows_all;
    const int token = there ? row / G : w.n - 1, head = there ? row - token * G : 0;
    sees[t] = min(P + token, end - 1);
    first_sees[t] = __builtin_amdgcn_readfirstlane(sees[t]);
    const u32x4 *src = (const u32x4 *)a.q + ((size_t)(w.row0 + token) * Hq + (size_t)h * G + head) * (D / 8);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (there) x = src[2 * s + hf];
      qf[t][s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  // what the wavefront's last row sees: behind it there is nothing for it to do
  const int last_sees = __builtin_amdgcn_readlane(max(sees[0], sees[1]), 31);

  // ---- keys' way to LDS ---------------------------------------------------------------------------------------------
  const int n_tiles = (end - begin + KT - 1) / KT;
  const bool no_rows = w.t * S::kRows + wave * 64 >= rows_all;
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
    const int k0 = begin + i * KT;
    if (wide_pages && k0 + KT <= P && i < n_tiles)
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        // through the scalar cache: a vector load here would wait for every load of keys that is under way
        const int id = ((table_t)bt)[(k0 + (wave + NW * x) * S::kKeysPerLoad) >> page_shift];
        ids[x] = id < 0 ? 0 : id >= a.d.num_blocks ? a.d.num_blocks - 1 : id;
      }
  };
  uint64_t k_from[S::kPer], v_from[S::kPer];  // a lane's addresses
  auto place = [&](int i) {                    // ... of tile i (past the last: of the last once more)
    const int ti = i < n_tiles ? i : n_tiles - 1;
    const int k0 = begin + ti * KT;
    if (wide_pages && k0 + KT <= P && i < n_tiles) {
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {  // a load's keys lie in one page
        const size_t from = (((size_t)ids[x] * Hkv + h) * page + ((k0 + (wave + NW * x) * S::kKeysPerLoad) & (page - 1))) * S::kRowBytes;
        k_from[x] = (uint64_t)kp + from + (lkey * S::kRowBytes + k_piece);
        v_from[x] = (uint64_t)vp + from + (lkey * S::kRowBytes + v_piece);
      }
    } else if (k0 >= P && k0 + KT <= end) {
      size_t from = ((size_t)(w.row0 + k0 - P + wave * S::kKeysPerLoad) * Hkv + h) * S::kRowBytes;
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        k_from[x] = (uint64_t)kr + from + (lkey * row_bytes + k_piece);
        v_from[x] = (uint64_t)vr + from + (lkey * row_bytes + v_piece);
        from += (size_t)(NW * S::kKeysPerLoad) * row_bytes;
      }
    } else {  // the end of the prefix, the end of the keys, narrow pages: every key for itself
#pragma unroll
      for (int x = 0; x < S::kPer; ++x) {
        int pos = k0 + (wave + NW * x) * S::kKeysPerLoad + lkey;
        pos = pos < end ? pos : end - 1;
        const bool old = pos < P;
        size_t row = (size_t)(w.row0 + pos - P) * Hkv + h;
        if (old) row = ((size_t)page_at(pos >> page_shift) * Hkv + h) * page + (pos & (page - 1));
        k_from[x] = (uint64_t)(old ? kp : kr) + row * S::kRowBytes + k_piece;
        v_from[x] = (uint64_t)(old ? vp : vr) + row * S::kRowBytes + v_piece;
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
  f32x16 o[2][DT], s[2];
  bf16x8 kf[2][KS], vf[2][DT][2], pb[2][2];  // keys and values of an even and of an odd block: none is ever copied
  float ref[2], limit[2], l[2];  // base-2 reference of a row's scores, the unscaled score that it holds up to, sum of weights
  const float c1 = a.d.softmax_scale * kLog2e;
#pragma unroll 1
  for (int careful = 0;; careful = 1) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    ref[t] = 0.f;
    limit[t] = HB_NEG_INF;
    l[t] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[t][dt] = (f32x16)(0.f);
#pragma unroll
    for (int c = 0; c < 2; ++c) pb[t][c] = (bf16x8)((__bf16)0.f);
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int c = 0; c < 2; ++c) vf[0][dt][c] = (bf16x8)((__bf16)0.f);

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

  // masks, and the row's reference moved where a score has outgrown it; block of keys from k0
  auto settle = [&](int t, int k0, float top) {
    if (k0 + 31 > first_sees[t]) {  // uniform: some row does not see some key
      const int lim = sees[t] - k0 - 4 * hf;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = 8 * (r >> 2) + (r & 3) <= lim ? s[t][r] : HB_NEG_INF;
      top = max16(s[t]);
    }
    if (__any(!(top <= limit[t]))) {
      asm volatile("" ::: "memory");
      const float mx = half_max(top) * c1;
      const bool none = limit[t] == HB_NEG_INF;  // nothing accumulated yet
      const bool grow = mx > (none ? HB_NEG_INF : ref[t] + kSlack);
      const float next = grow ? mx : ref[t];
      const float alpha = none || !grow ? 1.f : __builtin_amdgcn_exp2f(ref[t] - mx);
      ref[t] = next;
      limit[t] = none && !grow ? HB_NEG_INF : (next + kSlack) / c1;
      l[t] *= alpha;
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[t][dt] *= alpha;
      }
    }
  };

  // One step: the scores of tile t (settled) become weights, while the matrix core makes the other tile's next scores (first)
  // and adds the other tile's last weights' products.  None needs what another makes, so that they can be laid side by side
  // by hand: an instruction of the matrix core (32 clocks), then a sixteenth of the vector work and of the reads from LDS,
  // and a fence for the scheduler, which would put them one behind the other.
  auto step = [&](auto T, const bf16x8 (&k)[KS], const bf16x8 (&v)[DT][2], float &top, auto read) {
    constexpr int t = decltype(T)::value, u = 1 - t, kAll = KS + 2 * DT, kEach = 16 / kAll;
    f32x16 sn, p;
    float m0 = 0.f, m1 = 0.f;
    uint32_t w[8];
#pragma unroll
    for (int x = 0; x < kAll; ++x) {
      __builtin_amdgcn_sched_barrier(0);
      if (x < KS)
        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[x], qf[u][x], x ? sn : (f32x16)(0.f), 0, 0, 0);
      else
        o[u][(x - KS) % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[(x - KS) % DT][(x - KS) / DT], pb[u][(x - KS) / DT], o[u][(x - KS) % DT], 0, 0, 0);
      read(x);
#pragma unroll
      for (int r = kEach * x; r < kEach * x + kEach; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], c1, -ref[t]));
        float y = p[r], sum = l[t];
        if (r > 0) sum += p[r - 1];
        if (r > 1 && r % 2 == 0) {
          uint32_t two = pack2(p[r - 2], p[r - 1]);
          asm volatile("" : "+v"(y), "+v"(sum), "+v"(two));
          w[r / 2 - 1] = two;
        } else {
          asm volatile("" : "+v"(y), "+v"(sum));
        }
        p[r] = y;
        l[t] = sum;
      }
      // the largest of the new scores, a sixth at a time
      if (x >= kAll - 3) {
        const int g = x - (kAll - 3);
        if (g == 0) {
          m0 = max3(sn[0], sn[1], sn[2]);
          m1 = max3(sn[3], sn[4], sn[5]);
        } else if (g == 1) {
          m0 = max3(m0, sn[6], sn[7]);
          m1 = max3(m1, sn[8], sn[9]);
        } else {
          m0 = max3(m0, sn[10], sn[11]);
          m1 = max3(m1, sn[12], sn[13]);
        }
        asm volatile("" : "+v"(m0), "+v"(m1));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    w[7] = pack2(p[14], p[15]);
    l[t] += p[15];
    pb[t][0] = __builtin_bit_cast(bf16x8, (u32x4){w[0], w[1], w[2], w[3]});
    pb[t][1] = __builtin_bit_cast(bf16x8, (u32x4){w[4], w[5], w[6], w[7]});
    s[u] = sn;
    top = fmaxf(max3(m0, sn[14], sn[15]), m1);
    asm volatile("" : "+v"(pb[t][0]), "+v"(pb[t][1]), "+v"(l[t]), "+v"(top));
  };

  // ---- the loop -----------------------------------------------------------------------------------------------------
#define HB_BARRIER() asm volatile("s_barrier" ::: "memory")
  constexpr int kKeep = 2 * S::kPer * (NS - 3);
  constexpr int kWait = (kKeep & 15) | ((kKeep >> 4) << 14) | (7 << 4) | (15 << 8);  // vmcnt alone
  constexpr int kWaitFirst = (2 * S::kPer * (NS - 2) & 15) | ((2 * S::kPer * (NS - 2) >> 4) << 14) | (7 << 4) | (15 << 8);
  fetch(0);
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) {
    place(i);
#pragma unroll
    for (int x = 0; x < 2 * S::kPer; ++x) load(i, x);
    fetch(i + 1);
  }
  __builtin_amdgcn_s_waitcnt(kWaitFirst);
  if (careful) clean(0);
  HB_BARRIER();
  float top;
#pragma unroll
  for (int q = 0; q < KS; ++q) kf[0][q] = one_k(k_at(smem, 0), q);
  s[0] = (f32x16)(0.f);
#pragma unroll
  for (int q = 0; q < KS; ++q) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0][q], qf[0][q], s[0], 0, 0, 0);
  top = max16(s[0]);
  settle(0, begin, top);

#pragma unroll 1
  for (int i = 0; i < n_tiles; ++i) {
    const unsigned char *st = smem + (i % NS) * S::kStage, *next = smem + ((i + 1) % NS) * S::kStage;
    const int k0 = begin + i * KT;
    const bool mine = i < my_tiles;
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) {
      if (b == S::kBlocks - 1) {
        // Tile i + 1 has landed, for everybody; and everybody is done with tile i - 1, whose stage takes tile i + NS - 1.
        __builtin_amdgcn_s_waitcnt(kWait);
        if (careful) clean(i + 1);
        HB_BARRIER();
        place(i + NS - 1);
        fetch(i + NS);
        if (!mine)
#pragma unroll
          for (int x = 0; x < 2 * S::kPer; ++x) load(i + NS - 1, x);
      }
      if (mine) {
        const int now = b, then = 1 - b;
        const unsigned char *pk = k_at(b == S::kBlocks - 1 ? next : st, (b + 1) % S::kBlocks), *pv = v_at(st, b);
        step(std::integral_constant<int, 0>(), kf[now], vf[now], top, [&](int x) {
          if (x < KS) kf[then][x] = one_k(pk, x);
          if (b == S::kBlocks - 1 && x < 2 * S::kPer) load(i + NS - 1, x);
        });
        settle(1, k0 + 32 * b, top);
        step(std::integral_constant<int, 1>(), kf[then], vf[then], top, [&](int x) {
          if (x < DT) vf[then][x][0] = one_v(pv, x, 0);
          else if (x < 2 * DT) vf[then][x - DT][1] = one_v(pv, x - DT, 1);
        });
        settle(0, k0 + 32 * b + 32, top);
      }
    }
  }
  // the last weights of the second tile
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[1][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[0][dt][c], pb[1][c], o[1][dt], 0, 0, 0);
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));  // loads past the end land before the workgroup gives up its LDS

  // Keys that a row does not see have weight 0 in the products, and 0 times a value that is not finite is no number.  Where
  // that, or anything else, has made results that are not finite, the workgroup does its part once more, `careful`: such
  // values of keys that some row does not see are zeros in LDS, and are added here to the rows that see them.  Rows that do
  // not get the bits that they get from any other value there.
  if (careful) {
    for (int kk = max(begin, all_see + 1); kk < end; ++kk) {  // a row of the prompt: the prefix is seen by all
      const bf16_t *vs = vr + ((size_t)(w.row0 + kk - P) * Hkv + h) * D;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (kk <= sees[t])
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float y = bf16_to_f32(vs[32 * dt + 8 * (r >> 2) + 4 * hf + (r & 3)]);
              if (!(fabsf(y) < __builtin_huge_valf())) o[t][dt][r] += y;
            }
    }
    break;
  }
  bool wrong = false;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) wrong |= !(fabsf(o[t][dt][r]) < __builtin_huge_valf());
  if (!__syncthreads_or(wrong && !no_rows)) break;
  }  // careful

  // ---- results ------------------------------------------------------------------------------------------------------
  // (the arguments are read again, so that the loop need not keep them in its registers)
  const PromptArgs &z = again(a);
  const int zHq = z.d.num_q_heads, zHkv = z.d.num_kv_heads, zG = zHq / zHkv;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float sum = half_sum(l[t]);
    const int r0 = wave * 64 + 32 * t + j, row = w.t * S::kRows + r0;
    if (row >= w.n * zG) continue;
    if (w.parts == 1) {
      const int token = row / zG;
      const size_t at = (size_t)(w.row0 + token) * zHq + (size_t)h * zG + (row - token * zG);
      const float inv = 1.f / sum;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          u32x2 x;
          x[0] = pack_bf16(o[t][dt][4 * g] * inv, o[t][dt][4 * g + 1] * inv);
          x[1] = pack_bf16(o[t][dt][4 * g + 2] * inv, o[t][dt][4 * g + 3] * inv);
          *(u32x2 *)((bf16_t *)z.out + at * D + 32 * dt + 8 * g + 4 * hf) = x;
        }
      if (z.lse && hf == 0) z.lse[at] = (ref[t] + log2f(sum)) * kLn2;
    } else {
      const size_t slot = (((size_t)(blockIdx.x / zHkv) * zHkv + h) * z.parts + blockIdx.y) * S::kRows + r0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 x;
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] = o[t][dt][4 * g + r];
          *(f32x4 *)(z.part_o + slot * D + 32 * dt + 8 * g + 4 * hf) = x;
        }
      if (hf == 0) {
        z.part_ml[slot * 2] = limit[t] == HB_NEG_INF ? HB_NEG_INF : ref[t];
        z.part_ml[slot * 2 + 1] = sum;
      }
    }
  }
#undef HB_BARRIER
}

template <int D, int NW, int KT, int NS>
hipError_t launch(const PromptArgs &a, hipStream_t s) {
  using S = Shape<D, NW, KT, NS>;
  auto kern = prompt_mfma_kernel<D, NW, KT, NS>;
  hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kLds);
  if (e != hipSuccess) return e;
  kern<<<dim3(a.tiles * a.d.num_kv_heads, a.parts), 64 * NW, S::kLds, s>>>(
      a, __builtin_ctz(a.d.page_size), (const bf16_t *)a.k, (const bf16_t *)a.v, (const bf16_t *)a.k_pool, (const bf16_t *)a.v_pool,
      a.block_table);
  e = hipGetLastError();
  if (e == hipSuccess && a.parts > 1) e = launch_prompt_join(a, S::kRows, KT, s);
  return e;
}

}  // namespace

bool prompt_mfma_supports(const hb_attn_desc &d) {
  return d.dtype == HB_BF16 && (d.head_dim == 64 || d.head_dim == 128) && (d.page_size & (d.page_size - 1)) == 0 &&
         d.softmax_scale > 0.f && d.softmax_scale < 1e30f;
}

int32_t prompt_mfma_rows(const hb_attn_desc &) { return 256; }

hipError_t launch_prompt_mfma(const PromptArgs &a, hipStream_t s) {
  return a.d.head_dim == 128 ? launch<128, 4, 64, 4>(a, s) : launch<64, 4, 64, 4>(a, s);
}

}  // namespace hb
