// Attention of prompts for every shape and type (hb_prompt_attn): float32 throughout, on the float32 matrix instructions.
//
// One workgroup owns one tile of 16 rows (prompt.h) and one part of its keys.  64 keys at a time are widened to float32 in LDS,
// the next ones under way to registers meanwhile; each of four wavefronts has sixteen of them, and its own softmax and result of
// the rows, which are joined in LDS at the end.  As in the bf16 kernels the products are transposed, so that no score crosses
// lanes between them:
//   S^T = K Q^T     16x16x4: A = 16 keys x 4 of D, B = 4 of D x 16 rows
//   O^T = V^T P^T   16x16x4: A = 16 of D x 4 keys, B = 4 keys x 16 rows
// The accumulator of lane (j, g), j = lane % 16, g = lane / 16, holds row j's scores for keys 4g + r, r = 0..3: what the
// r-th instruction of the second product wants in that lane when its four keys are r, 4 + r, 8 + r, 12 + r.
// What bounds it: for heads of 64 a tile's products are 32 matrix instructions of 32 clocks for each wavefront, 0.5 us; the tile takes 2
// alone on a CU (pages, keys, LDS and the softmax between the products, one behind the other), and several workgroups on a CU
// fill each other's gaps, up to what L2 gives: every 16 rows bring all keys.  4 heads of 64 on one of keys: 2 prompts of 200 to 256
// rows 11.6 us; one of 2048 rows 65, of 8192 510 (68 TFLOP/s of the 153 that a large float32 product has).  With sixteen rows for each
// wavefront, which share the keys, the first two are 20.3 (four times fewer workgroups, and a join of parts) and 72.  Page ids asked for a
// tile ahead: one row over 16 K whole 533 -> 441 us, but the prompts 12.8 and 70, and 8192 rows with heads of 128 1056 -> 1701.
// Softmax is online per row in base 2.  Rows of K and V are four floats apart from a multiple of 64 in LDS: no operand read
// has a bank conflict.  A head dimension between the sizes built here is filled up with zeros.
#pragma once
#include "prompt.h"

namespace hb {

namespace {

constexpr int kAnyKeys = 64;  // of a tile
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
#define HB_NEG_INF (-__builtin_huge_valf())

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
  const f32x4 lo = *(const f32x4 *)p, hi = *(const f32x4 *)(p + 4);
  for (int i = 0; i < 4; ++i) {
    x[i] = lo[i];
    x[4 + i] = hi[i];
  }
}
template <int DP>
constexpr int any_lds_floats = 2 * kAnyKeys * (DP + 4) + 4;

__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
  *(f32x4 *)p = (f32x4){x[0], x[1], x[2], x[3]};
  *(f32x4 *)(p + 4) = (f32x4){x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&x)[8]) {
  *(u32x4 *)p = (u32x4){pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

// 16 bytes or 32 of K or V as they are in memory
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  f32x4 lo, hi;
  __device__ __forceinline__ void load(const float *p) {
    lo = *(const f32x4 *)p;
    hi = *(const f32x4 *)(p + 4);
  }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = lo[i];
      x[4 + i] = hi[i];
    }
  }
};
template <>
struct Raw<bf16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t *p) { w = *(const u32x4 *)p; }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};

// Rows first .. first + 15 of (sequence, kv head h) by four wavefronts, which all call it: their keys w.begin .. w.end - 1, to the
// results, or to the partial results from `slot0` on.  lds: any_lds_floats<DP>.
template <typename T, int DP>
__device__ __forceinline__ void prompt_any_rows(const PromptArgs &a, const PromptTile &w, int h, int first, size_t slot0, float *lds) {
  constexpr int kKeys = kAnyKeys, kRow = DP + 4, kTiles = DP / 16, kSteps = DP / 4, kPieces = DP / 8, kAsks = kKeys * kPieces / 256;
  float *lk = lds, *lv = lds + kKeys * kRow;
  int &bad = *(int *)(lds + 2 * kKeys * kRow);  // a value of this tile's is left out, see below
  int &anew = *(int *)(lds + 2 * kKeys * kRow + 1);  // rows (a bit each) that are done once more, see below
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j = lane & 15, kg = lane >> 4;
  const int G = a.d.num_q_heads / a.d.num_kv_heads, D = a.d.head_dim, Hkv = a.d.num_kv_heads;
  const int own = wave * 16;  // this wavefront's first key of a tile

  const int row = first + j;
  const bool there = (int64_t)row < (int64_t)w.n * G;
  const int token = there ? row / G : w.n - 1, head = there ? row - token * G : 0;
  const size_t at = (size_t)(w.row0 + token) * a.d.num_q_heads + (size_t)h * G + head;
  const int sees = w.P + token;  // the last key of this row
  const int all_see = w.P + first / G;  // ... and of the first

  float qf[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) qf[s] = there && 4 * s + kg < D ? load_f32((const T *)a.q + at * D + 4 * s + kg) : 0.f;
  f32x4 o[kTiles];
  float m, l;
  const float c1 = a.d.softmax_scale * kLog2e;

  // the next tile is on its way to registers while this one is worked on
  const int key0 = tid / kPieces, d0 = tid % kPieces * 8;
  Raw<T> kx[kAsks], vx[kAsks];
  auto ask = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kAsks; ++i) {
      const int kk = k0 + key0 + i * (256 / kPieces);
      kx[i] = vx[i] = Raw<T>{};
      if (kk < w.end && d0 < D) {
        const T *ks, *vs;
        size_t from;
        if (kk < w.P) {
          const int page = kk / a.d.page_size;
          int id = a.block_table[(size_t)w.b * a.d.max_blocks_per_seq + page];
          id = id < 0 ? 0 : id >= a.d.num_blocks ? a.d.num_blocks - 1 : id;
          from = (((size_t)id * Hkv + h) * a.d.page_size + (kk - page * a.d.page_size)) * D;
          ks = (const T *)a.k_pool;
          vs = (const T *)a.v_pool;
        } else {
          from = ((size_t)(w.row0 + kk - w.P) * Hkv + h) * D;
          ks = (const T *)a.k;
          vs = (const T *)a.v;
        }
        kx[i].load(ks + from + d0);
        vx[i].load(vs + from + d0);
      }
    }
  };

  // Weights of at most 1, times values near float32's largest, may have a sum that is beyond it where their mean is not.  Where
  // a wavefront's results of a row are not finite, the tile is done once more: such a row's weights are 2^raise times smaller
  // then, so that their sum is a half at most; the others are as they were.  (A value that is not finite comes here for nothing.)
  if (tid == 0) anew = 0;
  float raise = 0.f, smaller = 1.f;
  for (int again = 0;; ++again) {
  ask(w.begin);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) o[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
  m = HB_NEG_INF;
  l = 0.f;
#pragma unroll 1
  for (int k0 = w.begin; k0 < w.end; k0 += kKeys) {
    __syncthreads();
    if (tid == 0) bad = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAsks; ++i) {
      const int key = key0 + i * (256 / kPieces);
      float x[8], y[8];
      kx[i].widen(x);
      vx[i].widen(y);
      // a key that some row does not see has weight 0 there, and 0 times a value that is not finite is none: such values
      // are added below, to the rows that see them
      if (k0 + key > all_see) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(fabsf(y[e]) < __builtin_huge_valf())) {
            y[e] = 0.f;
            bad = 1;
          }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lk[key * kRow + d0 + e] = x[e];
        lv[key * kRow + d0 + e] = y[e];
      }
    }
    __syncthreads();
    ask(k0 + kKeys);

    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(lk[(own + j) * kRow + 4 * s + kg], qf[s], sc, 0, 0, 0);
    // masked scores are replaced before anything is made of them
    float top = HB_NEG_INF;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int kk = k0 + own + 4 * kg + r;
      sc[r] = kk <= sees && kk < w.end ? sc[r] * c1 : HB_NEG_INF;
      top = fmaxf(top, sc[r]);
    }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float next = fmaxf(m, top), ref = next == HB_NEG_INF ? 0.f : next;
    const float alpha = m == next ? 1.f : exp2_of(m - ref);  // m may be -infinity: nothing so far
    m = next;
    l *= alpha;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) o[t] *= alpha;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = exp2_of(sc[r] - ref) * smaller;
      l += p;
      const float *vr = lv + (own + 4 * kg + r) * kRow + j;
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[16 * dt], p, o[dt], 0, 0, 0);
    }
    if (bad) {  // every thread's: it is set in front of a barrier
      const int last = min(min(sees, w.end - 1), k0 + own + 15);
      for (int kk = max(k0 + own, all_see + 1); kk <= last; ++kk) {  // prompt rows: the prefix is seen by all
        const T *vs = (const T *)a.v + ((size_t)(w.row0 + kk - w.P) * Hkv + h) * D;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = 16 * dt + 4 * kg + r;
            const float y = d < D ? load_f32(vs + d) : 0.f;
            if (!(fabsf(y) < __builtin_huge_valf())) o[dt][r] += y;
          }
      }
    }
  }

  if (again) {
    __syncthreads();
    break;
  }
  float none = 0.f;  // or no number
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) none = fmaf(o[t][r], 0.f, none);
  const unsigned long long lanes = __ballot(there && none != none);  // four lanes share a row
  if (lanes && lane == 0) atomicOr(&anew, (int)((lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffff));
  __syncthreads();
  if (anew == 0) break;
  if (anew >> j & 1) {
    const int more = 33 - __builtin_clz(w.end - w.begin);  // 2^more is more than twice the keys
    raise = (float)more;
    smaller = __uint_as_float((uint32_t)(127 - more) << 23);
  }
  }

  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  // one result of the wavefronts': through LDS, where the keys were
  float *lo = lds, *ml = lds + 64 * kRow;  // [wavefront][row]
#pragma unroll
  for (int dt = 0; dt < kTiles; ++dt) *(f32x4 *)(lo + (wave * 16 + j) * kRow + 16 * dt + 4 * kg) = o[dt];
  if (kg == 0) {
    ml[2 * (wave * 16 + j)] = m + raise;
    ml[2 * (wave * 16 + j) + 1] = l;
  }
  __syncthreads();
  float scale[4], most = HB_NEG_INF, sum = 0.f;
  const int r = tid >> 4, of = tid & 15;  // this thread's row, and its pieces of eight: of, of + 16
#pragma unroll
  for (int v = 0; v < 4; ++v) most = fmaxf(most, ml[2 * (16 * v + r)]);
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float mv = ml[2 * (16 * v + r)], lv = ml[2 * (16 * v + r) + 1];
    scale[v] = mv == HB_NEG_INF && lv == 0.f ? 0.f : exp2_of(mv - most);  // 0: sees none of those keys
    sum += scale[v] * lv;
  }
  const int mine = first + r, t2 = mine / G;
  if ((int64_t)mine >= (int64_t)w.n * G) return;
  const size_t to = (size_t)(w.row0 + t2) * a.d.num_q_heads + (size_t)h * G + (mine - t2 * G);
  // four results that are finite each: quarters of them, and of what divides them
  const float inv = w.parts == 1 ? 1.f / (0.25f * sum) : 1.f;
  for (int d0 = 8 * of; d0 < D; d0 += 128) {
    float x[8] = {};
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += 0.25f * scale[v] * lo[(v * 16 + r) * kRow + d0 + e];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    if (w.parts == 1)
      store8((T *)a.out + to * D + d0, x);
    else
      store8(a.part_o + (slot0 + r) * D + d0, x);
  }
  if (of == 0 && w.parts > 1) *(f32x4 *)(a.part_ml + (slot0 + r) * 4) = (f32x4){most, 0.25f * sum, sum, 0.f};
  if (of == 0 && w.parts == 1 && a.lse) a.lse[to] = (most + log2f(sum)) * kLn2;
}

}  // namespace

}  // namespace hb
