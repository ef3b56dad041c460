// Attention of prompts for every shape and type (hb_prompt_attn): float32 throughout, on the float32 matrix instructions.
//
// One workgroup owns one tile of 64 rows (prompt.h) and one part of its keys; four wavefronts with sixteen rows each share
// the keys, 32 at a time, widened to float32 in LDS.  As in the bf16 kernels the products are transposed, so that no score
// crosses lanes between them:
//   S^T = K Q^T     16x16x4: A = 16 keys x 4 of D, B = 4 of D x 16 rows
//   O^T = V^T P^T   16x16x4: A = 16 of D x 4 keys, B = 4 keys x 16 rows
// The accumulator of lane (j, g), j = lane % 16, g = lane / 16, holds row j's scores for keys 4g + r, r = 0..3: what the
// r-th instruction of the second product wants in that lane when its four keys are r, 4 + r, 8 + r, 12 + r.
// Softmax is online per row in base 2.  Rows of K and V are four floats apart from a multiple of 64 in LDS: no operand read
// has a bank conflict.  A head dimension between the sizes built here is filled up with zeros.
#pragma once
#include "prompt.h"

namespace hb {

namespace {

constexpr int kAnyKeys = 32;
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
__device__ __forceinline__ void load8(const bf16_t *p, float (&x)[8]) {
  const u32x4 w = *(const u32x4 *)p;
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// Rows first .. first + 16 NW - 1 of (sequence, kv head h) by NW wavefronts, which all call it: their keys w.begin .. w.end - 1,
// to the results, or to the partial results from `slot0` on.  lds: any_lds_floats<DP>.
template <int DP>
constexpr int any_lds_floats = 2 * kAnyKeys * (DP + 4) + 4;

__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
  *(f32x4 *)p = (f32x4){x[0], x[1], x[2], x[3]};
  *(f32x4 *)(p + 4) = (f32x4){x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&x)[8]) {
  *(u32x4 *)p = (u32x4){pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

template <typename T, int DP, int NW>
__device__ __forceinline__ void prompt_any_rows(const PromptArgs &a, const PromptTile &w, int h, int first, size_t slot0, float *lds) {
  constexpr int kKeys = kAnyKeys, kRow = DP + 4, kTiles = DP / 16, kSteps = DP / 4, kPieces = DP / 8;
  float *lk = lds, *lv = lds + kKeys * kRow;
  int &bad = *(int *)(lds + 2 * kKeys * kRow);  // a value of this tile's is left out, see below
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j = lane & 15, kg = lane >> 4;
  const int G = a.d.num_q_heads / a.d.num_kv_heads, D = a.d.head_dim, Hkv = a.d.num_kv_heads;

  const int row = first + wave * 16 + j;
  const bool there = (int64_t)row < (int64_t)w.n * G;
  const int token = there ? row / G : w.n - 1, head = there ? row - token * G : 0;
  const size_t at = (size_t)(w.row0 + token) * a.d.num_q_heads + (size_t)h * G + head;
  const int sees = w.P + token;  // the last key of this row
  const int all_see = w.P + first / G;  // ... and of the first

  float qf[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) qf[s] = there && 4 * s + kg < D ? load_f32((const T *)a.q + at * D + 4 * s + kg) : 0.f;
  f32x4 o[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) o[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
  float m = HB_NEG_INF, l = 0.f;
  const float c1 = a.d.softmax_scale * kLog2e;

  for (int k0 = w.begin; k0 < w.end; k0 += kKeys) {
    __syncthreads();
    if (tid == 0) bad = 0;
    __syncthreads();
    for (int i = tid; i < kKeys * kPieces; i += 64 * NW) {
      const int key = i / kPieces, d0 = i % kPieces * 8, kk = k0 + key;
      float x[8] = {}, y[8] = {};
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
        load8(ks + from + d0, x);
        load8(vs + from + d0, y);
      }
      // a key that some row does not see has weight 0 there, and 0 times a value that is not finite is none: such values
      // are added below, to the rows that see them
      if (kk > all_see) {
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

    f32x4 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(lk[(16 * t + j) * kRow + 4 * s + kg], qf[s], sc[t], 0, 0, 0);
    }
    // masked scores are replaced before anything is made of them
    float top = HB_NEG_INF;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int kk = k0 + 16 * t + 4 * kg + r;
        sc[t][r] = kk <= sees && kk < w.end ? sc[t][r] * c1 : HB_NEG_INF;
        top = fmaxf(top, sc[t][r]);
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
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = exp2_of(sc[t][r] - ref);
        l += p;
        const float *vr = lv + (16 * t + 4 * kg + r) * kRow + j;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[16 * dt], p, o[dt], 0, 0, 0);
      }
    if (bad) {  // every thread's: it is set in front of a barrier
      const int last = min(min(sees, w.end - 1), k0 + kKeys - 1);
      for (int kk = max(k0, all_see + 1); kk <= last; ++kk) {  // prompt rows: the prefix is seen by all
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

  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (!there) return;
  if (w.parts == 1) {
    const float inv = 1.f / l;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = 16 * dt + 4 * kg + r;
        if (d < D) store_f32((T *)a.out + at * D + d, o[dt][r] * inv);
      }
    if (a.lse && kg == 0) a.lse[at] = (m + log2f(l)) * kLn2;
  } else {
    const size_t slot = slot0 + wave * 16 + j;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = 16 * dt + 4 * kg + r;
        if (d < D) a.part_o[slot * D + d] = o[dt][r];
      }
    if (kg == 0) {
      *(f32x4 *)(a.part_ml + slot * 4) = (f32x4){m, l, l, 0.f};
    }
  }
}

}  // namespace

}  // namespace hb
