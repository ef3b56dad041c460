// hb_prompt_attn's kernel for every shape (prompt_any.h), and the join of the parts that a tile's keys were cut into.
#include "prompt_any.h"

namespace hb {

namespace {

template <typename T, int DP>
__global__ __launch_bounds__(256) void prompt_any_kernel(PromptArgs a) {
  constexpr int kRows = kPromptAnyRows;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int h = blockIdx.y;
  const PromptTile w = prompt_tile<kRows, kAnyKeys>(a, blockIdx.x, blockIdx.z);
  prompt_head<kRows>(a, w, blockIdx.x, h, blockIdx.z);
  if (w.t < 0) return;
  prompt_any_rows<T, DP>(a, w, h, w.t * kRows, (((size_t)blockIdx.x * a.d.num_kv_heads + h) * a.parts + blockIdx.z) * kRows, lds);
}

template <typename T, int DP>
hipError_t launch_any(const PromptArgs &a, hipStream_t s) {
  constexpr int kBytes = any_lds_floats<DP> * 4;
  auto kern = prompt_any_kernel<T, DP>;
  hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (e != hipSuccess) return e;
  kern<<<dim3(a.tiles, a.d.num_kv_heads, a.parts), 256, kBytes, s>>>(a);
  return hipGetLastError();
}

// out = sum of the parts' results, each scaled by 2^(its largest score - the largest of all), over the like sum of their sums.
// A thread has eight elements of a row, and four parts of them under way.  The time of a call is that of a few dependent reads, so
// what there is to do is read (PromptArgs::heads), not found out again: 14 -> 8 us for 64 rows over 8 K in four parts.  MANY: a
// row by a wavefront, whose lanes share its parts (a call with one token over 16 K, 28/4 heads, 36.5 -> 29.6 us; in float32 50 -> 19.7).
template <typename T, bool MANY>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a, int bm) {
  const PromptArgs::Head t = a.heads[blockIdx.x];
  if (t.parts <= 1) return;
  const int h = blockIdx.y, G = a.d.num_q_heads / a.d.num_kv_heads, D = a.d.head_dim, Hkv = a.d.num_kv_heads, pieces = D / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int width = MANY ? pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32 : 1;  // lanes that have one part's row
  const int groups = MANY ? 64 / width : 1, group = MANY ? lane / width : 0;
  const int end = MANY ? t.rows : t.rows * pieces, step = MANY ? gridDim.z * 4 : gridDim.z * 256;
  for (int i = MANY ? blockIdx.z * 4 + wave : blockIdx.z * 256 + threadIdx.x; i < end; i += step) {
    const int r = MANY ? i : i / pieces, piece = MANY ? lane % width : i % pieces, d0 = min(piece, pieces - 1) * 8;
    const int row = t.first + r, token = row / G;
    const size_t at = (size_t)(t.row0 + token) * a.d.num_q_heads + (size_t)h * G + (row - token * G);
    const size_t slot = (((size_t)blockIdx.x * Hkv + h) * a.parts) * bm + r;
    constexpr float kShare = 1.f / 512;  // 256 results at most that are finite each: their sum is
    float m = HB_NEG_INF, l = 0.f, whole = 0.f, x[8] = {};
    for (int p0 = group; p0 < t.parts; p0 += 4 * groups) {
      f32x4 ml[4];
      float y[4][8];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const size_t s = slot + (size_t)min(p0 + p * groups, t.parts - 1) * bm;
        ml[p] = *(const f32x4 *)(a.part_ml + s * 4);
        load8(a.part_o + s * D + d0, y[p]);
      }
      const float top = fmaxf(fmaxf(fmaxf(m, ml[0][0]), fmaxf(ml[1][0], ml[2][0])), ml[3][0]);  // (the last one again: no matter)
      const float alpha = m == top ? 1.f : exp2_of(m - top);
      m = top;
      l *= alpha;
      whole *= alpha;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= alpha;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        if (p0 + p * groups >= t.parts || (ml[p][0] == HB_NEG_INF && ml[p][1] == 0.f)) continue;  // ... or it sees none of this part's keys
        const float c = exp2_of(ml[p][0] - m);
        l += kShare * c * ml[p][1];
        whole += c * ml[p][2];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += kShare * c * y[p][e];
      }
    }
    if (MANY) {
      for (int other = width; other < 64; other <<= 1) {
        const float m2 = __shfl_xor(m, other, 64), top = fmaxf(m, m2);
        const float c = m == top ? 1.f : exp2_of(m - top), c2 = m2 == top ? 1.f : exp2_of(m2 - top);
        m = top;
        l = c * l + c2 * __shfl_xor(l, other, 64);
        whole = c * whole + c2 * __shfl_xor(whole, other, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = c * x[e] + c2 * __shfl_xor(x[e], other, 64);
      }
      if (group > 0 || piece >= pieces) continue;
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    store8((T *)a.out + at * D + d0, x);
    if (a.lse && d0 == 0) a.lse[at] = (m + log2f(whole)) * kLn2;
  }
}

}  // namespace

template <typename T>
static hipError_t go(const PromptArgs &a, hipStream_t s) {
  const int D = a.d.head_dim;
  return D <= 64 ? launch_any<T, 64>(a, s) : D <= 128 ? launch_any<T, 128>(a, s) : launch_any<T, 256>(a, s);
}

hipError_t launch_prompt_any(const PromptArgs &a, hipStream_t s) {
  hipError_t e = a.d.dtype == HB_F32 ? go<float>(a, s) : go<bf16_t>(a, s);
  if (e == hipSuccess && a.parts > 1) e = launch_prompt_join(a, kPromptAnyRows, s);
  return e;
}

hipError_t launch_prompt_join(const PromptArgs &a, int32_t rows, hipStream_t s) {
  // a thread for two pieces or fewer, or a wavefront for eight rows
  const bool many = a.parts > 16;
  const dim3 grid(a.tiles, a.d.num_kv_heads, many ? (rows + 31) / 32 : (rows * (a.d.head_dim / 8) + 511) / 512);
  if (a.d.dtype == HB_F32)
    (many ? prompt_join_kernel<float, true> : prompt_join_kernel<float, false>)<<<grid, 256, 0, s>>>(a, rows);
  else
    (many ? prompt_join_kernel<bf16_t, true> : prompt_join_kernel<bf16_t, false>)<<<grid, 256, 0, s>>>(a, rows);
  return hipGetLastError();
}

}  // namespace hb
