// hb_prompt_attn's kernel for every shape (prompt_any.h), and the join of the parts that a tile's keys were cut into.
#include "prompt_any.h"

namespace hb {

namespace {

template <typename T, int DP>
__global__ __launch_bounds__(256) void prompt_any_kernel(PromptArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int h = blockIdx.y;
  const PromptTile w = prompt_tile<kPromptAnyRows, kAnyKeys>(a, blockIdx.x, blockIdx.z);
  if (w.t < 0) return;
  prompt_any_rows<T, DP, 4>(a, w, h, w.t * kPromptAnyRows,
                            (((size_t)blockIdx.x * a.d.num_kv_heads + h) * a.parts + blockIdx.z) * kPromptAnyRows, lds);
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
// A thread has eight elements of a row.
template <typename T, int BM, int KEYS>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
  const int h = blockIdx.y, G = a.d.num_q_heads / a.d.num_kv_heads, D = a.d.head_dim, Hkv = a.d.num_kv_heads, pieces = D / 8;
  const PromptTile w = prompt_tile<BM, KEYS>(a, blockIdx.x, 0);
  if (w.t < 0 || w.parts == 1) return;
  const int64_t rows = (int64_t)w.n * G - (int64_t)w.t * BM;
  const int mine = (rows < BM ? (int)rows : BM) * pieces;
  for (int i = blockIdx.z * 256 + threadIdx.x; i < mine; i += gridDim.z * 256) {
    const int r = i / pieces, d0 = i % pieces * 8;
    const int64_t row = (int64_t)w.t * BM + r;
    const int64_t token = row / G;
    const size_t at = (size_t)(w.row0 + token) * a.d.num_q_heads + (size_t)h * G + (row - token * G);
    const size_t slot = (((size_t)blockIdx.x * Hkv + h) * a.parts) * BM + r;
    float m = HB_NEG_INF, l = 0.f, whole = 0.f, x[8] = {};
    for (int p = 0; p < w.parts; ++p) m = fmaxf(m, a.part_ml[(slot + (size_t)p * BM) * 4]);
    for (int p = 0; p < w.parts; ++p) {
      const size_t s = slot + (size_t)p * BM;
      const f32x4 ml = *(const f32x4 *)(a.part_ml + s * 4);
      if (ml[0] == HB_NEG_INF && ml[1] == 0.f) continue;  // sees none of this part's keys
      const float c = exp2_of(ml[0] - m);
      float y[8];
      load8(a.part_o + s * D + d0, y);
      l += c * ml[1];
      whole += c * ml[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += c * y[e];
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) store_f32((T *)a.out + at * D + d0 + e, x[e] * inv);
    if (a.lse && d0 == 0) a.lse[at] = (m + log2f(whole)) * kLn2;
  }
}

template <int BM, int KEYS>
hipError_t join(const PromptArgs &a, hipStream_t s) {
  // a thread for two pieces or fewer
  const dim3 grid(a.tiles, a.d.num_kv_heads, (BM * (a.d.head_dim / 8) + 511) / 512);
  if (a.d.dtype == HB_F32)
    prompt_join_kernel<float, BM, KEYS><<<grid, 256, 0, s>>>(a);
  else
    prompt_join_kernel<bf16_t, BM, KEYS><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

static hipError_t go(const PromptArgs &a, hipStream_t s) {
  const int D = a.d.head_dim;
  if (a.d.dtype == HB_F32) return D <= 64 ? launch_any<float, 64>(a, s) : D <= 128 ? launch_any<float, 128>(a, s) : launch_any<float, 256>(a, s);
  return D <= 64 ? launch_any<bf16_t, 64>(a, s) : D <= 128 ? launch_any<bf16_t, 128>(a, s) : launch_any<bf16_t, 256>(a, s);
}

hipError_t launch_prompt_any(const PromptArgs &a, hipStream_t s) {
  hipError_t e = go(a, s);
  if (e == hipSuccess && a.parts > 1) e = join<kPromptAnyRows, kAnyKeys>(a, s);
  return e;
}

hipError_t launch_prompt_join(const PromptArgs &a, int32_t rows, int32_t keys, hipStream_t s) {
  if (rows == 256) return join<256, 64>(a, s);
  return keys == 64 ? join<128, 64>(a, s) : join<64, 32>(a, s);
}

}  // namespace hb
