// A request's sampling rules applied to the logits of its tree's nodes (hb_rules_logits, hb_rules_probs, hb_rules_count).
//
//   c = how often the request has had the token, those on the node's own path below the root included
//   z = logit;  c > 0 or in the prompt: z / repetition where z > 0, else z * repetition
//   z = z - (presence [c > 0] + frequency c) + bias;  -infinity where the grammar forbids the token, or z is no number
//   p = exp((z - max z) / temperature) / sum;  temperature 0: 1 for the largest z, the lowest token among equals
//
// A workgroup has a chunk of a row.  Counts and masks are as long as the row and are read beside it; the few tokens of the path
// and of the biases are marked in a bitmap of the chunk in LDS, and a thread that meets a mark looks the token up in lists that
// are there too.  In float32, in the order that is written above, without contraction: two sides that follow it agree
// about which z is the largest.
#include "rules.h"

namespace hb {

namespace {

#pragma clang fp contract(off)

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kStep = kThreads * 8, kMostChunk = 32768, kBiases = 1024;
constexpr float kLog2e = 1.4426950408889634f;
#define HB_INF __builtin_huge_valf()

struct Row {
  int b, path;               // sequence (-1: nobody's row); tokens on the path
  int bias0, biases;
  float temperature, repetition, presence, frequency;
  const int32_t *counts;     // of its sequence, or null
  const uint8_t *mask;       // bytes of its mask, or null
};

struct RowLds {
  uint32_t marked[kMostChunk / 32];
  int32_t path[64];
  int32_t bias_id[kBiases];
  float bias_value[kBiases];
  int32_t found[4];
};

// The row's rules, and the marks of its chunk [v0, v1).  Every thread calls it; ends with a barrier.
__device__ __forceinline__ Row row_of(const RulesArgs &a, int t, int v0, int v1, RowLds &s) {
  const int tid = threadIdx.x, lane = tid & 63;
  Row r;
  r.b = -1;
  r.path = 0;
  int n0 = 0, nodes = 0;
  if (!a.node_offset) {
    r.b = t;
  } else {
    if (tid == 0) s.found[0] = -1;
    __syncthreads();
    for (int b = tid; b < a.batch; b += kThreads) {
      const int lo = a.node_offset[b], hi = a.node_offset[b + 1];
      if (lo >= 0 && lo <= t && t < hi) s.found[0] = b;  // one at most, of offsets that do not fall
    }
    __syncthreads();
    r.b = s.found[0];
    if (r.b < 0) return r;
    n0 = a.node_offset[r.b];
    nodes = min(min(a.node_offset[r.b + 1], a.rows) - n0, a.max_nodes);
  }
  r.temperature = r.repetition = 1.f;
  r.presence = r.frequency = 0.f;
  if (a.rules) {
    const f32x4 x = *(const f32x4 *)(a.rules + (size_t)r.b * 4);
    r.temperature = x[0];
    r.repetition = x[1];
    r.presence = x[2];
    r.frequency = x[3];
  }
  r.counts = a.counts ? a.counts + (size_t)r.b * a.V : nullptr;
  r.mask = nullptr;
  if (a.mask) {
    const int m = a.mask_row ? a.mask_row[t] : t;
    if (m >= 0 && m < a.num_masks) r.mask = (const uint8_t *)(a.mask + (size_t)m * ((a.V + 31) / 32));
  }
  r.bias0 = r.biases = 0;
  if (a.bias_offset) {
    const int lo = a.bias_offset[r.b], hi = a.bias_offset[r.b + 1];
    if (lo >= 0 && hi > lo && hi <= a.n_bias) {
      r.bias0 = lo;
      r.biases = hi - lo;
    }
  }
  for (int i = tid; i < (v1 - v0 + 31) / 32; i += kThreads) s.marked[i] = 0;
  if (tid < 64) {
    // the path: parents and tokens a lane each, walked by reading lanes
    int n = 0;
    const int node = t - n0;
    if (a.node_offset && a.parent && node < nodes) {
      const int par = lane < nodes ? a.parent[n0 + lane] : -1, token = lane < nodes ? a.draft_ids[n0 + lane] : -1;
      int at = node;
      for (int guard = 0; guard < 64; ++guard) {
        const int up = __builtin_amdgcn_readlane(par, at);
        if (up < 0 || up >= at) break;  // the root (or a malformed parent)
        const int x = __builtin_amdgcn_readlane(token, at);
        if (lane == 0) s.path[n] = x;
        ++n;
        at = up;
      }
    }
    if (lane == 0) s.found[1] = n;
  }
  for (int i = tid; i < min(r.biases, kBiases); i += kThreads) {
    s.bias_id[i] = a.bias_id[r.bias0 + i];
    s.bias_value[i] = a.bias_value[r.bias0 + i];
  }
  __syncthreads();
  r.path = s.found[1];
  auto mark = [&](int v) {
    if (v >= v0 && v < v1) atomicOr(&s.marked[(v - v0) >> 5], 1u << ((v - v0) & 31));
  };
  if (tid < r.path) mark(s.path[tid]);
  for (int i = tid; i < r.biases; i += kThreads) mark(i < kBiases ? s.bias_id[i] : a.bias_id[r.bias0 + i]);
  __syncthreads();
  return r;
}

// Eight tokens' values; `allowed` and `marked`: a bit each
__device__ __forceinline__ void apply(const RulesArgs &a, const Row &r, const RowLds &s, int v, const int (&count)[8], uint32_t allowed,
                                      uint32_t marked, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    int c = count[e];
    float bias = 0.f;
    const bool hit = marked >> e & 1u;
    if (c != 0 || hit) {
      bool seen = c & kPromptFlag;
      c &= kPromptFlag - 1;
      if (hit) {
        for (int i = 0; i < r.path; ++i) c += s.path[i] == v + e;
        for (int i = 0; i < r.biases; ++i) {
          const int id = i < kBiases ? s.bias_id[i] : a.bias_id[r.bias0 + i];
          if (id == v + e) bias += i < kBiases ? s.bias_value[i] : a.bias_value[r.bias0 + i];
        }
      }
      seen |= c > 0;
      if (seen) z[e] = z[e] > 0.f ? z[e] / r.repetition : z[e] * r.repetition;
      z[e] = z[e] - ((c > 0 ? r.presence : 0.f) + r.frequency * (float)c);
      z[e] = z[e] + bias;
    }
    if (!(allowed >> e & 1u) || !(z[e] == z[e])) z[e] = -HB_INF;
  }
}

template <typename T, bool WHOLE>
__device__ __forceinline__ void load_eight(const T *p, int n, float (&z)[8]);
template <>
__device__ __forceinline__ void load_eight<float, true>(const float *p, int, float (&z)[8]) {
  const f32x4 lo = *(const f32x4 *)p, hi = *(const f32x4 *)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[e] = lo[e];
    z[4 + e] = hi[e];
  }
}
template <>
__device__ __forceinline__ void load_eight<bf16_t, true>(const bf16_t *p, int, float (&z)[8]) {
  const u32x4 w = *(const u32x4 *)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[2 * e] = __uint_as_float(w[e] << 16);
    z[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void load_eight<float, false>(const float *p, int n, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = e < n ? p[e] : -HB_INF;
}
template <>
__device__ __forceinline__ void load_eight<bf16_t, false>(const bf16_t *p, int n, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = e < n ? bf16_to_f32(p[e]) : -HB_INF;
}

template <bool WHOLE>
__device__ __forceinline__ void store_eight(float *p, int n, const float (&z)[8]) {
  if (WHOLE) {
    *(f32x4 *)p = (f32x4){z[0], z[1], z[2], z[3]};
    *(f32x4 *)(p + 4) = (f32x4){z[4], z[5], z[6], z[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = z[e];
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store_eight(bf16_t *p, int n, const float (&z)[8]) {
  if (WHOLE) {
    *(u32x4 *)p = (u32x4){pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = f32_to_bf16(z[e]);
  }
}

// The adjusted values of tokens v .. v + 7 of row t; WHOLE: rows are a multiple of eight long, and pieces aligned
template <typename T, bool WHOLE>
__device__ __forceinline__ void values(const RulesArgs &a, const Row &r, const RowLds &s, int t, int v, int v0, float (&z)[8]) {
  const int n = a.V - v;
  load_eight<T, WHOLE>((const T *)a.logits + (size_t)t * a.V + v, n, z);
  int count[8] = {};
  if (r.counts) {
    if (WHOLE) {
      const u32x4 lo = *(const u32x4 *)(r.counts + v), hi = *(const u32x4 *)(r.counts + v + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        count[e] = (int)lo[e];
        count[4 + e] = (int)hi[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) count[e] = e < n ? r.counts[v + e] : 0;
    }
  }
  const uint32_t allowed = r.mask ? r.mask[v >> 3] : 0xffu;
  const uint32_t marked = s.marked[(v - v0) >> 5] >> ((v - v0) & 31) & 0xffu;
  apply(a, r, s, v, count, allowed, marked, z);
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rules_logits_kernel(RulesArgs a) {
  __shared__ RowLds s;
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of(a, t, v0, v1, s);
  if (r.b < 0) return;
  for (int v = v0 + (int)threadIdx.x * 8; v < v1; v += kStep) {
    float z[8];
    values<T, WHOLE>(a, r, s, t, v, v0, z);
    store_eight<WHOLE>((T *)a.out + (size_t)t * a.V + v, a.V - v, z);
  }
}

// largest value, the lowest token that has it, and the sum of 2^((z - largest) k)
struct Stat {
  float top, sum;
  int token;
};
__device__ __forceinline__ float weight_of(float z, float top, float k) {
  const float d = z == top ? 0.f : z - top;  // also where both are infinite
  return z > -HB_INF ? __builtin_amdgcn_exp2f(d * k) : 0.f;
}
__device__ __forceinline__ Stat joined(const Stat &x, const Stat &y, float k) {
  Stat j;
  const bool second = y.top > x.top || (y.top == x.top && y.token < x.token);
  j.top = second ? y.top : x.top;
  j.token = second ? y.token : x.token;
  j.sum = x.sum * weight_of(x.top, j.top, k) + y.sum * weight_of(y.top, j.top, k);
  return j;
}
__device__ __forceinline__ float slope_of(const Row &r) {
  return r.temperature > 0.f ? fminf(kLog2e / r.temperature, 3e38f) : 0.f;
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rules_stats_kernel(RulesArgs a) {
  __shared__ RowLds s;
  __shared__ Stat waves[kThreads / 64];
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of(a, t, v0, v1, s);
  if (r.b < 0) return;
  const float k = slope_of(r);
  Stat mine = {-HB_INF, 0.f, 0x7fffffff};
  for (int v = v0 + (int)threadIdx.x * 8; v < v1; v += kStep) {
    float z[8];
    values<T, WHOLE>(a, r, s, t, v, v0, z);
    float top = z[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, z[e]);
    if (top > mine.top) {
      mine.sum *= weight_of(mine.top, top, k);
      mine.top = top;
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (z[e] == top) mine.token = v + e;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) mine.sum += weight_of(z[e], mine.top, k);
  }
  for (int m = 32; m; m >>= 1) {
    Stat other;
    other.top = __shfl_xor(mine.top, m, 64);
    other.sum = __shfl_xor(mine.sum, m, 64);
    other.token = __shfl_xor(mine.token, m, 64);
    mine = joined(mine, other, k);
  }
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) mine = joined(mine, waves[w], k);
    float *at = a.stats + ((size_t)t * a.parts + blockIdx.y) * 4;
    at[0] = mine.top;
    at[1] = mine.sum;
    at[2] = __int_as_float(mine.token);
  }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rules_probs_kernel(RulesArgs a) {
  __shared__ RowLds s;
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of(a, t, v0, v1, s);
  if (r.b < 0) return;
  const float k = slope_of(r);
  Stat all = {-HB_INF, 0.f, 0x7fffffff};
  for (int p = 0; p < a.parts; ++p) {
    const float *at = a.stats + ((size_t)t * a.parts + p) * 4;
    all = joined(all, {at[0], at[1], __float_as_int(at[2])}, k);
  }
  const float scale = all.top > -HB_INF ? 1.f / all.sum : 0.f;
  float *out = (float *)a.out + (size_t)t * a.V;
  for (int v = v0 + (int)threadIdx.x * 8; v < v1; v += kStep) {
    float z[8];
    if (r.temperature > 0.f) {
      values<T, WHOLE>(a, r, s, t, v, v0, z);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = weight_of(z[e], all.top, k) * scale;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = all.top > -HB_INF && v + e == all.token ? 1.f : 0.f;
    }
    store_eight<WHOLE>(out + v, a.V - v, z);
  }
}

__global__ __launch_bounds__(kThreads) void rules_count_kernel(int B, int V, int n, const int32_t *row_offset, const int32_t *tokens,
                                                               int prompt, int32_t *counts) {
  const int b = blockIdx.x, each = n / B;
  int lo = b * each, hi = lo + each;
  if (row_offset) {
    lo = row_offset[b];
    hi = row_offset[b + 1];
    if (lo < 0 || hi > n) return;
  }
  for (int64_t i = lo + (int64_t)blockIdx.y * kThreads + threadIdx.x; i < hi; i += (int64_t)gridDim.y * kThreads) {
    const int v = tokens[i];
    if (v < 0 || v >= V) continue;
    int32_t *at = counts + (size_t)b * V + v;
    if (prompt)
      atomicOr(at, kPromptFlag);
    else
      atomicAdd(at, 1);
  }
}

template <typename T, bool WHOLE>
void go_probs(const RulesArgs &a, hipStream_t s) {
  const dim3 grid(a.rows, a.parts);
  rules_stats_kernel<T, WHOLE><<<grid, kThreads, 0, s>>>(a);
  rules_probs_kernel<T, WHOLE><<<grid, kThreads, 0, s>>>(a);
}
template <typename T, bool WHOLE>
void go_logits(const RulesArgs &a, hipStream_t s) {
  rules_logits_kernel<T, WHOLE><<<dim3(a.rows, a.parts), kThreads, 0, s>>>(a);
}

}  // namespace

int32_t rules_parts(int32_t rows, int32_t V, int32_t *chunk) {
  const int64_t most = ((int64_t)V + kStep - 1) / kStep;
  int64_t parts = rows > 0 ? (4096 + rows - 1) / rows : 1;
  parts = parts < 1 ? 1 : parts > most ? most : parts;
  int64_t len = (((int64_t)V + parts - 1) / parts + kStep - 1) / kStep * kStep;
  if (len > kMostChunk) len = kMostChunk;
  *chunk = (int32_t)len;
  return (int32_t)(((int64_t)V + len - 1) / len);
}

hipError_t launch_rules_logits(RulesArgs a, hipStream_t s) {
  a.parts = rules_parts(a.rows, a.V, &a.chunk);
  if (a.dtype == HB_F32)
    a.V % 8 ? go_logits<float, false>(a, s) : go_logits<float, true>(a, s);
  else
    a.V % 8 ? go_logits<bf16_t, false>(a, s) : go_logits<bf16_t, true>(a, s);
  return hipGetLastError();
}

hipError_t launch_rules_probs(RulesArgs a, hipStream_t s) {
  a.parts = rules_parts(a.rows, a.V, &a.chunk);
  if (a.dtype == HB_F32)
    a.V % 8 ? go_probs<float, false>(a, s) : go_probs<float, true>(a, s);
  else
    a.V % 8 ? go_probs<bf16_t, false>(a, s) : go_probs<bf16_t, true>(a, s);
  return hipGetLastError();
}

hipError_t launch_rules_count(int32_t B, int32_t V, int32_t n, const int32_t *row_offset, const int32_t *tokens, int32_t prompt,
                              int32_t *counts, hipStream_t s) {
  const int64_t y = ((int64_t)n / B + 2 * kThreads - 1) / (2 * kThreads);
  rules_count_kernel<<<dim3(B, (unsigned)(y < 1 ? 1 : y > 64 ? 64 : y)), kThreads, 0, s>>>(B, V, n, row_offset, tokens, prompt, counts);
  return hipGetLastError();
}

}  // namespace hb
