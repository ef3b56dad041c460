// A request's sampling rules applied to the logits of its tree's nodes (hb_rules_logits, hb_rules_probs, hb_rules_count).
//
//   c = how often the request has had the token, those on the node's own path below the root included
//   z = logit;  c > 0 or in the prompt: z / repetition where z > 0, else z * repetition
//   z = z - (presence [c > 0] + frequency c) + bias;  -infinity where the grammar forbids the token, or z is no number
//   p = exp((z - max z) / temperature) / sum;  temperature 0: 1 for the largest z, the lowest token among equals
//
// A workgroup has a row, or a chunk of one.  Few tokens have anything to them but their logit and their mask: those with a
// count, those on the path and those with a bias.  It finds them first (one pass over the counts, which all nodes of a tree
// share), marks them in a bitmap in LDS and puts what is to be done to each into a table there, in the order of the tokens, so that
// a token's place is the number of marks in front of it.  What is then done for every token is little, and a wavefront that
// meets marks takes one of each lane's at a time.  (With the penalties' code at each of a thread's eight tokens the loop was
// twenty times as long: 16 trees of 60 nodes over 152064 tokens 472 us.)
// In float32, in the order that is written above, without contraction: two sides that follow it agree about which z is the
// largest.
#include "rules.h"
#include "wave_ops.h"

namespace hb {

namespace {

#pragma clang fp contract(off)

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kSplit = 256, kStep = kSplit * 8, kMostChunk = 32768, kBiases = 1024;  // threads of a workgroup that has a chunk of a row
constexpr int kWhole = 1024, kMostWhole = 1 << 18;  // ... that has a row, and tokens of one
constexpr float kLog2e = 1.4426950408889634f;
#define HB_INF __builtin_huge_valf()

struct Row {
  int b;                     // sequence (-1: nobody's row)
  float temperature, repetition, presence, frequency;
  const int32_t *counts;     // of its sequence, or null
  const uint8_t *mask;       // bytes of its mask, or null
  int path, bias0, biases;   // tokens on the path; biases
  const uint32_t *marked;    // a bit for every token of the chunk
  const uint16_t *before;    // marks in front of every 32 (at most 65535)
};

extern __shared__ uint32_t chunk_lds[];  // marked and before

// What is done to marked tokens, for the first `kEntries` of them; the others are looked up again
template <int kThreads>
struct RowLds {
  static constexpr int kEntries = kThreads * 4;
  float less[kEntries], more[kEntries];  // the penalty that is subtracted, and the bias
  uint8_t seen[kEntries];
  int32_t path[64];
  int32_t bias_id[kBiases];
  float bias_value[kBiases];
  int32_t sums[kThreads / 64];
  int32_t found[2];
};

// What is done to token v
template <int kThreads>
__device__ __forceinline__ void look_up(const RulesArgs &a, const Row &r, const RowLds<kThreads> &s, int v, bool &seen, float &less, float &more) {
  const int had = r.counts ? r.counts[v] : 0;
  int c = had & (kPromptFlag - 1);
  for (int i = 0; i < r.path; ++i) c += s.path[i] == v;
  seen = c > 0 || (had & kPromptFlag);
  less = (c > 0 ? r.presence : 0.f) + r.frequency * (float)c;
  more = 0.f;
  for (int i = 0; i < r.biases; ++i) {
    const int id = i < kBiases ? s.bias_id[i] : a.bias_id[r.bias0 + i];
    if (id == v) more += i < kBiases ? s.bias_value[i] : a.bias_value[r.bias0 + i];
  }
}

// The row's rules, and the marks of its chunk [v0, v1).  Every one of kThreads threads calls it; ends with a barrier.
template <int kThreads>
__device__ __forceinline__ Row row_of(const RulesArgs &a, int t, int v0, int v1, RowLds<kThreads> &s) {
  const int tid = threadIdx.x, lane = tid & 63;
  Row r;
  r.b = -1;
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
  const int words = (v1 - v0 + 31) / 32;
  uint32_t *marked = chunk_lds;
  uint16_t *before = (uint16_t *)(chunk_lds + words);
  for (int i = tid; i < words; i += kThreads) marked[i] = 0;
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
    if (v >= v0 && v < v1) atomicOr(&marked[(v - v0) >> 5], 1u << ((v - v0) & 31));
  };
  if (tid < r.path) mark(s.path[tid]);
  for (int i = tid; i < r.biases; i += kThreads) mark(i < kBiases ? s.bias_id[i] : a.bias_id[r.bias0 + i]);
  if (r.counts) {
    if (a.V % 4 == 0) {
#pragma unroll 4
      for (int v = v0 + tid * 4; v < v1; v += kThreads * 4) {
        const u32x4 c = *(const u32x4 *)(r.counts + v);
        const uint32_t bits = (c[0] ? 1u : 0u) | (c[1] ? 2u : 0u) | (c[2] ? 4u : 0u) | (c[3] ? 8u : 0u);
        if (bits) atomicOr(&marked[(v - v0) >> 5], bits << ((v - v0) & 31));  // a chunk is a multiple of 32 tokens, or the last
      }
    } else {
      for (int v = v0 + tid; v < v1; v += kThreads)
        if (r.counts[v]) mark(v);
    }
  }
  __syncthreads();
  // marks in front of every word: a thread has a run of words
  const int each = (words + kThreads - 1) / kThreads, w0 = min(tid * each, words), w1 = min(w0 + each, words);
  int mine = 0;
  for (int i = w0; i < w1; ++i) mine += __popc(marked[i]);
  int upto = scan_lanes(mine);
  if (lane == 63) s.sums[tid >> 6] = upto;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < tid >> 6) upto += s.sums[w];
    total += s.sums[w];
  }
  int at = upto - mine;
  for (int i = w0; i < w1; ++i) {
    before[i] = (uint16_t)min(at, 65535);
    for (uint32_t m = marked[i]; m; m &= m - 1, ++at)
      if (at < RowLds<kThreads>::kEntries) s.more[at] = __int_as_float(v0 + 32 * i + __ffs(m) - 1);  // the token, for the next step
  }
  r.marked = marked;
  r.before = before;
  __syncthreads();
  for (int i = tid; i < min(total, RowLds<kThreads>::kEntries); i += kThreads) {
    bool seen;
    float less, more;
    look_up(a, r, s, __float_as_int(s.more[i]), seen, less, more);
    s.seen[i] = seen;
    s.less[i] = less;
    s.more[i] = more;
  }
  __syncthreads();
  return r;
}

// Eight tokens' values from v on; `allowed`: a bit each
template <int kThreads>
__device__ __forceinline__ void apply(const RulesArgs &a, const Row &r, const RowLds<kThreads> &s, int v, int v0, uint32_t allowed, float (&z)[8]) {
  const int rel = v - v0;
  const uint32_t word = r.marked[rel >> 5];
  uint32_t rare = word >> (rel & 31) & 0xffu;
  while (rare) {
    const int e = __ffs(rare) - 1;
    rare &= rare - 1;
    float x = z[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) x = e == i ? z[i] : x;
    const int at = r.before[rel >> 5] + __popc(word & ((1u << ((rel & 31) + e)) - 1u));
    bool seen;
    float less, more;
    if (at < RowLds<kThreads>::kEntries) {
      seen = s.seen[at];
      less = s.less[at];
      more = s.more[at];
    } else {
      look_up(a, r, s, v + e, seen, less, more);
    }
    if (seen) x = x > 0.f ? x / r.repetition : x * r.repetition;
    x = x - less;
    x = x + more;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = e == i ? x : z[i];
  }
  // -infinity where the bit is not set; and what is no number gives way to it
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t keep = (uint32_t)((int32_t)(allowed << (31 - e)) >> 31);
    z[e] = fmaxf(__uint_as_float((__float_as_uint(z[e]) & keep) | (0xff800000u & ~keep)), -HB_INF);
  }
}

// Eight tokens' logits and bits as they lie in memory; WHOLE: rows are a multiple of eight long, and pieces aligned
template <typename T, bool WHOLE>
struct Piece {
  T x[8];
};
template <>
struct Piece<float, true> {
  f32x4 x[2];
};
template <>
struct Piece<bf16_t, true> {
  u32x4 x;
};
template <typename T>
__device__ __forceinline__ void load_piece(const T *p, int n, Piece<T, false> &y) {
#pragma unroll
  for (int e = 0; e < 8; ++e) y.x[e] = e < n ? p[e] : T(0);
}
__device__ __forceinline__ void load_piece(const float *p, int, Piece<float, true> &y) {
  y.x[0] = *(const f32x4 *)p;
  y.x[1] = *(const f32x4 *)(p + 4);
}
__device__ __forceinline__ void load_piece(const bf16_t *p, int, Piece<bf16_t, true> &y) { y.x = *(const u32x4 *)p; }
template <typename T>
__device__ __forceinline__ void widen(const Piece<T, false> &y, int n, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = e < n ? load_f32(&y.x[e]) : -HB_INF;
}
__device__ __forceinline__ void widen(const Piece<float, true> &y, int, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = y.x[e / 4][e % 4];
}
__device__ __forceinline__ void widen(const Piece<bf16_t, true> &y, int, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[2 * e] = __uint_as_float(y.x[e] << 16);
    z[2 * e + 1] = __uint_as_float(y.x[e] & 0xffff0000u);
  }
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

// What row t has to tokens v0 .. v1 - 1, eight at a time: f(v, adjusted values).  The logits of the next two turns are asked for
// before this one's are worked on.
template <typename T, bool WHOLE, int kThreads, typename F>
__device__ __forceinline__ void each_eight(const RulesArgs &a, const Row &r, const RowLds<kThreads> &s, int t, int v0, int v1, F f) {
  constexpr int kTurn = kThreads * 8, kDeep = 2;
  const T *row = (const T *)a.logits + (size_t)t * a.V;
  Piece<T, WHOLE> y[kDeep];
  uint32_t allowed[kDeep];
  const int first = v0 + (int)threadIdx.x * 8;
  auto ask = [&](int v, int at) {
    if (v >= v1) return;
    load_piece(row + v, a.V - v, y[at]);
    allowed[at] = r.mask ? r.mask[v >> 3] : 0xffu;
  };
#pragma unroll
  for (int i = 0; i < kDeep; ++i) ask(first + i * kTurn, i);
  for (int v = first; v < v1; v += kDeep * kTurn)
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int at = v + i * kTurn;
      if (at >= v1) break;
      float z[8];
      widen(y[i], a.V - at, z);
      const uint32_t bits = allowed[i];
      ask(at + kDeep * kTurn, i);
      apply(a, r, s, at, v0, bits, z);
      f(at, z);
    }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(kSplit) void rules_logits_kernel(RulesArgs a) {
  __shared__ RowLds<kSplit> s;
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of<kSplit>(a, t, v0, v1, s);
  if (r.b < 0) return;
  each_eight<T, WHOLE>(a, r, s, t, v0, v1, [&](int v, float (&z)[8]) { store_eight<WHOLE>((T *)a.out + (size_t)t * a.V + v, a.V - v, z); });
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
// eight values' weights: plainly where the largest is finite and k above 0 (-infinity gives 0 then)
__device__ __forceinline__ void weigh(float (&z)[8], float top, float k, bool plain) {
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = plain ? __builtin_amdgcn_exp2f((z[e] - top) * k) : weight_of(z[e], top, k);
}
__device__ __forceinline__ Stat joined(const Stat x, const Stat y, float k) {
  Stat j;
  const bool second = y.top > x.top || (y.top == x.top && y.token < x.token);
  j.top = second ? y.top : x.top;
  j.token = second ? y.token : x.token;
  j.sum = x.sum * weight_of(x.top, j.top, k) + y.sum * weight_of(y.top, j.top, k);
  return j;
}
__device__ __forceinline__ Stat joined_lanes(Stat x, float k) {
  for (int m = 32; m; m >>= 1) {
    Stat y;
    y.top = __shfl_xor(x.top, m, 64);
    y.sum = __shfl_xor(x.sum, m, 64);
    y.token = __shfl_xor(x.token, m, 64);
    x = joined(x, y, k);
  }
  return x;
}
__device__ __forceinline__ float slope_of(const Row &r) {
  return r.temperature > 0.f ? fminf(kLog2e / r.temperature, 3e38f) : 0.f;
}

// Of tokens v0 .. v1 - 1, over all of the workgroup's kThreads threads
template <typename T, bool WHOLE, int kThreads>
__device__ __forceinline__ Stat stat_of(const RulesArgs &a, const Row &r, const RowLds<kThreads> &s, int t, int v0, int v1, float k) {
  __shared__ Stat waves[kThreads / 64];
  Stat mine = {-HB_INF, 0.f, 0x7fffffff};
  each_eight<T, WHOLE>(a, r, s, t, v0, v1, [&](int v, float (&z)[8]) {
    float top = z[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, z[e]);
    if (top > mine.top) {  // seldom, after the first few
      mine.sum *= weight_of(mine.top, top, k);
      mine.top = top;
#pragma unroll
      for (int e = 7; e >= 0; --e)
        if (z[e] == top) mine.token = v + e;
    }
    if (k > 0.f) {
      weigh(z, mine.top, k, fabsf(mine.top) < HB_INF && k < 3e38f);
      mine.sum += ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
    } else if (r.temperature > 0.f) {  // without end: all the same
#pragma unroll
      for (int e = 0; e < 8; ++e) mine.sum += weight_of(z[e], mine.top, k);
    }
  });
  mine = joined_lanes(mine, k);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = mine;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  return joined_lanes(lane < kThreads / 64 ? waves[lane] : Stat{-HB_INF, 0.f, 0x7fffffff}, k);
}

template <typename T, bool WHOLE, int kThreads>
__device__ __forceinline__ void probs_of(const RulesArgs &a, const Row &r, const RowLds<kThreads> &s, int t, int v0, int v1, const Stat &all, float k) {
  float *out = (float *)a.out + (size_t)t * a.V;
  if (r.temperature > 0.f) {
    const float scale = all.top > -HB_INF ? 1.f / all.sum : 0.f;
    const bool plain = fabsf(all.top) < HB_INF && k > 0.f && k < 3e38f;
    each_eight<T, WHOLE>(a, r, s, t, v0, v1, [&](int v, float (&z)[8]) {
      weigh(z, all.top, k, plain);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] *= scale;
      store_eight<WHOLE>(out + v, a.V - v, z);
    });
  } else {
    for (int v = v0 + (int)threadIdx.x * 8; v < v1; v += kThreads * 8) {
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = all.top > -HB_INF && v + e == all.token ? 1.f : 0.f;
      store_eight<WHOLE>(out + v, a.V - v, z);
    }
  }
}

// A row by one workgroup: twice over it, the second time out of the last cache
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kWhole) void rules_row_kernel(RulesArgs a) {
  __shared__ RowLds<kWhole> s;
  const int t = blockIdx.x;
  const Row r = row_of<kWhole>(a, t, 0, a.V, s);
  if (r.b < 0) return;
  const float k = slope_of(r);
  const Stat all = stat_of<T, WHOLE, kWhole>(a, r, s, t, 0, a.V, k);
  probs_of<T, WHOLE>(a, r, s, t, 0, a.V, all, k);
}

// A row by several, for few rows: what each finds in its chunk, and then, the row
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kSplit) void rules_stats_kernel(RulesArgs a) {
  __shared__ RowLds<kSplit> s;
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of<kSplit>(a, t, v0, v1, s);
  if (r.b < 0) return;
  const Stat mine = stat_of<T, WHOLE, kSplit>(a, r, s, t, v0, v1, slope_of(r));
  if (threadIdx.x == 0)
    *(f32x4 *)(a.stats + ((size_t)t * a.parts + blockIdx.y) * 4) = (f32x4){mine.top, mine.sum, __int_as_float(mine.token), 0.f};
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(kSplit) void rules_probs_kernel(RulesArgs a) {
  __shared__ RowLds<kSplit> s;
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of<kSplit>(a, t, v0, v1, s);
  if (r.b < 0) return;
  const float k = slope_of(r);
  Stat all = {-HB_INF, 0.f, 0x7fffffff};
  for (int p = threadIdx.x & 63; p < a.parts; p += 64) {  // (chunks in front have the lower tokens)
    const f32x4 x = *(const f32x4 *)(a.stats + ((size_t)t * a.parts + p) * 4);
    all = joined(all, {x[0], x[1], __float_as_int(x[2])}, k);
  }
  all = joined_lanes(all, k);
  probs_of<T, WHOLE>(a, r, s, t, v0, v1, all, k);
}

__global__ __launch_bounds__(kSplit) void rules_count_kernel(int B, int V, int n, const int32_t *row_offset, const int32_t *tokens,
                                                               int prompt, int32_t *counts) {
  const int b = blockIdx.x, each = n / B;
  int lo = b * each, hi = lo + each;
  if (row_offset) {
    lo = row_offset[b];
    hi = row_offset[b + 1];
    if (lo < 0 || hi > n) return;
  }
  for (int64_t i = lo + (int64_t)blockIdx.y * kSplit + threadIdx.x; i < hi; i += (int64_t)gridDim.y * kSplit) {
    const int v = tokens[i];
    if (v < 0 || v >= V) continue;
    int32_t *at = counts + (size_t)b * V + v;
    if (prompt)
      atomicOr(at, kPromptFlag);
    else
      atomicAdd(at, 1);
  }
}

size_t chunk_bytes(int32_t tokens) { return ((size_t)tokens + 31) / 32 * 6 + 2; }

template <typename T, bool WHOLE>
hipError_t go_probs(const RulesArgs &a, hipStream_t s) {
  if (a.parts == 0) {
    const size_t bytes = chunk_bytes(a.V);
    auto kern = rules_row_kernel<T, WHOLE>;
    hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)chunk_bytes(kMostWhole));
    if (e != hipSuccess) return e;
    kern<<<a.rows, kWhole, bytes, s>>>(a);
    return hipGetLastError();
  }
  const dim3 grid(a.rows, a.parts);
  rules_stats_kernel<T, WHOLE><<<grid, kSplit, chunk_bytes(a.chunk), s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  rules_probs_kernel<T, WHOLE><<<grid, kSplit, chunk_bytes(a.chunk), s>>>(a);
  return hipGetLastError();
}
template <typename T, bool WHOLE>
hipError_t go_logits(const RulesArgs &a, hipStream_t s) {
  rules_logits_kernel<T, WHOLE><<<dim3(a.rows, a.parts), kSplit, chunk_bytes(a.chunk), s>>>(a);
  return hipGetLastError();
}

}  // namespace

// workgroups that share a row, and their chunks of it
static int32_t split(int32_t rows, int32_t V, int32_t *chunk) {
  const int64_t most = ((int64_t)V + kStep - 1) / kStep;
  int64_t parts = rows > 0 ? (4096 + rows - 1) / rows : 1;
  parts = parts < 1 ? 1 : parts > most ? most : parts;
  int64_t len = (((int64_t)V + parts - 1) / parts + kStep - 1) / kStep * kStep;
  if (len > kMostChunk) len = kMostChunk;
  *chunk = (int32_t)len;
  return (int32_t)(((int64_t)V + len - 1) / len);
}

// 0: a workgroup has a row for itself
int32_t rules_parts(int32_t rows, int32_t V, int32_t *chunk) {
  return rows >= 128 && V <= kMostWhole ? 0 : split(rows, V, chunk);
}

hipError_t launch_rules_logits(RulesArgs a, hipStream_t s) {
  a.parts = split(a.rows, a.V, &a.chunk);
  if (a.dtype == HB_F32) return a.V % 8 ? go_logits<float, false>(a, s) : go_logits<float, true>(a, s);
  return a.V % 8 ? go_logits<bf16_t, false>(a, s) : go_logits<bf16_t, true>(a, s);
}

hipError_t launch_rules_probs(RulesArgs a, hipStream_t s) {
  a.parts = rules_parts(a.rows, a.V, &a.chunk);
  if (a.dtype == HB_F32) return a.V % 8 ? go_probs<float, false>(a, s) : go_probs<float, true>(a, s);
  return a.V % 8 ? go_probs<bf16_t, false>(a, s) : go_probs<bf16_t, true>(a, s);
}

hipError_t launch_rules_count(int32_t B, int32_t V, int32_t n, const int32_t *row_offset, const int32_t *tokens, int32_t prompt,
                              int32_t *counts, hipStream_t s) {
  const int64_t y = ((int64_t)n / B + 2 * kSplit - 1) / (2 * kSplit);
  rules_count_kernel<<<dim3(B, (unsigned)(y < 1 ? 1 : y > 64 ? 64 : y)), kSplit, 0, s>>>(B, V, n, row_offset, tokens, prompt, counts);
  return hipGetLastError();
}

}  // namespace hb
