// A request's sampling rules applied to the logits of its tree's nodes (hb_rules_logits, hb_rules_probs, hb_rules_count).
//
//   c = how often the request has had the token, those on the node's own path below the root included
//   z = logit;  c > 0 or in the prompt: z / repetition where z > 0, else z * repetition
//   z = z - (presence [c > 0] + frequency c) + bias;  -infinity where the grammar forbids the token, or z is no number
//   p = exp((z - max z) / temperature) / sum;  temperature 0: 1 for the largest z, the lowest token among equals
//
// A workgroup has a row, or a chunk of one.  Few tokens have anything to them but their logit and their mask: those with a
// count, those on the path and those with a bias.  It finds them first (one pass over the counts, which all nodes of a tree
// share, and make first where they are several) and marks them in a bitmap in LDS.  The row is then gone through without them,
// four tokens a thread and little to do for each, and they are done behind it, a thread each.  16 trees of 60 nodes over 152064
// tokens: with the penalties' code at each of a thread's tokens 472 us; with a loop over the marks that a wavefront meets 331
// (one token in a hundred is marked: nearly every wavefront meets some); so 241.  What bounds it are the bytes past L2: logits and
// masks from memory (307 MB), the logits again from the last cache, 592 MB of stores, 1.19 GB at 4.9 TB/s, where a copy has 5.1;
// fewer vector instructions, or more loads under way, change nothing.  Biases go to their tokens' places among the marked ones:
// looked for at each marked token instead, 29 rows of 1148 tokens with up to 242 each took 68 us, so 26.  (A row held in 76 registers a thread between the passes: 392,
// with one workgroup a CU.)
// In float32, in the order that is written above, without contraction: two sides that follow it agree about which z is the
// largest.
#include "rules.h"
#include "wave_ops.h"

namespace hb {

namespace {

#pragma clang fp contract(off)

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kSplit = 256, kStep = kSplit * 8, kMostChunk = 32768;  // threads of a workgroup that has a chunk of a row
constexpr int kWhole = 1024, kMostWhole = 1 << 18;  // ... that has a row, and tokens of one
constexpr float kLog2e = 1.4426950408889634f;
#define HB_INF __builtin_huge_valf()

struct Row {
  int b;                     // sequence (-1: nobody's row)
  float temperature, repetition, presence, frequency;
  const int32_t *counts;     // of its sequence, or null
  const uint8_t *mask;       // bytes of its mask, or null
  int path, bias0, biases;   // tokens on the path; biases
  int marks, first;          // marked tokens of the chunk, and those of the threads in front of this one
};

extern __shared__ uint32_t marked_lds[];  // a bit for every token of the chunk

template <int kThreads>
struct RowLds {
  static constexpr int kSome = 2 * kThreads;
  uint32_t some[kSome];  // marked tokens, so many at a time (with kBiased, kSeveral: those that have a bias, or several), and
  float value[kSome];    // their biases, then their values
  int32_t path[64];
  int32_t first[kThreads];  // marked tokens of the threads in front of each
  int32_t sums[kThreads / 64];
  int32_t found[2];
};
constexpr uint32_t kBiased = 1u << 30, kSeveral = 1u << 31;  // V is at most 2^30

// The row's rules, and the marks of its chunk [v0, v1), which nobody changes behind it.  Every one of kThreads threads calls it.
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
  uint32_t *marked = marked_lds;
  // where many rows have the same counts, their marks have been made already
  const bool made = a.marks && r.counts;
  for (int i = tid; i < words; i += kThreads) marked[i] = made ? a.marks[(size_t)r.b * ((a.V + 31) / 32) + v0 / 32 + i] : 0;
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
  __syncthreads();
  r.path = s.found[1];
  auto mark = [&](int v) {
    if (v >= v0 && v < v1) atomicOr(&marked[(v - v0) >> 5], 1u << ((v - v0) & 31));
  };
  if (tid < r.path) mark(s.path[tid]);
  for (int i = tid; i < r.biases; i += kThreads) mark(a.bias_id[r.bias0 + i]);
  if (r.counts && !made) {
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
  // a thread has every kThreads-th word: marks come in heaps
  int mine = 0;
  for (int i = tid; i < words; i += kThreads) mine += __popc(marked[i]);
  int upto = scan_lanes(mine);
  if (lane == 63) s.sums[tid >> 6] = upto;
  __syncthreads();
  r.marks = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < tid >> 6) upto += s.sums[w];
    r.marks += s.sums[w];
  }
  r.first = s.first[tid] = upto - mine;
  return r;
}

// f(v, its adjusted value) for the marked tokens of the chunk [v0, v1).  Every thread calls it; it begins with a barrier.
// again: it has been called before, with the same arguments.
template <typename T, int kThreads, typename F>
__device__ __forceinline__ void each_marked(const RulesArgs &a, const Row &r, RowLds<kThreads> &s, int t, int v0, int v1, bool again, F f) {
  constexpr int kSome = RowLds<kThreads>::kSome;
  const int words = (v1 - v0 + 31) / 32;
  if (again && r.marks <= kSome) {
    __syncthreads();
    for (int i = threadIdx.x; i < r.marks; i += kThreads) f((int)s.some[i], s.value[i]);
    return;
  }
  for (int from = 0; from < r.marks; from += kSome) {
    __syncthreads();
    int at = r.first - from;
    for (int i = threadIdx.x; i < words && at < kSome; i += kThreads)
      for (uint32_t m = marked_lds[i]; m; m &= m - 1, ++at)
        if (at >= 0 && at < kSome) s.some[at] = v0 + 32 * i + __ffs(m) - 1;
    __syncthreads();
    // each bias to its token's place among the marks: those of the threads in front, of this thread's words in front, of the word
    for (int i = threadIdx.x; i < r.biases; i += kThreads) {
      const int v = a.bias_id[r.bias0 + i];
      if (v < v0 || v >= v1) continue;
      const int at_v = v - v0, word = at_v >> 5, owner = word % kThreads;
      int place = s.first[owner] - from + __popc(marked_lds[word] & ((1u << (at_v & 31)) - 1));
      for (int x = owner; x < word; x += kThreads) place += __popc(marked_lds[x]);
      if (place < 0 || place >= kSome) continue;
      if (atomicOr(&s.some[place], kBiased) & kBiased) atomicOr(&s.some[place], kSeveral);
      s.value[place] = a.bias_value[r.bias0 + i];
    }
    if (r.biases > 0) __syncthreads();
    for (int i = threadIdx.x; i < min(r.marks - from, kSome); i += kThreads) {
      const uint32_t found = s.some[i];
      const int v = (int)(found & (kBiased - 1));
      s.some[i] = (uint32_t)v;
      float z = load_f32((const T *)a.logits + (size_t)t * a.V + v);
      const uint32_t bits = r.mask ? r.mask[v >> 3] : 0xffu;
      const int had = r.counts ? r.counts[v] : 0;
      int c = had & (kPromptFlag - 1);
      for (int p = 0; p < r.path; ++p) c += s.path[p] == v;
      const bool seen = c > 0 || (had & kPromptFlag);
      const float less = c > 0 ? r.presence + r.frequency * (float)c : 0.f;  // (an infinite penalty times none is none)
      float more = found & kBiased ? s.value[i] : 0.f;
      if (found & kSeveral) {  // in their order
        more = 0.f;
        for (int x = 0; x < r.biases; ++x)
          if (a.bias_id[r.bias0 + x] == v) more += a.bias_value[r.bias0 + x];
      }
      if (seen) z = z > 0.f ? z / r.repetition : z * r.repetition;
      z = z - less;
      z = z + more;
      z = (bits >> (v & 7) & 1) && z == z ? z : -HB_INF;
      s.value[i] = z;
      f(v, z);
    }
  }
}

// -infinity where the bit of `keep` is not set; and what is no number gives way to it
template <int N>
__device__ __forceinline__ void keep_of(uint32_t keep, float (&z)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const uint32_t k = (uint32_t)((int32_t)(keep << (31 - e)) >> 31);
    z[e] = fmaxf(__uint_as_float((__float_as_uint(z[e]) & k) | (0xff800000u & ~k)), -HB_INF);
  }
}

// N tokens' logits as they lie in memory; WHOLE: rows are a multiple of four long, and pieces of four aligned
template <typename T, bool WHOLE, int N>
struct Piece {
  T x[N];
};
template <>
struct Piece<float, true, 4> {
  f32x4 x;
};
template <>
struct Piece<bf16_t, true, 4> {
  u32x2 x;
};
template <>
struct Piece<bf16_t, true, 8> {
  u32x2 x[2];
};
template <typename T, int N>
__device__ __forceinline__ void load_piece(const T *p, int n, Piece<T, false, N> &y) {
#pragma unroll
  for (int e = 0; e < N; ++e) y.x[e] = e < n ? p[e] : T(0);
}
__device__ __forceinline__ void load_piece(const float *p, int, Piece<float, true, 4> &y) { y.x = *(const f32x4 *)p; }
__device__ __forceinline__ void load_piece(const bf16_t *p, int, Piece<bf16_t, true, 4> &y) { y.x = *(const u32x2 *)p; }
__device__ __forceinline__ void load_piece(const bf16_t *p, int n, Piece<bf16_t, true, 8> &y) {
  typedef uint32_t half_aligned __attribute__((ext_vector_type(4), aligned(8)));
  if (n >= 8) {
    const half_aligned x = *(const half_aligned *)p;
    y.x[0] = x.xy;
    y.x[1] = x.zw;
  } else {
    y.x[0] = *(const u32x2 *)p;
    y.x[1] = (u32x2)0xff80ff80u;  // -infinity
  }
}
template <typename T, int N>
__device__ __forceinline__ void widen(const Piece<T, false, N> &y, int n, float (&z)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) z[e] = e < n ? load_f32(&y.x[e]) : -HB_INF;
}
__device__ __forceinline__ void widen(const Piece<float, true, 4> &y, int, float (&z)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) z[e] = y.x[e];
}
__device__ __forceinline__ void widen_two(uint32_t x, float *z) {
  z[0] = __uint_as_float(x << 16);
  z[1] = __uint_as_float(x & 0xffff0000u);
}
__device__ __forceinline__ void widen(const Piece<bf16_t, true, 4> &y, int, float (&z)[4]) {
#pragma unroll
  for (int e = 0; e < 2; ++e) widen_two(y.x[e], z + 2 * e);
}
__device__ __forceinline__ void widen(const Piece<bf16_t, true, 8> &y, int, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) widen_two(y.x[e / 2][e % 2], z + 2 * e);
}

// PAST: the caches, which then keep the logits for the second time over them (16 trees of 60 nodes over 152064 tokens 274 -> 253 us)
template <bool WHOLE, bool PAST = false>
__device__ __forceinline__ void store_four(float *p, int n, const float (&z)[4]) {
  const f32x4 x = {z[0], z[1], z[2], z[3]};
  if (WHOLE && PAST) {
    __builtin_nontemporal_store(x, (f32x4 *)p);
  } else if (WHOLE) {
    *(f32x4 *)p = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = z[e];
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store_four(bf16_t *p, int n, const float (&z)[4]) {
  if (WHOLE) {
    *(u32x2 *)p = (u32x2){pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = f32_to_bf16(z[e]);
  }
}

// Tokens v0 .. v1 - 1, N at a time: f(v, values), those of marked tokens -infinity, or (MARKED) as they are.  The logits of the next
// turns are asked for before this one's are worked on.  N is four where something is stored: what a wavefront stores is whole
// lines then (with eight, in two halves of 16 bytes, half the requests to L2 were for parts of one).
template <typename T, bool WHOLE, int N, bool MARKED, int kThreads, typename F>
__device__ __forceinline__ void each_piece(const RulesArgs &a, const Row &r, const RowLds<kThreads> &, int t, int v0, int v1, F f) {
  constexpr int kTurn = kThreads * N, kDeep = 2;
  const T *row = (const T *)a.logits + (size_t)t * a.V;
  Piece<T, WHOLE, N> y[kDeep];
  uint32_t allowed[kDeep];
  const int first = v0 + (int)threadIdx.x * N;
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
      float z[N];
      widen(y[i], a.V - at, z);
      const uint32_t bits = allowed[i] >> (at & (8 - N)), marked = marked_lds[(at - v0) >> 5] >> ((at - v0) & 31);
      ask(at + kDeep * kTurn, i);
      keep_of(MARKED ? bits | marked : bits & ~marked, z);
      f(at, z);
    }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(kSplit) void rules_logits_kernel(RulesArgs a) {
  __shared__ RowLds<kSplit> s;
  const int t = blockIdx.x, v0 = blockIdx.y * a.chunk, v1 = min(a.V, v0 + a.chunk);
  const Row r = row_of<kSplit>(a, t, v0, v1, s);
  if (r.b < 0) return;
  T *out = (T *)a.out + (size_t)t * a.V;
  each_piece<T, WHOLE, 4, true>(a, r, s, t, v0, v1, [&](int v, float (&z)[4]) { store_four<WHOLE>(out + v, a.V - v, z); });
  // (which may have been written where the logits are: marked ones as they were)
  each_marked<T>(a, r, s, t, v0, v1, false, [&](int v, float z) { store_f32(out + v, z); });
}

// What is known of some tokens of a row: of a greedy one (k = 0) the largest value and the lowest token that has it; of the
// others the largest value, or the lowest that there is, and the sum of 2^((z - largest) / 2 * k), 0 where nothing is left
struct Stat {
  float top, sum;
  int token;
};
constexpr float kLowest = -3.402823466e38f;
// Half the difference, which float32 has for all finite values (and no further rounding); k is more than 0, so that what is infinite stays so.
__device__ __forceinline__ float weight_of(float z, float top, float k) {
  const float d = z == top ? 0.f : fmaf(z, 0.5f, -0.5f * top);  // also where both are infinite
  return __builtin_amdgcn_exp2f(d * k);
}
// Some values' weights.  Plainly they are what they should be for every finite `top`: -infinity gives 0.
template <int N>
__device__ __forceinline__ void weigh(float (&z)[N], float top, float k) {
  if (__any(!(top < HB_INF))) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = weight_of(z[e], top, k);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = __builtin_amdgcn_exp2f(fmaf(z[e], 0.5f, -0.5f * top) * k);
  }
}
__device__ __forceinline__ Stat joined(const Stat x, const Stat y, float k, bool greedy) {
  Stat j;
  const bool second = y.top > x.top || (y.top == x.top && y.token < x.token);
  j.top = second ? y.top : x.top;
  j.token = second ? y.token : x.token;
  j.sum = greedy ? 0.f : x.sum * weight_of(x.top, j.top, k) + y.sum * weight_of(y.top, j.top, k);
  return j;
}
__device__ __forceinline__ Stat joined_lanes(Stat x, float k, bool greedy) {
  for (int m = 32; m; m >>= 1) {
    Stat y;
    y.top = __shfl_xor(x.top, m, 64);
    y.sum = __shfl_xor(x.sum, m, 64);
    y.token = __shfl_xor(x.token, m, 64);
    x = joined(x, y, k, greedy);
  }
  return x;
}
__device__ __forceinline__ Stat nothing_of(bool greedy) { return {greedy ? -HB_INF : kLowest, 0.f, 0x7fffffff}; }
// (the same in every lane, and known to be.  An infinite temperature has a slope that leaves finite values alike to 2^-21.)
__device__ __forceinline__ float slope_of(const Row &r) {
  const float k = fminf(fmaxf(2.f * (kLog2e / r.temperature), 1e-45f), 3e38f);
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(r.temperature > 0.f ? k : 0.f)));
}
__device__ __forceinline__ bool greedy_of(const Row &r) { return __builtin_amdgcn_readfirstlane(!(r.temperature > 0.f)); }

// Of tokens v0 .. v1 - 1, over all of the workgroup's kThreads threads
template <typename T, bool WHOLE, int kThreads>
__device__ __forceinline__ Stat stat_of(const RulesArgs &a, const Row &r, RowLds<kThreads> &s, int t, int v0, int v1, float k) {
  __shared__ Stat waves[kThreads / 64];
  constexpr int N = sizeof(T) == 2 ? 8 : 4;  // 16 bytes
  const bool greedy = greedy_of(r);
  Stat mine = nothing_of(greedy);
  if (greedy)
    each_piece<T, WHOLE, N, false>(a, r, s, t, v0, v1, [&](int v, float (&z)[N]) {
      float top = z[0];
#pragma unroll
      for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
      if (top > mine.top) {
        mine.top = top;
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
          if (z[e] == top) mine.token = v + e;
      }
    });
  else
    each_piece<T, WHOLE, N, false>(a, r, s, t, v0, v1, [&](int, float (&z)[N]) {
      const float last = mine.top;
#pragma unroll
      for (int e = 0; e < N; ++e) mine.top = fmaxf(mine.top, z[e]);
      if (__any(last != mine.top)) mine.sum *= weight_of(last, mine.top, k);
      weigh(z, mine.top, k);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < N; e += 4) sum += (z[e] + z[e + 1]) + (z[e + 2] + z[e + 3]);
      mine.sum += sum;
    });
  each_marked<T>(a, r, s, t, v0, v1, false, [&](int v, float z) {
    if (z > -HB_INF) mine = joined(mine, {z, 1.f, v}, k, greedy);
  });
  mine = joined_lanes(mine, k, greedy);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = mine;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  return joined_lanes(lane < kThreads / 64 ? waves[lane] : nothing_of(greedy), k, greedy);
}

template <typename T, bool WHOLE, int kThreads>
__device__ __forceinline__ void probs_of(const RulesArgs &a, const Row &r, RowLds<kThreads> &s, int t, int v0, int v1, const Stat &all, float k, bool again) {
  float *out = (float *)a.out + (size_t)t * a.V;
  if (!greedy_of(r)) {
    const float scale = all.sum > 0.f ? 1.f / all.sum : 0.f;
    each_piece<T, WHOLE, 4, false>(a, r, s, t, v0, v1, [&](int v, float (&z)[4]) {
      weigh(z, all.top, k);
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] *= scale;
      store_four<WHOLE, kThreads == kWhole>(out + v, a.V - v, z);
    });
    each_marked<T>(a, r, s, t, v0, v1, again, [&](int v, float z) { out[v] = weight_of(z, all.top, k) * scale; });
  } else {
    for (int v = v0 + (int)threadIdx.x * 4; v < v1; v += kThreads * 4) {
      float z[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = all.top > -HB_INF && v + e == all.token ? 1.f : 0.f;
      store_four<WHOLE, kThreads == kWhole>(out + v, a.V - v, z);
    }
  }
}

// A bit for every token that has a count, [batch][words]
__global__ __launch_bounds__(kSplit) void rules_marks_kernel(const int32_t *counts, int V, uint32_t *marks) {
  const int words = (V + 31) / 32, lane = threadIdx.x & 63;
  const int32_t *row = counts + (size_t)blockIdx.x * V;
  for (int64_t v = ((int64_t)blockIdx.y * kSplit + threadIdx.x); v < (int64_t)words * 32; v += (int64_t)gridDim.y * kSplit) {
    const unsigned long long bits = __ballot(v < V && row[v] != 0);  // of two words, by a wavefront
    const int word = (int)(v >> 5);
    if ((lane & 31) == 0) marks[(size_t)blockIdx.x * words + word] = (uint32_t)(bits >> (lane & 32));
  }
}

// A row by one workgroup: twice over it, the second time out of the last cache
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kWhole, 8) void rules_row_kernel(RulesArgs a) {
  __shared__ RowLds<kWhole> s;
  // consecutive workgroups land on different dies: rows are dealt so that a die has neighbours, which share their counts
  const int each = gridDim.x / 8, t = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if (t >= a.rows) return;
  const Row r = row_of<kWhole>(a, t, 0, a.V, s);
  if (r.b < 0) return;
  const float k = slope_of(r);
  const Stat all = stat_of<T, WHOLE, kWhole>(a, r, s, t, 0, a.V, k);
  probs_of<T, WHOLE>(a, r, s, t, 0, a.V, all, k, true);
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
  const bool greedy = greedy_of(r);
  Stat all = nothing_of(greedy);
  for (int p = threadIdx.x & 63; p < a.parts; p += 64) {  // (chunks in front have the lower tokens)
    const f32x4 x = *(const f32x4 *)(a.stats + ((size_t)t * a.parts + p) * 4);
    all = joined(all, {x[0], x[1], __float_as_int(x[2])}, k, greedy);
  }
  all = joined_lanes(all, k, greedy);
  probs_of<T, WHOLE>(a, r, s, t, v0, v1, all, k, false);
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

size_t chunk_bytes(int32_t tokens) { return ((size_t)tokens + 31) / 32 * 4; }

template <typename T, bool WHOLE>
hipError_t go_probs(const RulesArgs &a, hipStream_t s) {
  if (a.parts == 0) {
    const size_t bytes = chunk_bytes(a.V);
    if (a.marks) {
      const int64_t y = ((int64_t)a.V + 4 * kSplit - 1) / (4 * kSplit);
      rules_marks_kernel<<<dim3(a.batch, (unsigned)(y > 64 ? 64 : y)), kSplit, 0, s>>>(a.counts, a.V, a.marks);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    auto kern = rules_row_kernel<T, WHOLE>;
    hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)chunk_bytes(kMostWhole));
    if (e != hipSuccess) return e;
    kern<<<(unsigned)((a.rows + 7) / 8 * 8), kWhole, bytes, s>>>(a);
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
  // Some 1024 workgroups: what each does before it reads its chunk is as much as 2000 tokens of it.  152064 tokens, with 256, 512, 1024, 2048,
  // 4096: 42 rows of 7 sequences 49, 38, 34, 35, 44 us; 64 rows 61, 47, 41, 42, 46; their logits alone 33, 27, 24, 24, 26; 8 rows 20, 18, 18, 18, 18
  int64_t parts = rows > 0 ? (1024 + rows - 1) / rows : 1;
  parts = parts < 1 ? 1 : parts > most ? most : parts;
  int64_t len = (((int64_t)V + parts - 1) / parts + kStep - 1) / kStep * kStep;
  if (len > kMostChunk) len = kMostChunk;
  *chunk = (int32_t)len;
  return (int32_t)(((int64_t)V + len - 1) / len);
}

bool rules_marks(int32_t B, int32_t T) { return T >= 4 * (int64_t)B; }

// 0: a workgroup has a row for itself.  152064 tokens, a workgroup and several: 90 rows 54 and 48 us, 120 rows 55 to 63 and 57 to 61, 160 rows 59 to 66
// and 69 to 77, 480 rows 114 and 197
int32_t rules_parts(int32_t rows, int32_t V, int32_t *chunk) {
  return rows >= 128 && V <= kMostWhole ? 0 : split(rows, V, chunk);
}

hipError_t launch_rules_logits(RulesArgs a, hipStream_t s) {
  a.parts = split(a.rows, a.V, &a.chunk);
  if (a.dtype == HB_F32) return a.V % 4 ? go_logits<float, false>(a, s) : go_logits<float, true>(a, s);
  return a.V % 4 ? go_logits<bf16_t, false>(a, s) : go_logits<bf16_t, true>(a, s);
}

hipError_t launch_rules_probs(RulesArgs a, hipStream_t s) {
  a.parts = rules_parts(a.rows, a.V, &a.chunk);
  if (a.dtype == HB_F32) return a.V % 4 ? go_probs<float, false>(a, s) : go_probs<float, true>(a, s);
  return a.V % 4 ? go_probs<bf16_t, false>(a, s) : go_probs<bf16_t, true>(a, s);
}

hipError_t launch_rules_count(int32_t B, int32_t V, int32_t n, const int32_t *row_offset, const int32_t *tokens, int32_t prompt,
                              int32_t *counts, hipStream_t s) {
  const int64_t y = ((int64_t)n / B + 2 * kSplit - 1) / (2 * kSplit);
  rules_count_kernel<<<dim3(B, (unsigned)(y < 1 ? 1 : y > 64 ? 64 : y)), kSplit, 0, s>>>(B, V, n, row_offset, tokens, prompt, counts);
  return hipGetLastError();
}

}  // namespace hb
