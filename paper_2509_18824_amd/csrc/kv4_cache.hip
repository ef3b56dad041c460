// Rows into and out of the 4-bit cache, and the eviction of positions from it.
#include "kv4.h"
#include "wave_ops.h"

namespace hb {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// eight elements of a row as float32
__device__ inline void load8(const float *p, float (&x)[8]) {
  const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
__device__ inline void load8(const bf16_t *p, float (&x)[8]) {
  const u32x4 a = *(const u32x4 *)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(a[e] << 16);
    x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
  }
}
__device__ inline void store8(float *p, const float (&x)[8]) {
  *(f32x4 *)p = (f32x4){x[0], x[1], x[2], x[3]};
  *(f32x4 *)(p + 4) = (f32x4){x[4], x[5], x[6], x[7]};
}
__device__ inline void store8(bf16_t *p, const float (&x)[8]) {
  *(u32x4 *)p = (u32x4){pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

// The sequence of row r, its rows [from, to) and where it starts, in one round trip up to 64 sequences (one to a lane, so every
// lane of the wavefront has to ask).
struct Place {
  int b, from, to, start;
};
__device__ inline Place place_of(const int32_t *__restrict__ offset, const int32_t *__restrict__ start, int batch, int r) {
  Place x;
  if (batch > 64) {  // uniform
    x.b = kv4_sequence(offset, batch, r);
    x.from = offset[x.b];
    x.to = offset[x.b + 1];
    x.start = start[x.b];
    return x;
  }
  const int lane = min((int)threadIdx.x & 63, batch - 1), from = offset[lane], to = offset[lane + 1], at = start[lane];
  x.b = 0;
  for (int i = 1; i < batch; ++i) x.b = __builtin_amdgcn_readlane(from, i) <= r ? i : x.b;
  x.from = __shfl(from, x.b, 64);
  x.to = __shfl(to, x.b, 64);
  x.start = __shfl(at, x.b, 64);
  return x;
}

// Quantises rows into the pages.  A thread takes eight elements of K and of V, four threads a block of 32: its largest
// magnitude is two exchanges away.  Threads run over the pieces of a head's row, then over rows, then over heads:
// neighbouring rows of a head are neighbours in a page.  PATH: the rows that a path names, max_path to a sequence.
// What bounds it is memory, and round trips in a row, to lengths, page and store: 11320 rows of 4 heads of 128 in two prompts, 29 MB,
// take 8.8 us (5.8 at the rate of a copy), 96 rows of paths 3.5.  K and V by threads of their own and a search for the sequence: 11.6
// us; sixteen elements to a thread: 0.3 us more for both directions.
template <typename T, bool PATH>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4AppendArgs a) {
  const hb_attn_desc &d = a.d;
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  for (long b = gid; a.new_len && b < d.batch; b += (long)gridDim.x * 256) {
    const int rows = a.row_offset[b + 1] - a.row_offset[b];
    int n = !PATH ? rows : rows > 0 && a.src_rows > 0 ? a.accept_len[b] : 0;
    n = n < 0 ? 0 : PATH && n > a.max_path ? a.max_path : n;
    const int L = a.prefix_len[b];
    a.new_len[b] = (L < 0 ? 0 : L) + n;
  }
  // pieces is a multiple of four: a block's threads leave together.  (32 bits hold what a launch may have)
  const unsigned pieces = d.head_dim / 8, item = (unsigned)gid / pieces;
  const int piece = (int)((unsigned)gid - item * pieces);
  if (a.rows == 0) return;
  const int h = (int)(item / (unsigned)a.rows), r = (int)(item - (unsigned)h * (unsigned)a.rows);
  Place at;
  if (!PATH) at = place_of(a.row_offset, a.prefix_len, d.batch, r);
  if (gid >= (long)a.rows * d.num_kv_heads * pieces) return;
  int b, j, L, src = r;
  bool live;
  float x[2][8];
  auto load = [&](int row) {
    const size_t from = ((size_t)row * d.num_kv_heads + h) * d.head_dim + piece * 8;
    load8((const T *)a.k + from, x[0]);
    load8((const T *)a.v + from, x[1]);
  };
  if (!PATH) load(r);
  if (PATH) {
    b = r / a.max_path;
    j = r - b * a.max_path;
    const int n0 = a.row_offset[b], n = a.row_offset[b + 1] - n0;
    live = j < a.accept_len[b] && n > 0 && a.src_rows > 0;  // a tree without nodes has no path, whatever accept_len says
    int node = live ? a.accept_path[(size_t)b * a.max_path + j] : 0;
    node = node < 0 ? 0 : (node >= n ? n - 1 : node);
    src = n0 + node;
    src = src < 0 ? 0 : (src >= a.src_rows ? a.src_rows - 1 : src);
    L = a.prefix_len[b];
  } else {
    b = at.b;
    j = r - at.from;
    live = j >= 0 && r < at.to;
    L = at.start;
  }
  L = L < 0 ? 0 : L;
  const long p = (long)L + j;
  const bool in_table = live && p < (long)d.max_blocks_per_seq * d.page_size;
  if (PATH && a.out_slots && h == 0 && piece == 0) {
    int slot = -1;
    if (in_table) {
      const size_t row = kv4_row(d, a.block_table, b, 0, (int)p);
      slot = (int)(row / ((size_t)d.num_kv_heads * d.page_size)) * d.page_size + (int)(row % d.page_size);
    }
    a.out_slots[r] = slot;
  }
  if (!in_table) return;
  const size_t row = kv4_row(d, a.block_table, b, h, (int)p);
  if (PATH) load(src);
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    uint32_t top = 0;  // magnitudes compare as their bits do, and what is not finite is above the rest
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[v][e]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const uint32_t s = kv4_scale_of(top);
    uint32_t codes = 0;  // to the nearest, ties to even; above 6: 6
    if (s != kKv4NaN) {
      const float scale = kv4_scale(s);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[v][0], x[v][1], scale, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[v][2], x[v][3], scale, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[v][4], x[v][5], scale, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[v][6], x[v][7], scale, 3);
    }
    *(uint32_t *)((v ? a.v_codes : a.k_codes) + row * (d.head_dim / 2) + piece * 4) = codes;
    if (piece % 4 == 0) (v ? a.v_scales : a.k_scales)[row * (d.head_dim / kKv4Block) + piece / 4] = (uint8_t)s;
  }
  if (piece == 0) {
    const size_t slot = ((size_t)b * d.num_kv_heads + h) * d.max_blocks_per_seq * d.page_size + p;
    if (a.weight) a.weight[slot] = 0.f;
    if (a.pos) a.pos[slot] = (a.seq_len ? a.seq_len[b] : L) + j;
  }
}

// The other way: rows as the cache holds them; positions that the table does not cover read as zero.  The same 29 MB: 8.4 to 10 us.
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(hb_attn_desc d, int rows, Kv4Pool kp, Kv4Pool vp,
                                                       const int32_t *__restrict__ block_table, const int32_t *__restrict__ first,
                                                       const int32_t *__restrict__ row_offset, T *__restrict__ k, T *__restrict__ v) {
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  const unsigned pieces = d.head_dim / 8, item = (unsigned)gid / pieces;
  const int piece = (int)((unsigned)gid - item * pieces);
  const int h = (int)(item / (unsigned)rows), r = (int)(item - (unsigned)h * (unsigned)rows);
  const Place at = place_of(row_offset, first, d.batch, r);
  if (gid >= (long)rows * d.num_kv_heads * pieces) return;
  const int b = at.b;
  const long p = (long)at.start + r - at.from;
  const bool there = p >= 0 && p < (long)d.max_blocks_per_seq * d.page_size;
  uint32_t codes[2] = {0, 0}, scales[2] = {127, 127};
  if (there) {
    const size_t row = kv4_row(d, block_table, b, h, (int)p), code = row * (d.head_dim / 2) + piece * 4,
                 scale = row * (d.head_dim / kKv4Block) + piece / 4;
    codes[0] = *(const uint32_t *)(kp.codes + code);
    codes[1] = *(const uint32_t *)(vp.codes + code);
    scales[0] = kp.scales[scale];
    scales[1] = vp.scales[scale];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t c = codes[i];
    const float s = kv4_scale(scales[i]);
    const kv4_f32x2 p0 = kv4_pair<0>(c, s), p1 = kv4_pair<1>(c, s), p2 = kv4_pair<2>(c, s), p3 = kv4_pair<3>(c, s);
    const float x[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    store8((i ? v : k) + ((size_t)r * d.num_kv_heads + h) * d.head_dim + piece * 8, x);
  }
}

// ---- eviction ------------------------------------------------------------------------------------------
// order-preserving bits of a weight; not a number counts as the least, protected positions as more than any
__device__ inline uint32_t weight_key(float w, bool safe) {
  w = fmaxf(w, -__builtin_huge_valf()) + 0.f;  // a number; and -0 weighs what 0 does
  const uint32_t u = __float_as_uint(w);
  return safe ? 0xffffffffu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kRounds = 8;                               // of four slots to a thread
constexpr int kPart = 256;                               // slots that a wavefront takes in a round
constexpr int kSlab = kSelectThreads * 4 * kRounds;      // 32768 slots
constexpr int kBins = 2048;                              // digits of 11, 11 and 10 bits
constexpr int kCopies = 4;                               // of a histogram, for a quarter of the lanes each: weights share few digits

// keys of four slots from s on; a slot past the length gets key 0, which no slot in front of it has
__device__ inline void load_keys(const float *w, const int32_t *pos, int s, int L, bool vec, int recent_from, int sinks,
                                 uint32_t (&key)[4], f32x4 &x, int32_t (&p)[4]) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  x = (f32x4){0.f, 0.f, 0.f, 0.f};
  i32x4 y = {0, 0, 0, 0};
  if (vec && s + 3 < L) {
    x = *(const f32x4 *)(w + s);
    y = *(const i32x4 *)(pos + s);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (s + e < L) {
        x[e] = w[s + e];
        y[e] = pos[s + e];
      }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    p[e] = y[e];
    key[e] = weight_key(x[e], y[e] >= recent_from || y[e] < sinks);
  }
  if (s + 3 >= L)
#pragma unroll
    for (int e = 0; e < 4; ++e) key[e] = s + e < L ? key[e] : 0u;
}

// number of the wavefront's slots in front of this lane's first one that a flag of theirs is set for: flag e of a lane is slot
// 4 lane + e; and of all
__device__ inline int lanes_before(const unsigned long long (&m)[4]) {
  int n = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) n += __builtin_amdgcn_mbcnt_hi((uint32_t)(m[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m[e], 0));
  return n;
}
__device__ inline int all_of(const unsigned long long (&m)[4]) {
  return __popcll(m[0]) + __popcll(m[1]) + __popcll(m[2]) + __popcll(m[3]);
}

// slots in which vectors of four may be loaded
__device__ inline bool in_fours(const Kv4EvictArgs &a, size_t cap) {
  return cap % 4 == 0 && (((uintptr_t)a.weight | (uintptr_t)a.pos) & 15) == 0;
}

// One workgroup per (sequence, head) finds the least key that stays, digit by digit (11 bits, a histogram each: the exponent's eight
// alone would send most weights to a few counters), how many of the positions that have it stay (the first ones do), and how
// many stay in front of every 256 slots.  What bounds it is one CU: of 32768 slots' 46 K clocks its vector units work 19 K (32 keys to a
// thread, 1170 instructions to a wavefront, as many scalar ones) and its wavefronts wait for 60 % of theirs, at the barriers of
// three digits and for what lies between them, so what can be done by more CUs is left to the next launch.  Up to 32768 slots their keys
// stay in registers; longer rows are read again for every digit.  Eight heads of 32768 slots 19 us, four of 2048 8 us; a histogram for each quarter of
// the lanes takes half a microsecond off both.  (One launch that also ranked and listed: 55 and 30 us.)
__global__ __launch_bounds__(kSelectThreads) void kv4_select_kernel(Kv4EvictArgs a) {
  const hb_attn_desc &d = a.d;
  __shared__ int hist[kCopies * kBins], s_sum[kSelectWaves];
  __shared__ int s_above[kRounds * kSelectWaves], s_ties[kRounds * kSelectWaves];
  __shared__ int s_digit, s_need;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x / d.num_kv_heads;
  const size_t cap = (size_t)d.max_blocks_per_seq * d.page_size;
  const int L = kv4_length(d, a.prefix_len, b), stays = L < a.budget ? L : a.budget;
  const float *w = a.weight + (size_t)blockIdx.x * cap;
  const int32_t *pos = a.pos + (size_t)blockIdx.x * cap;
  const int recent_from = a.seq_len[b] - a.recent;
  const bool vec = in_fours(a, cap);
  if (tid == 0) {
    if (blockIdx.x % d.num_kv_heads == 0 && a.new_len) a.new_len[b] = stays;
    if (stays == L) a.counts[blockIdx.x] = 0;  // else the next launch counts
  }
  const int slabs = (L + kSlab - 1) / kSlab;
  uint32_t keys[kRounds][4];
  auto load = [&](int slab) {
    f32x4 x;
    int32_t p[4];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int s = slab * kSlab + r * kSelectThreads * 4;
      keys[r][0] = keys[r][1] = keys[r][2] = keys[r][3] = 0;
      if (s < L) load_keys(w, pos, s + tid * 4, L, vec, recent_from, a.sinks, keys[r], x, p);  // uniform
    }
  };
  if (slabs == 1) load(0);
  uint32_t least = 0;  // the least key that stays, as far as it is known
  int need = 0;        // positions with that key that stay
  if (stays < L) {
    need = stays;
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048, known = pass == 2 ? 10 : 21;
      for (int i = tid; i < kCopies * bins; i += kSelectThreads) hist[i] = 0;
      __syncthreads();
      for (int slab = 0; slab < slabs; ++slab) {
        if (slabs > 1) load(slab);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
          if (slab * kSlab + r * kSelectThreads * 4 >= L) break;  // uniform
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t k = keys[r][e];
            // (the slots past the length fall into counter 0, which is above every position's digit: never reached)
            if (pass == 0 || ((k ^ least) >> known) == 0) atomicAdd(&hist[((k >> shift) & (bins - 1)) * kCopies + (lane & (kCopies - 1))], 1);
          }
        }
      }
      __syncthreads();
      // a thread's two counters, the largest digits first: the digit is where their running sum passes `need`
      const int top = bins - 1 - 2 * tid;
      int c0 = 0, c1 = 0;
      if (top > 0) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          c0 += hist[top * kCopies + i];
          c1 += hist[(top - 1) * kCopies + i];
        }
      }
      const int up = scan_lanes(c0 + c1);
      if (lane == 63) s_sum[wave] = up;
      __syncthreads();
      const int waves = scan_lanes(lane < kSelectWaves ? s_sum[lane] : 0);
      const int before = up - c0 - c1 + (wave ? __builtin_amdgcn_readlane(waves, wave - 1) : 0);
      if (before < need && before + c0 + c1 >= need) {  // one thread
        const bool first = before + c0 >= need;
        s_digit = first ? top : top - 1;
        s_need = need - before - (first ? 0 : c0);
      }
      __syncthreads();
      least |= (uint32_t)s_digit << shift;
      need = s_need;
    }
  }
  if (tid == 0) {
    a.least[blockIdx.x * 2] = (int32_t)least;
    a.least[blockIdx.x * 2 + 1] = need;
  }
  int32_t *parts = a.parts + (size_t)blockIdx.x * a.parts_each * 2;
  int above = 0, ties = 0;  // in front of the slab
  for (int slab = 0; slab < slabs; ++slab) {
    if (slabs > 1) load(slab);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (slab * kSlab + r * kSelectThreads * 4 >= L) break;  // uniform; what nobody counts, nobody reads: the parts end there
      unsigned long long ma[4], mt[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ma[e] = __ballot(keys[r][e] > least);
        mt[e] = __ballot(keys[r][e] == least && least != 0);
      }
      if (lane == 0) {
        s_above[r * kSelectWaves + wave] = all_of(ma);
        s_ties[r * kSelectWaves + wave] = all_of(mt);
      }
    }
    __syncthreads();
    if (wave == 0) {  // two of the slab's 128 parts to a lane
      const int x0 = s_above[2 * lane], x1 = s_above[2 * lane + 1], y0 = s_ties[2 * lane], y1 = s_ties[2 * lane + 1];
      const int x = above + scan_lanes(x0 + x1), y = ties + scan_lanes(y0 + y1);
      const int part = slab * (kSlab / kPart) + 2 * lane;
      if (part < a.parts_each) {
        parts[part * 2] = x - x0 - x1;
        parts[part * 2 + 1] = y - y0 - y1;
      }
      if (part + 1 < a.parts_each) {
        parts[part * 2 + 2] = x - x1;
        parts[part * 2 + 3] = y - y1;
      }
      if (lane == 63) {
        s_sum[0] = x;
        s_sum[1] = y;
      }
    }
    __syncthreads();
    above = s_sum[0];
    ties = s_sum[1];
    __syncthreads();
  }
}

// What stays where, 256 slots to a wavefront (eight heads of 32768 slots: 5 us): kept positions in front of the new length stay in their slot; the others are
// listed from the last one on, the slots that come free from the first.
__global__ __launch_bounds__(256) void kv4_list_kernel(Kv4EvictArgs a) {
  const hb_attn_desc &d = a.d;
  const int lane = threadIdx.x & 63, unit = blockIdx.y, b = unit / d.num_kv_heads;
  const size_t cap = (size_t)d.max_blocks_per_seq * d.page_size;
  const int L = kv4_length(d, a.prefix_len, b), stays = L < a.budget ? L : a.budget;
  int32_t *kept = a.kept + (size_t)unit * a.budget;
  for (long s = (long)stays + blockIdx.x * 256 + threadIdx.x; s < a.budget; s += (long)a.list_step * 64) kept[s] = -1;
  const uint32_t least = (uint32_t)a.least[unit * 2];
  const int need = a.least[unit * 2 + 1];
  const float *w = a.weight + unit * cap;
  const int32_t *pos = a.pos + unit * cap;
  // one part to a wavefront, more only where the row is longer than the host's bound
  for (int part = blockIdx.x * 4 + (threadIdx.x >> 6), s0 = part * kPart; s0 < L; part += a.list_step, s0 = part * kPart) {
    const int32_t *before = a.parts + ((size_t)unit * a.parts_each + part) * 2;
    const int above = before[0], ties = before[1];
    uint32_t key[4];
    f32x4 x;
    int32_t p[4];
    const int s = s0 + lane * 4;
    load_keys(w, pos, s, L, in_fours(a, cap), a.seq_len[b] - a.recent, a.sinks, key, x, p);
    unsigned long long m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = __ballot(key[e] == least && least != 0);
    int tie = ties + lanes_before(m);
    bool stay[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool t = key[e] == least && least != 0;
      stay[e] = key[e] > least || (t && tie < need);
      tie += t ? 1 : 0;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = __ballot(stay[e]);
    int n = above + min(ties, need) + lanes_before(m);  // that stay in front of slot s + e
    int32_t *from = a.moves + (size_t)unit * 2 * a.budget, *to = from + a.budget;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = s + e;
      if (at == stays && at < L) a.counts[unit] = stays - n;
      if (stay[e] && at < stays) {
        kept[at] = at;
        a.weight_out[unit * cap + at] = x[e];
        a.pos_out[unit * cap + at] = p[e];
      } else if (stay[e]) {
        from[stays - 1 - n] = at;
      } else if (at < stays) {
        to[at - n] = at;
      }
      n += stay[e] ? 1 : 0;
    }
  }
}

// Rows of K and V to the slots that came free for them: a lane takes a block of K or V (16 bytes and a scale), 2 D / 32 lanes a
// move, so that a wavefront has several in flight.  49 K rows of heads of 128, 13.4 MB read and written, scattered: 6 us, 2.2 TB/s (a wavefront a row: 22).
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4EvictArgs a) {
  const hb_attn_desc &d = a.d;
  const int blocks = d.head_dim / kKv4Block, lanes = 2 * blocks, each = 64 / lanes;
  const int lane = threadIdx.x & 63, part = lane % lanes, unit = blockIdx.y;
  int i = ((int)blockIdx.x * 4 + (threadIdx.x >> 6)) * each + lane / lanes;
  const int count = a.counts[unit];
  if (lane >= each * lanes || i >= count) return;
  const int b = unit / d.num_kv_heads, h = unit % d.num_kv_heads;
  const size_t cap = (size_t)d.max_blocks_per_seq * d.page_size;
  const int32_t *moves = a.moves + (size_t)unit * 2 * a.budget;
  auto move = [&] {
    const int src = moves[count - 1 - i], dst = moves[a.budget + i];
    const size_t s = kv4_row(d, a.block_table, b, h, src), t = kv4_row(d, a.block_table, b, h, dst);
    const bool value = part >= blocks;
    const int blk = value ? part - blocks : part;
    uint8_t *codes = value ? a.v_codes : a.k_codes, *scales = value ? a.v_scales : a.k_scales;
    ((u32x4 *)codes)[t * blocks + blk] = ((const u32x4 *)codes)[s * blocks + blk];
    scales[t * blocks + blk] = scales[s * blocks + blk];
    if (part == 0) {
      a.kept[(size_t)unit * a.budget + dst] = src;
      a.weight_out[unit * cap + dst] = a.weight[unit * cap + src];
    } else if (part == 1) {
      a.pos_out[unit * cap + dst] = a.pos[unit * cap + src];
    }
  };
  move();
  for (i += a.move_step; i < count; i += a.move_step) move();  // where the row is longer than the host's bound
}

}  // namespace

hipError_t launch_kv4_append(const Kv4AppendArgs &a, hipStream_t s) {
  const long threads = (long)a.rows * a.d.num_kv_heads * (a.d.head_dim / 8);
  const unsigned grid = (unsigned)(threads ? (threads + 255) / 256 : 1);
  const bool path = a.accept_path != nullptr;
  if (a.d.dtype == HB_F32) {
    if (path) kv4_append_kernel<float, true><<<grid, 256, 0, s>>>(a);
    else kv4_append_kernel<float, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (path) kv4_append_kernel<bf16_t, true><<<grid, 256, 0, s>>>(a);
    else kv4_append_kernel<bf16_t, false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_read(const hb_attn_desc &d, int32_t rows, const Kv4Pool &k, const Kv4Pool &v, const int32_t *block_table,
                           const int32_t *first, const int32_t *row_offset, void *k_rows, void *v_rows, hipStream_t s) {
  const long threads = (long)rows * d.num_kv_heads * (d.head_dim / 8);
  const unsigned grid = (unsigned)((threads + 255) / 256);
  if (d.dtype == HB_F32)
    kv4_read_kernel<float><<<grid, 256, 0, s>>>(d, rows, k, v, block_table, first, row_offset, (float *)k_rows, (float *)v_rows);
  else
    kv4_read_kernel<bf16_t><<<grid, 256, 0, s>>>(d, rows, k, v, block_table, first, row_offset, (bf16_t *)k_rows, (bf16_t *)v_rows);
  return hipGetLastError();
}

hipError_t launch_kv4_evict(Kv4EvictArgs a, hipStream_t s) {
  const int units = a.d.batch * a.d.num_kv_heads;
  const unsigned lists = (unsigned)((a.longest + 4 * kPart - 1) / (4 * kPart));
  const int each = 4 * (64 / (2 * (a.d.head_dim / kKv4Block)));  // moves of a workgroup
  const int most = a.budget < a.longest ? a.budget : a.longest;
  const unsigned moves = (unsigned)((most + each - 1) / each);
  a.list_step = (int32_t)lists * 4;
  a.move_step = (int32_t)moves * each;
  kv4_select_kernel<<<units, kSelectThreads, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  kv4_list_kernel<<<dim3(lists, (unsigned)units), 256, 0, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  kv4_move_kernel<<<dim3(moves, (unsigned)units), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace hb
