// Attention weights of cached positions on the matrix cores (heads of 64 and 128, pages of a multiple of 16).
//
//   S = Q K^T   v_mfma_f32_16x16x32_bf16: A = 16 query rows, B = 16 cached keys, widened to bf16, which is exact
//   w_p = decay w_p + sum over rows of exp(S[row][p] - lse[row])
// The weights are 32-bit results, so the scores are too.  float32 queries are taken as three bf16 pieces (kv4.h), smallest first.
//
// Each key is 4 bits an element and 8 bytes for its weight; up to some ten rows that bounds it, from there on the exponentials
// (16 clocks for 64 of them): six nodes of 28/4 heads are 42 rows.  16 sequences of 1024 to 8192 positions, 23 MB, take 15 to 17 us (4.5 at
// the rate of a copy), of which the matrix cores work 1 and the vector unit 4; the rest are round trips, to lengths, paths and
// pages, to codes, to queries, and workgroups that find their chunk behind the end of a sequence.  One token over 2048: 5 us.
// A wavefront takes 64 keys, requested in one go; lane
// (j, kg) holds block kg of key j of each 16, and as the products' order of d is free, the block is its operand as it is.  The
// rows' queries lie in LDS, 64 rows (float32: 32) at a time, shared by the workgroup; a lane's sum over its rows
// crosses lanes once, at the end.
#include "kv4.h"

namespace hb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int swap2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;
constexpr int kKeys = 64;  // of a wavefront
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float group_sum(float x) {
  swap2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// eight elements of a row as bf16 pieces, largest first
__device__ __forceinline__ void pieces_of(const bf16_t *p, u32x4 (&x)[1]) { x[0] = *(const u32x4 *)p; }
__device__ __forceinline__ void pieces_of(const float *p, u32x4 (&x)[3]) {
  const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float lo = e < 2 ? a[2 * e] : b[2 * e - 4], hi = e < 2 ? a[2 * e + 1] : b[2 * e - 3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const uint32_t w = i == 0 ? kv4_pack_cut(lo, hi) : pack_bf16(lo, hi);
      x[i][e] = w;
      lo -= __uint_as_float(w << 16);
      hi -= __uint_as_float(w & 0xffff0000u);
    }
  }
}

// (three wavefronts to a SIMD: 16 sequences 16.7 us, with registers for two 18.8, for four 17.3; float32's allow three untold)
template <typename T, int DB>
__global__ __launch_bounds__(64 * kWaves, sizeof(T) == 4 ? 2 : 3) void kv4_weight_kernel(Kv4WeightArgs a, uint32_t page_magic, int rounds, int stride) {
  constexpr int P = sizeof(T) == 4 ? 3 : 1, kRows = sizeof(T) == 4 ? 32 : 64, D = 32 * DB;
  const hb_attn_desc &d = a.d;
  // 16-byte pieces [row][piece of bf16][d / 8], the last index XORed with the row so that 16 rows' reads spread over the banks
  __shared__ u32x4 s_q[kRows * P * 4 * DB];
  __shared__ float s_lse[kRows];
  __shared__ int s_path[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, kg = lane >> 4;
  // units are neighbours, not chunks: workgroup ids go round the XCDs, and the chunks behind short sequences are empty
  const int h = blockIdx.x % d.num_kv_heads, b = blockIdx.x / d.num_kv_heads, G = d.num_q_heads / d.num_kv_heads;
  // a wavefront's keys: 64 in each round, the first at k0; what has to be known first is asked for in one go
  const int share = rounds * kWaves * kKeys;
  int begin = (int)(blockIdx.z * gridDim.y + blockIdx.y) * share, k0 = begin + wave * kKeys;
  const int cap16 = d.max_blocks_per_seq * (d.page_size / 16);
  const int32_t *table = a.block_table + (size_t)b * d.max_blocks_per_seq;
  // lane 4 r + t: the page of the t-th 16 keys of round r
  auto ask_pages = [&] {
    const int at16 = min((k0 >> 4) + (lane >> 2) * (kWaves * 4) + (lane & 3), cap16 - 1);
    return table[page_magic ? (int)__umulhi((uint32_t)at16, page_magic) : at16];
  };
  int pages = ask_pages();
  const int n0 = a.node_offset[b], n1 = a.node_offset[b + 1], accepted = a.accept_path ? a.accept_len[b] : 0;
  const bool short_path = a.accept_path && a.max_path <= 64;
  if (short_path && tid < a.max_path) s_path[tid] = a.accept_path[(size_t)b * a.max_path + tid];
  const int L = kv4_length(d, a.prefix_len, b);
  if (begin >= L) return;
  int end = min(L, begin + share);
  const int n = n1 - n0 < 0 || n0 < 0 || n1 > d.total_nodes ? 0 : n1 - n0;
  int nodes = a.accept_path ? accepted : n;
  nodes = nodes < 0 || n == 0 ? 0 : a.accept_path && nodes > a.max_path ? a.max_path : nodes;
  const int rows = nodes * G;
  const float c1 = d.softmax_scale * kLog2e;
  float *weight = a.weight + ((size_t)b * d.num_kv_heads + h) * d.max_blocks_per_seq * d.page_size;
  pages = max(0, min(pages, d.num_blocks - 1));

  struct Keys {
    u32x4 k[4];
    uint32_t scale[4];
    float old[4];
  };
  auto load = [&](int round, Keys &x) {
    const int first = k0 + round * kWaves * kKeys;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      x.k[t] = (u32x4){0u, 0u, 0u, 0u};
      x.scale[t] = 127;
      x.old[t] = 0.f;
      if (first + 16 * t < end) {  // uniform
        const int at = (first >> 4) + t, page = page_magic ? (int)__umulhi((uint32_t)at, page_magic) : at;
        const int blk = __builtin_amdgcn_readlane(pages, 4 * round + t);
        const size_t row = ((size_t)blk * d.num_kv_heads + h) * d.page_size + (at * 16 - page * d.page_size) + j;
        if (DB == 4 || kg < DB) {
          x.k[t] = *(const u32x4 *)(a.kp.codes + row * (D / 2) + kg * 16);
          x.scale[t] = a.kp.scales[row * DB + kg];
        }
        if (first + 16 * t + j < end) x.old[t] = weight[first + 16 * t + j];
      }
    }
  };

  // rows r0 .. r0 + kRows - 1 into LDS, a thread's pieces of them asked for in one go; past the last: zeros that weigh nothing
  auto stage = [&](int r0) {
    constexpr int kItems = kRows * 4 * DB / (64 * kWaves);
    const int there = min(kRows, (rows - r0 + 15) / 16 * 16);
    u32x4 x[kItems][P];
    float lse[kItems];
#pragma unroll
    for (int q = 0; q < kItems; ++q) {
      const int i = tid + q * 64 * kWaves, piece = i % (4 * DB), row = r0 + i / (4 * DB);
#pragma unroll
      for (int p = 0; p < P; ++p) x[q][p] = (u32x4){0u, 0u, 0u, 0u};
      lse[q] = __builtin_huge_valf();
      if (row < rows) {
        // row / G for both below 2^22: the quotient of the reciprocal is at most one off
        int node = (int)((float)row * __builtin_amdgcn_rcpf((float)G));
        node += (node + 1) * G <= row ? 1 : 0;
        node -= node * G > row ? 1 : 0;
        const int hg = row - node * G;
        if (a.accept_path) node = short_path ? s_path[node] : a.accept_path[(size_t)b * a.max_path + node];
        node = node < 0 ? 0 : node >= n ? n - 1 : node;
        const size_t at = (size_t)(n0 + node) * d.num_q_heads + h * G + hg;
        pieces_of((const T *)a.q + at * D + piece * 8, x[q]);
        if (piece == 0) lse[q] = a.lse[at] * kLog2e;
      }
    }
#pragma unroll
    for (int q = 0; q < kItems; ++q) {
      const int i = tid + q * 64 * kWaves, piece = i % (4 * DB), r = i / (4 * DB);
      if (r >= there) continue;
      if (piece == 0) s_lse[r] = lse[q];
#pragma unroll
      for (int p = 0; p < P; ++p) s_q[(r * P + p) * 4 * DB + (piece ^ (r & (4 * DB - 1)))] = x[q][p];
    }
  };

  Keys x;
  load(0, x);
  const bool one_batch = rows <= kRows;
  __syncthreads();  // the path
  if (one_batch) {
    stage(0);
    __syncthreads();
  }
  // every wavefront goes round as often as the others: there are barriers inside where rows come in batches
  for (;;) {
    for (int round = 0; begin + round * kWaves * kKeys < end; ++round) {
      const int first = k0 + round * kWaves * kKeys;
      float old[4];
      bf16x8 bk[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        old[t] = x.old[t];
        const float s = __uint_as_float(x.scale[t] << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4 y;
          y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[t][i], s, 0));
          y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[t][i], s, 1));
          y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[t][i], s, 2));
          y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.k[t][i], s, 3));
          bk[t][i] = __builtin_bit_cast(bf16x8, y);
        }
      }
      load(round + 1, x);  // on its way during the products
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      for (int r0 = 0; r0 < rows; r0 += kRows) {
        if (!one_batch) {
          __syncthreads();  // the batch before has been read
          stage(r0);
          __syncthreads();
        }
        const int tiles = (min(kRows, rows - r0) + 15) / 16;
        for (int rt = 0; rt < tiles; ++rt) {
          f32x4 sc[4] = {};
#pragma unroll
          for (int p = P - 1; p >= 0; --p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = rt * 16 + j;
              // d = 32 kg + 8 i + 0 .. 7; where a head has two blocks, the keys' other lanes hold zeros
              const int piece = DB == 4 ? 4 * kg + i : 4 * (kg & 1) + i;
              const bf16x8 q = __builtin_bit_cast(bf16x8, s_q[(r * P + p) * 4 * DB + (piece ^ (r & (4 * DB - 1)))]);
#pragma unroll
              for (int t = 0; t < 4; ++t) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, bk[t][i], sc[t], 0, 0, 0);
            }
          const f32x4 lse = *(const f32x4 *)&s_lse[rt * 16 + 4 * kg];
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[t] += __builtin_amdgcn_exp2f(fmaf(sc[t][r], c1, -lse[r]));
        }
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float all = group_sum(sum[t]);
        // lane group t writes the t-th 16 keys
        if (kg == t && first + 16 * t + j < end) weight[first + 16 * t + j] = fmaf(old[t], a.decay, all);
      }
    }
    if (L - begin <= stride) break;  // always, but where the prefix is longer than the host's bound
    begin += stride;
    k0 += stride;
    end = min(L, begin + share);
    pages = max(0, min(ask_pages(), d.num_blocks - 1));
    load(0, x);
  }
}

}  // namespace

bool kv4_weight_supports(const hb_attn_desc &d) {
  return (d.head_dim == 64 || d.head_dim == 128) && d.page_size % 16 == 0 && d.page_size <= 1024;
}

hipError_t launch_kv4_weight_mfma(const Kv4WeightArgs &a, int32_t longest, hipStream_t s) {
  const int page16 = a.d.page_size / 16;
  const uint32_t magic = page16 == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + page16 - 1) / page16);
  const int64_t units = (int64_t)a.d.batch * a.d.num_kv_heads;
  // 256 keys to a workgroup, more where that gives more than four workgroups a CU: their queries are staged once
  int64_t rounds = units * longest / (256 * 1024);
  rounds = rounds < 1 ? 1 : rounds > 8 ? 8 : rounds;  // a wavefront holds the pages of sixteen rounds
  const int keys = (int)rounds * kWaves * kKeys;
  const unsigned chunks = (unsigned)((longest + keys - 1) / keys), rows_of_grid = chunks < 32768 ? chunks : 32768;
  const dim3 grid((unsigned)units, rows_of_grid, (chunks + rows_of_grid - 1) / rows_of_grid);
  const int stride = (int)(grid.y * grid.z) * keys;  // of all workgroups of a unit
  const bool f32 = a.d.dtype == HB_F32;
  if (a.d.head_dim == 128) {
    if (f32) kv4_weight_kernel<float, 4><<<grid, 64 * kWaves, 0, s>>>(a, magic, (int)rounds, stride);
    else kv4_weight_kernel<bf16_t, 4><<<grid, 64 * kWaves, 0, s>>>(a, magic, (int)rounds, stride);
  } else {
    if (f32) kv4_weight_kernel<float, 2><<<grid, 64 * kWaves, 0, s>>>(a, magic, (int)rounds, stride);
    else kv4_weight_kernel<bf16_t, 2><<<grid, 64 * kWaves, 0, s>>>(a, magic, (int)rounds, stride);
  }
  return hipGetLastError();
}

}  // namespace hb
