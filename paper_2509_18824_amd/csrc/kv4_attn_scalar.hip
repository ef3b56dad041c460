// Attention and attention weights over the 4-bit cache in 32-bit arithmetic, for every type, head size and page size: one
// workgroup per (node, query head, chunk of the prefix); the wavefronts deal out blocks of 64 keys.  A lane takes one key of a
// block for the scores and two elements of the head (or four) for the values.  It is the kernel for heads that are neither 64 nor
// 128, for pages that are no multiple of 16 and for scales that are not positive, and bounded by the round trips of a block: one
// to the pages, one to the keys, four to the values.  (Four nodes of four float32 heads of 64 over 256 positions: 17 us.)
#include "kv4.h"

namespace hb {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kRowsInFlight = 16;  // of values

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline float wave_max(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
  return x;
}
__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// <q, k> of one cached row; q in LDS
__device__ inline float dot_row(const hb_attn_desc &d, const Kv4Pool &pool, size_t row, const float *q) {
  const u32x4 *codes = (const u32x4 *)(pool.codes + row * (d.head_dim / 2));
  const uint8_t *scales = pool.scales + row * (d.head_dim / kKv4Block);
  float sum = 0.f;
  for (int blk = 0; blk < d.head_dim / kKv4Block; ++blk) {
    const u32x4 c = codes[blk];
    const uint32_t scale = scales[blk];
    // scaled one by one, which costs nothing and is exact: queries times codes alone may be larger than any product
    const float s = __uint_as_float((scale == kKv4NaN ? 127u : scale) << 23);
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float *x = q + blk * kKv4Block + i * 8;
      const kv4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 1);
      const kv4_f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 3);
      part = fmaf(a[0], x[0], part), part = fmaf(a[1], x[1], part), part = fmaf(b[0], x[2], part), part = fmaf(b[1], x[3], part);
      part = fmaf(e[0], x[4], part), part = fmaf(e[1], x[5], part), part = fmaf(f[0], x[6], part), part = fmaf(f[1], x[7], part);
    }
    sum += scale == kKv4NaN ? __builtin_nanf("") : part;
  }
  return sum;
}

// running softmax of a wavefront: reference, sum (lane 0 .. 63 all hold it), accumulated values of the lane's elements
struct State {
  float m, l, acc[4];
};

// Moves the reference to cover a block's scores; returns this lane's weight.  Scores of -inf weigh nothing, also where there
// is nothing else yet.
__device__ inline float block_weight(State &st, float score, bool there) {
  const float m = fmaxf(st.m, wave_max(there ? score : -__builtin_huge_valf()));
  const float ref = m == -__builtin_huge_valf() ? 0.f : m;
  const float corr = expf(st.m - ref);
  const float p = there ? expf(score - ref) : 0.f;
  st.m = m;
  st.l = st.l * corr + wave_sum(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) st.acc[e] *= corr;
  return p;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_attn_scalar_kernel(Kv4AttnArgs a) {
  const hb_attn_desc &d = a.d;
  __shared__ float q[256], ml[kWaves][2], part[kWaves][256];
  __shared__ unsigned long long s_path;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.x, node = r / d.num_q_heads, head = r % d.num_q_heads, c = blockIdx.y;
  const int g = head / (d.num_q_heads / d.num_kv_heads), D = d.head_dim;
  const int b = kv4_sequence(a.node_offset, d.batch, node);
  const int n0 = a.node_offset[b];
  int n = a.node_offset[b + 1] - n0;
  n = n < 0 ? 0 : n > d.max_nodes_per_tree ? d.max_nodes_per_tree : n;
  if (n0 < 0 || n0 + n > d.total_nodes) n = 0;
  if (node < n0 || node >= n0 + n) return;  // malformed offsets
  const int L = kv4_length(d, a.prefix_len, b);
  const int begin = c * a.chunk, end = c + 1 == a.splits ? L : min(L, begin + a.chunk);  // (lengths beyond the host's bound)
  for (int i = tid; i < D; i += kThreads) q[i] = load_f32((const T *)a.q + (size_t)r * D + i) * d.softmax_scale;
  if (tid == 0) {
    unsigned long long path = 0;
    for (int x = node - n0, guard = 0; x >= 0 && guard < 64; ++guard) {
      path |= 1ull << x;
      const int up = a.parent[n0 + x];
      x = up < x ? up : -1;
    }
    s_path = path;
  }
  __syncthreads();
  State st = {-__builtin_huge_valf(), 0.f, {0.f, 0.f, 0.f, 0.f}};
  for (int k0 = begin + wave * 64; k0 < end; k0 += kThreads) {
    const int p = k0 + lane;
    const bool there = p < end;
    const size_t row = there ? kv4_row(d, a.block_table, b, g, p) : 0;
    const float w = block_weight(st, there ? dot_row(d, a.kp, row, q) : 0.f, there);
    // values, kRowsInFlight rows asked for before the first is used; a key past the end weighs nothing and reads the block's
    // first row, whose values are zeroed
    const int keys = min(64, end - k0);
    for (int i0 = 0; i0 < keys; i0 += kRowsInFlight) {
      uint32_t v[kRowsInFlight][2], vs[kRowsInFlight][2];
#pragma unroll
      for (int i = 0; i < kRowsInFlight; ++i) {
        const int from = i0 + i < keys ? i0 + i : 0;
        const size_t vr = ((size_t)(uint32_t)__shfl((int)(row >> 32), from, 64) << 32) | (uint32_t)__shfl((int)row, from, 64);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int byte = lane + 64 * e;  // elements 2 byte, 2 byte + 1
          v[i][e] = 0;
          vs[i][e] = 127;
          if (byte < D / 2 && i0 + i < keys) {
            v[i][e] = a.vp.codes[vr * (D / 2) + byte];
            vs[i][e] = a.vp.scales[vr * (D / kKv4Block) + byte / 16];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kRowsInFlight; ++i) {
        const float pi = __shfl(w, i0 + i, 64);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const kv4_f32x2 x = kv4_pair<0>(v[i][e], kv4_scale(vs[i][e]));
          st.acc[2 * e] = fmaf(pi, x[0], st.acc[2 * e]);
          st.acc[2 * e + 1] = fmaf(pi, x[1], st.acc[2 * e + 1]);
        }
      }
    }
  }
  if (c == 0 && wave == 0) {  // the node's own path
    const bool there = lane < n && ((s_path >> lane) & 1);
    float s = 0.f;
    if (there) {
      const T *k = (const T *)a.k_tree + ((size_t)(n0 + lane) * d.num_kv_heads + g) * D;
#pragma unroll 16
      for (int i = 0; i < D; ++i) s = fmaf(load_f32(k + i), q[i], s);
    }
    const float w = block_weight(st, s, there);
    for (int i = 0; i < n; ++i) {
      const float pi = __shfl(w, i, 64);
      if (!((s_path >> i) & 1)) continue;
      const T *v = (const T *)a.v_tree + ((size_t)(n0 + i) * d.num_kv_heads + g) * D;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int byte = lane + 64 * e;
        if (byte < D / 2) {
          st.acc[2 * e] = fmaf(pi, load_f32(v + 2 * byte), st.acc[2 * e]);
          st.acc[2 * e + 1] = fmaf(pi, load_f32(v + 2 * byte + 1), st.acc[2 * e + 1]);
        }
      }
    }
  }
  if (lane == 0) {
    ml[wave][0] = st.m;
    ml[wave][1] = st.l;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (lane + 64 * e < D / 2) {
      part[wave][2 * (lane + 64 * e)] = st.acc[2 * e];
      part[wave][2 * (lane + 64 * e) + 1] = st.acc[2 * e + 1];
    }
  __syncthreads();
  float m = -__builtin_huge_valf(), l = 0.f;
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w][0]);
  const float ref = m == -__builtin_huge_valf() ? 0.f : m;
  for (int w = 0; w < kWaves; ++w) l += ml[w][1] * expf(ml[w][0] - ref);
  for (int i = tid; i < D; i += kThreads) {
    float o = 0.f;
    for (int w = 0; w < kWaves; ++w) o += part[w][i] * expf(ml[w][0] - ref);
    if (a.splits == 1) store_f32((T *)a.out + (size_t)r * D + i, o / l);
    else a.part_o[((size_t)r * a.splits + c) * D + i] = o;
  }
  if (tid == 0) {
    if (a.splits > 1) {
      a.part_ml[((size_t)r * a.splits + c) * 2] = m;
      a.part_ml[((size_t)r * a.splits + c) * 2 + 1] = l;
    } else if (a.lse) {
      a.lse[r] = m + logf(l);
    }
  }
}

// Joins the chunks' partial results of a row: every slot is filled, one without keys with sum 0.
template <typename T>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4AttnArgs a) {
  const int D = a.d.head_dim, tpr = D / 4;
  const long gid = (long)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(gid / tpr), piece = (int)(gid % tpr);
  if (row >= a.d.total_nodes * a.d.num_q_heads) return;
  const float *ml = a.part_ml + (size_t)row * a.splits * 2;
  float m = -__builtin_huge_valf(), l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int c = 0; c < a.splits; ++c) m = fmaxf(m, ml[2 * c]);
  const float ref = m == -__builtin_huge_valf() ? 0.f : m;
  for (int c = 0; c < a.splits; ++c) {
    if (ml[2 * c + 1] == 0.f) continue;
    const float w = expf(ml[2 * c] - ref);
    l = fmaf(ml[2 * c + 1], w, l);
    const float *p = a.part_o + ((size_t)row * a.splits + c) * D + piece * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(p[e], w, o[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) store_f32((T *)a.out + (size_t)row * D + piece * 4 + e, o[e] / l);
  if (a.lse && piece == 0) a.lse[row] = m + logf(l);
}

// Attention weight that every cached position received: a lane takes one position, a wavefront 64 of them.
template <typename T>
__global__ __launch_bounds__(kThreads) void kv4_weight_scalar_kernel(Kv4WeightArgs a) {
  const hb_attn_desc &d = a.d;
  __shared__ float q[256];
  const int tid = threadIdx.x, h = blockIdx.y % d.num_kv_heads, b = blockIdx.y / d.num_kv_heads, G = d.num_q_heads / d.num_kv_heads;
  const int L = kv4_length(d, a.prefix_len, b);
  const int n0 = a.node_offset[b];
  int n = a.node_offset[b + 1] - n0;
  n = n < 0 || n0 < 0 || n0 + n > d.total_nodes ? 0 : n;
  int rows = a.accept_path ? a.accept_len[b] : n;
  rows = rows < 0 || n == 0 ? 0 : a.accept_path && rows > a.max_path ? a.max_path : rows;
  // once, but where the prefix is longer than the host's bound
  for (int s0 = blockIdx.x * kThreads; s0 < L; s0 += gridDim.x * kThreads) {
    const int s = s0 + tid;
    const size_t row = s < L ? kv4_row(d, a.block_table, b, h, s) : 0;
    float sum = 0.f;
    for (int i = 0; i < rows * G; ++i) {
      int node = a.accept_path ? a.accept_path[(size_t)b * a.max_path + i / G] : i / G;
      node = node < 0 ? 0 : node >= n ? n - 1 : node;
      const size_t r = (size_t)(n0 + node) * d.num_q_heads + h * G + i % G;
      __syncthreads();
      for (int e = tid; e < d.head_dim; e += kThreads) q[e] = load_f32((const T *)a.q + r * d.head_dim + e) * d.softmax_scale;
      __syncthreads();
      if (s < L) sum += expf(dot_row(d, a.kp, row, q) - a.lse[r]);
    }
    if (s < L) {
      float *w = a.weight + ((size_t)b * d.num_kv_heads + h) * d.max_blocks_per_seq * d.page_size + s;
      *w = fmaf(*w, a.decay, sum);
    }
  }
}

}  // namespace

hipError_t launch_kv4_attn_scalar(const Kv4AttnArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(a.d.total_nodes * a.d.num_q_heads), (unsigned)a.splits);
  if (a.d.dtype == HB_F32) kv4_attn_scalar_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else kv4_attn_scalar_kernel<bf16_t><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv4_merge(const Kv4AttnArgs &a, hipStream_t s) {
  const long threads = (long)a.d.total_nodes * a.d.num_q_heads * (a.d.head_dim / 4);
  const unsigned grid = (unsigned)((threads + 255) / 256);
  if (a.d.dtype == HB_F32) kv4_merge_kernel<float><<<grid, 256, 0, s>>>(a);
  else kv4_merge_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv4_weight_scalar(const Kv4WeightArgs &a, int32_t longest, hipStream_t s) {
  const dim3 grid((unsigned)((longest + kThreads - 1) / kThreads), (unsigned)(a.d.batch * a.d.num_kv_heads));
  if (a.d.dtype == HB_F32) kv4_weight_scalar_kernel<float><<<grid, kThreads, 0, s>>>(a);
  else kv4_weight_scalar_kernel<bf16_t><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace hb
