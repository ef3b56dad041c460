// Pages of the paged cache: taken from a list of free ones for requests that grow, given back by those that end or are cut
// (hb_pages_take, hb_pages_give), and rows of K and V written to their slots (hb_kv_append).
//
// Taking and giving are prefix sums over the requests' page counts.  Every workgroup makes the sums that it needs by itself
// (a few thousand numbers that everybody reads sit in L2; a second launch would cost more), writes the entries and slots of
// one sequence, or of a share of its rows, and no workgroup reads what another writes.  What bounds them is a launch and the round
// trips to lengths, sums and pages: 16 sequences of 8 new rows 4.9 us, 256 prompts of up to 1024 rows 5.0, 64 sequences that give 3.6.
#include "pages.h"

namespace hb {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Taken {
  int64_t len, rows, want, have, need;  // positions (negative: an empty place), new rows, pages wanted, pages there, pages to take
  bool fits;
};
__device__ __forceinline__ Taken wanted(const PagesArgs &a, int b) {
  Taken t;
  const int64_t cap = (int64_t)a.max_blocks * a.page;
  const int32_t len = a.len[b], have = a.have[b];
  t.len = len > cap ? cap : len;
  t.have = have < 0 ? 0 : have > a.max_blocks ? a.max_blocks : have;
  const int64_t r0 = a.row_offset[b], r1 = a.row_offset[b + 1];
  const bool hold = r0 >= 0 && r1 >= r0 && (!a.slots || r1 <= a.n_rows);  // the slots hold its rows
  t.rows = hold ? r1 - r0 : 0;
  t.want = (t.len + t.rows + a.reserve + a.page - 1) / a.page;
  t.fits = hold && len >= 0 && t.want <= a.max_blocks;
  t.need = t.fits && t.want > t.have ? t.want - t.have : 0;
  return t;
}

__device__ __forceinline__ int64_t sum_block(int64_t x, int64_t *lds) {
  for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  x = lds[0] + lds[1] + lds[2] + lds[3];
  __syncthreads();
  return x;
}

__global__ __launch_bounds__(256) void pages_take_kernel(PagesArgs a) {
  __shared__ int64_t lds[4];
  const int b = blockIdx.x, tid = threadIdx.x;
  int64_t excl = 0;
  for (int i = tid; i < b; i += 256) excl += wanted(a, i).need;
  excl = sum_block(excl, lds);
  const Taken t = wanted(a, b);
  int64_t count = *a.free_count;
  count = count < 0 ? 0 : count > a.num_blocks ? a.num_blocks : count;
  const bool granted = t.fits && (t.need == 0 || excl + t.need <= count);

  if (blockIdx.y == 0) {
    if (tid == 0) {
      a.have_out[b] = (int32_t)(granted && t.want > t.have ? t.want : t.have);
      if (a.new_len) a.new_len[b] = (int32_t)(granted ? t.len + t.rows : t.len);
      if (a.granted) a.granted[b] = granted;
    }
    if (b == a.batch - 1) {
      // pages taken: the largest of the sums up to a sequence that there are pages for
      int64_t taken = 0, before = 0;
      for (int i0 = 0; i0 < a.batch; i0 += 256) {
        int64_t x = i0 + tid < a.batch ? wanted(a, i0 + tid).need : 0;
        for (int m = 1; m < 64; m <<= 1) {
          const int64_t y = __shfl_up(x, m, 64);
          if ((tid & 63) >= m) x += y;
        }
        if ((tid & 63) == 63) lds[tid >> 6] = x;
        __syncthreads();
        for (int w = 0; w < tid >> 6; ++w) x += lds[w];
        x += before;
        before += lds[0] + lds[1] + lds[2] + lds[3];
        __syncthreads();
        if (x <= count && x > taken) taken = x;
      }
      for (int m = 32; m; m >>= 1) {
        const int64_t y = __shfl_xor(taken, m, 64);
        taken = y > taken ? y : taken;
      }
      if ((tid & 63) == 0) lds[tid >> 6] = taken;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < 4; ++w) taken = lds[w] > taken ? lds[w] : taken;
        *a.left = (int32_t)(count - taken);
      }
    }
  }

  // page of table entry e >= have
  auto page_of = [&](int64_t e) {
    const int64_t at = count - 1 - (excl + e - t.have);
    return a.free_pages[at < 0 ? 0 : at];  // at < count <= num_blocks
  };
  int32_t *row = a.table + (size_t)b * a.max_blocks;
  const int step = gridDim.y * 256, first = blockIdx.y * 256 + tid;
  if (granted)
    for (int64_t e = t.have + first; e < t.want; e += step) row[e] = page_of(e);
  if (!a.slots) return;
  for (int64_t j = first; j < t.rows; j += step) {
    int32_t slot = -1;
    if (granted) {
      const int64_t p = t.len + j, e = p / a.page;
      const int32_t id = e < t.have ? row[e] : page_of(e);
      if (id >= 0 && id < a.num_blocks) slot = (int32_t)((int64_t)id * a.page + (p - e * a.page));
    }
    a.slots[a.row_offset[b] + j] = slot;
  }
}

__global__ __launch_bounds__(256) void pages_give_kernel(PagesArgs a) {
  __shared__ int64_t lds[4];
  const int b = blockIdx.x, tid = threadIdx.x;
  auto given = [&](int i, int64_t &keep) {
    int64_t have = a.have[i], len = a.len[i];
    have = have < 0 ? 0 : have > a.max_blocks ? a.max_blocks : have;
    keep = len <= 0 ? 0 : (len + a.page - 1) / a.page;
    keep = keep > have ? have : keep;
    return have - keep;
  };
  int64_t excl = 0, total = 0, keep;
  for (int i = tid; i < a.batch; i += 256) {
    const int64_t n = given(i, keep);
    total += n;
    if (i < b) excl += n;
  }
  excl = sum_block(excl, lds);
  total = sum_block(total, lds);
  const int64_t n = given(b, keep);
  int64_t count = *a.free_count;
  count = count < 0 ? 0 : count > a.num_blocks ? a.num_blocks : count;
  if (blockIdx.y == 0 && tid == 0) {
    a.have_out[b] = (int32_t)keep;
    if (b == 0) *a.left = (int32_t)(count + total < a.num_blocks ? count + total : a.num_blocks);
  }
  const int32_t *row = a.table + (size_t)b * a.max_blocks;
  for (int64_t i = blockIdx.y * 256 + tid; i < n; i += gridDim.y * 256) {
    const int64_t at = count + total - 1 - (excl + i);
    if (at < a.num_blocks) a.free_out[at] = row[keep + i];
  }
}

// A wavefront copies a row of K and of V, 16 bytes a lane and step.
__global__ __launch_bounds__(256) void kv_append_kernel(int n, int Hkv, int page, int pieces, int64_t slots_end, const u32x4 *k, const u32x4 *v,
                                                        const int32_t *slots, u32x4 *k_pool, u32x4 *v_pool) {
  const int lane = threadIdx.x & 63, each = Hkv * pieces;
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < n; r += (int64_t)gridDim.x * 4) {
    const int32_t slot = slots[r];
    if (slot < 0 || slot >= slots_end) continue;
    const int id = slot / page, off = slot - id * page;
    for (int i = lane; i < each; i += 64) {
      const int h = i / pieces;
      const size_t to = (((size_t)id * Hkv + h) * page + off) * pieces + (i - h * pieces), from = (size_t)r * each + i;
      const u32x4 x = k[from], y = v[from];
      k_pool[to] = x;
      v_pool[to] = y;
    }
  }
}

// workgroups of a sequence, of which each writes some thousand items
unsigned shares(int64_t items) {
  const int64_t y = (items + 1023) / 1024;
  return (unsigned)(y < 1 ? 1 : y > 64 ? 64 : y);
}

}  // namespace

hipError_t launch_pages_take(const PagesArgs &a, hipStream_t s) {
  pages_take_kernel<<<dim3(a.batch, shares(a.slots ? a.n_rows / a.batch : a.max_blocks)), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_give(const PagesArgs &a, hipStream_t s) {
  pages_give_kernel<<<dim3(a.batch, shares(a.num_blocks / a.batch)), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_append(const hb_attn_desc &d, int32_t n, const void *k, const void *v, const int32_t *slots, void *k_pool,
                            void *v_pool, hipStream_t s) {
  const int pieces = d.head_dim * (d.dtype == HB_F32 ? 4 : 2) / 16;
  const int64_t groups = ((int64_t)n + 3) / 4;
  kv_append_kernel<<<(unsigned)(groups < 1 << 20 ? groups : 1 << 20), 256, 0, s>>>(
      n, d.num_kv_heads, d.page_size, pieces, (int64_t)d.num_blocks * d.page_size, (const u32x4 *)k, (const u32x4 *)v, slots,
      (u32x4 *)k_pool, (u32x4 *)v_pool);
  return hipGetLastError();
}

}  // namespace hb
