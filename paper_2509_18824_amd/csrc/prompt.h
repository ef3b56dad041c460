// What the kernels of hb_prompt_attn share: the call's arguments, and what a workgroup finds out about its work by itself.
//
// The query rows of a (sequence, kv head) are the pairs (prompt row, query head of the group), row = token * G + head: every
// key tile is read once for all heads of the group, and a short prompt fills a tile of rows G times as fast.  A tile is `bm`
// such rows.  Keys are one line: the prefix positions 0 .. P - 1, then the prompt's own rows; token i sees keys 0 .. P + i.
// The host knows neither lengths nor tiles: it launches a workgroup for every tile that `total_nodes` rows in `batch`
// sequences can have, and for every part that a tile's keys may be cut into.  Each workgroup reads the lengths (a lane a
// sequence), finds its tile, and from the work of all tiles the length of a part.
#pragma once
#include "hb_internal.h"
#include "wave_ops.h"

namespace hb {

struct PromptArgs {
  hb_attn_desc d;
  const void *q, *k, *v, *k_pool, *v_pool;               // the pools and the two below may be null: no prefix
  const int32_t *block_table, *prefix_len, *row_offset;
  void *out;
  float *lse;             // may be null
  float *part_o, *part_ml;  // [tile][kv head][part][row of bm][D], and [..][4]: largest score (base 2), sum that
                            // results are divided by, sum for the log-sum-exp, nothing
  int32_t tiles, parts;   // tiles of all sequences at most; parts of a tile's keys at most
  int32_t units;          // (tile, part, kv head) that the launch should come to
};

struct PromptTile {
  int b, t;        // sequence; tile of it (-1: this workgroup has none)
  int n, P;        // its prompt rows and prefix positions
  int row0;        // its first prompt row
  int tokens_end;  // keys that the tile's last row sees, less P
  int parts, begin, end;  // parts of the tile's keys; this one's keys
};

__device__ __forceinline__ int prompt_rows_of(const PromptArgs &a, int b, int &row0) {
  row0 = a.row_offset[b];
  int n = a.row_offset[b + 1] - row0;
  if (row0 < 0 || n < 0 || row0 > a.d.total_nodes - n) n = 0;  // malformed offsets: touch nothing
  return n;
}

// Every lane of the wavefront calls it with the same arguments.  Tiles of a sequence are numbered from its last (which sees
// the most keys) to its first, so that the longest work begins first.
template <int BM, int KEYS>
__device__ __forceinline__ PromptTile prompt_tile(const PromptArgs &a, int tile, int part) {
  const int lane = threadIdx.x & 63, G = a.d.num_q_heads / a.d.num_kv_heads;
  const int64_t cap = (int64_t)a.d.max_blocks_per_seq * a.d.page_size;
  PromptTile w;
  w.b = w.t = -1;
  w.n = w.P = w.row0 = 0;
  int before = 0;
  float work = 0.f;
  for (int b0 = 0; b0 < a.d.batch; b0 += 64) {
    const int b = b0 + lane;
    int n = 0, row0 = 0, P = 0;
    if (b < a.d.batch) {
      n = prompt_rows_of(a, b, row0);
      P = a.prefix_len ? a.prefix_len[b] : 0;
      P = P < 0 ? 0 : P > cap ? (int)cap : P;
    }
    const int tiles = (int)(((uint32_t)(n * G) + BM - 1) / BM);  // total_nodes * Hq is at most 2^30
    if (a.parts > 1) work += (float)tiles * ((float)P + 0.5f * (float)n);
    const int upto = scan_lanes(tiles) + before;
    if (w.b < 0) {
      const unsigned long long hit = __ballot(upto > tile);
      if (hit) {
        const int at = __builtin_ctzll(hit);  // everything from here on is the same in every lane, and known to be
        w.b = b0 + at;
        w.n = __builtin_amdgcn_readlane(n, at);
        w.P = __builtin_amdgcn_readlane(P, at);
        w.row0 = __builtin_amdgcn_readlane(row0, at);
        w.t = __builtin_amdgcn_readlane(upto, at) - 1 - tile;
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
    if (w.b >= 0 && a.parts <= 1) break;
  }
  if (w.b < 0) return w;
  const int last = (int)(((uint32_t)(w.t + 1) * BM + G - 1) / (uint32_t)G);  // tokens up to the tile's last row
  w.tokens_end = last < w.n ? last : w.n;
  const int keys = w.P + w.tokens_end;
  w.parts = 1;
  w.begin = 0;
  w.end = keys;
  if (a.parts > 1) {
    for (int m = 32; m; m >>= 1) work += __shfl_xor(work, m, 64);
    float each = work * (float)a.d.num_kv_heads / (float)a.units;
    each = fmaxf(each, (float)(4 * KEYS));
    const float n = ceilf((float)keys / each);
    w.parts = __builtin_amdgcn_readfirstlane(n < (float)a.parts ? (int)n : a.parts);
    if (w.parts > 1) {
      const int len = ((keys + w.parts - 1) / w.parts + KEYS - 1) / KEYS * KEYS;
      w.parts = (keys + len - 1) / len;
      w.begin = part * len;
      w.end = w.begin + len < keys ? w.begin + len : keys;
    }
  }
  if (part >= w.parts) w.t = -1;
  return w;
}

bool prompt_mfma_supports(const hb_attn_desc &d);
int32_t prompt_mfma_rows(const hb_attn_desc &d);  // of a tile
hipError_t launch_prompt_mfma(const PromptArgs &a, hipStream_t s);
// for tiles of `rows` rows whose parts begin at multiples of `keys`
hipError_t launch_prompt_join(const PromptArgs &a, int32_t rows, int32_t keys, hipStream_t s);
constexpr int kPromptAnyRows = 64;
hipError_t launch_prompt_any(const PromptArgs &a, hipStream_t s);

}  // namespace hb
