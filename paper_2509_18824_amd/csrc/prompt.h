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
  // [tile]: first row of the sequence in the batch, rows (token, head) in front of the tile's, its rows, parts of its keys.  Where
  // a tile's keys may be cut, the workgroups of part 0 write it, for the join.
  struct Head {
    int32_t row0, first, rows, parts;
  } *heads;
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

// What the lanes know about sequences b0 .. b0 + 63
struct PromptLane {
  int n, P, row0, tiles;
};
template <int BM>
__device__ __forceinline__ PromptLane prompt_lane(const PromptArgs &a, int b) {
  const int G = a.d.num_q_heads / a.d.num_kv_heads, cap = a.d.max_blocks_per_seq * a.d.page_size;
  PromptLane s = {0, 0, 0, 0};
  if (b < a.d.batch) {
    s.n = prompt_rows_of(a, b, s.row0);
    s.P = a.prefix_len ? a.prefix_len[b] : 0;
    s.P = s.P < 0 ? 0 : s.P > cap ? cap : s.P;
    s.tiles = (int)(((uint32_t)(s.n * G) + BM - 1) / BM);  // total_nodes * Hq is at most 2^30
  }
  return s;
}

// Length of a part of a tile's keys.  Lane c looks at the length that makes (c + 1) / 8 of `units` parts of all the work, and
// says when such a plan is done, in keys: whole rounds of the longest part where all are alike, or the work of a unit and a
// shortest part where they are not (the shortest begin last); and what parts cost beside their keys.
template <int BM, int KEYS>
__device__ __forceinline__ float prompt_part(const PromptArgs &a, float work) {
  // Of a part (its start, its results written), of the join, and of every part to it.  Workgroups go round the dies and
  // their shader engines in turn, so that a round is full at nine tenths.  One prompt of 1024, 2048, 4096 rows whole 36, 64, 137 us,
  // cut 52, 71, 186; 512 rows over 32 K in 1, 2, 3, 4 parts 814, 440, 309, 263, in 5 (252 of 256 CUs, nominally) 393, in 9 350;
  // 64 rows over 8 K in 4, 8, 12, 16 parts 79, 58, 56, 59.
  constexpr float kCost = 512.f, kJoin = 768.f, kEach = 64.f, kFull = 0.9f;
  const int lane = threadIdx.x & 63;
  const float units = (float)a.units, heads = (float)a.d.num_kv_heads;
  const float each = fmaxf(work * heads * 8.f / (units * (float)(lane + 1)), 2.f * KEYS);
  float parts = 0.f, longest = 0.f, shortest = 3e38f;
  float deepest = 1.f;
  for (int b0 = 0; b0 < a.d.batch; b0 += 64) {
    const PromptLane s = prompt_lane<BM>(a, b0 + lane);
    for (unsigned long long left = __ballot(s.tiles > 0); left; left &= left - 1) {
      const int at = __builtin_ctzll(left);
      const float tiles = (float)__builtin_amdgcn_readlane(s.tiles, at), P = (float)__builtin_amdgcn_readlane(s.P, at),
                  n = (float)__builtin_amdgcn_readlane(s.n, at);
      const float most = (float)a.parts, cuts = fminf(ceilf((P + n) / each), most);
      parts += 0.5f * tiles * (cuts + fminf(fmaxf(ceilf((P + 0.5f * n) / each), 1.f), most));
      longest = fmaxf(longest, cuts > 1.f ? fmaxf(each, (P + n) / most) : P + n);
      shortest = fminf(shortest, (P + n / tiles) / cuts);
      deepest = fmaxf(deepest, cuts);
    }
  }
  const float rounds = ceilf(parts * heads / (kFull * units)) * longest, mixed = work * heads / units + shortest;
  const float cost = fmaxf(longest, fminf(rounds, mixed)) + kCost * fmaxf(parts * heads / units, 1.f) + (deepest > 1.f ? kJoin + kEach * deepest : 0.f);
  float best = cost;
  for (int m = 32; m; m >>= 1) best = fminf(best, __shfl_xor(best, m, 64));
  const unsigned long long win = __ballot(cost == best);
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(each), win ? __builtin_ctzll(win) : 0));
}

// Every lane of the wavefront calls it with the same arguments.  Tiles of a sequence are numbered from its last (which sees
// the most keys) to its first, so that the longest work begins first.
template <int BM, int KEYS>
__device__ __forceinline__ PromptTile prompt_tile(const PromptArgs &a, int tile, int part) {
  const int lane = threadIdx.x & 63, G = a.d.num_q_heads / a.d.num_kv_heads;
  PromptTile w;
  w.b = w.t = -1;
  w.n = w.P = w.row0 = 0;
  int before = 0;
  float work = 0.f;
  for (int b0 = 0; b0 < a.d.batch; b0 += 64) {
    const PromptLane s = prompt_lane<BM>(a, b0 + lane);
    if (a.parts > 1) work += (float)s.tiles * ((float)s.P + 0.5f * (float)s.n);
    const int upto = scan_lanes(s.tiles) + before;
    if (w.b < 0) {
      const unsigned long long hit = __ballot(upto > tile);
      if (hit) {
        const int at = __builtin_ctzll(hit);  // everything from here on is the same in every lane, and known to be
        w.b = b0 + at;
        w.n = __builtin_amdgcn_readlane(s.n, at);
        w.P = __builtin_amdgcn_readlane(s.P, at);
        w.row0 = __builtin_amdgcn_readlane(s.row0, at);
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
    const float n = ceilf((float)keys / prompt_part<BM, KEYS>(a, work));
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

// by every workgroup, before it leaves
template <int BM>
__device__ __forceinline__ void prompt_head(const PromptArgs &a, const PromptTile &w, int tile, int h, int part) {
  if (a.parts > 1 && h == 0 && part == 0 && threadIdx.x == 0) {
    const int G = a.d.num_q_heads / a.d.num_kv_heads, first = w.t * BM;
    a.heads[tile] = w.b < 0 ? PromptArgs::Head{0, 0, 0, 1} : PromptArgs::Head{w.row0, first, min(BM, w.n * G - first), w.parts};
  }
}

bool prompt_mfma_supports(const hb_attn_desc &d);
int32_t prompt_mfma_rows(const hb_attn_desc &d);  // of a tile
hipError_t launch_prompt_mfma(const PromptArgs &a, hipStream_t s);
hipError_t launch_prompt_join(const PromptArgs &a, int32_t rows, hipStream_t s);  // for tiles of `rows` rows
constexpr int kPromptAnyRows = 16;
hipError_t launch_prompt_any(const PromptArgs &a, hipStream_t s);

}  // namespace hb
