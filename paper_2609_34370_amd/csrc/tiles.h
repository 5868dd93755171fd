// Parameters and launches of the attention of many query rows, of the attention weights and of evictions by them.
#pragma once

#include <math.h>

#include <algorithm>

#include "kernels.h"

namespace spexis {

constexpr float kLn2 = 0.693147180559945309f, kLog2E = 1.44269504088896341f;

// Attention of many query rows at once (whole prompts; batches that share prefixes): workgroups of kTileRows rows of a KV
// head that step through tile_keys(head_dim) keys at a time.
constexpr int kTileRows = 128;
__host__ __device__ constexpr int tile_keys(int head_dim) { return head_dim == 128 ? 32 : 64; }   // of a step
constexpr int kTileHdrInts = 8;
constexpr int kTileLeastKeys = 512;   // the fewest keys of a part
constexpr int kTileSlots = 768;   // workgroups that run at a time: three a CU
struct TileAttnParams {
  const void* k_cache;
  const void* v_cache;
  const float* scales;          // 8-bit cache: [num_blocks][hkv][2], K and V
  const int32_t* qsl;
  const int32_t* seq_lens;
  const int32_t* block_tables;
  const int32_t* group_start;   // [num_groups + 1] and [num_groups]; num_groups 0: nothing is shared
  const int32_t* prefix_lens;
  const void* q;
  void* out;
  float* lse;                   // or null
  int32_t* units_hdr;           // [units][kTileHdrInts]
  int32_t* groups_hdr;          // [num_groups][4]
  float* ws_prefix;             // [prefix_units][hkv][slot of kTileRows rows]
  float* ws_seq;                // [units][hkv][slot of pitch rows]
  int num_blocks, hkv, block_size, head_dim, num_seqs, num_groups, max_blocks, total_tokens, max_query_len;
  int hq, group;
  int pitch;                    // most rows of a sequence's tile
  int step;                     // tile_keys(head_dim)
  int shares;                   // row tiles (without a merge those of prefixes alone) are cut into parts, about so many a head; 0: not
  int units, prefix_units;      // the most units a head of either launch
  int merge;                    // prefixes and sequences in one launch, tile_merge_kernel joins partials
  int single;                   // (launcher) every segment has one tile at most: unit u is segment u
  int seg_lo, seg_hi;           // (launcher) its segments: the groups' prefixes are 0 .. num_groups - 1, then the sequences
  uint32_t q_sign;              // a negative scale turns q's signs over
  float scale_log2e, lazy;      // |scale| log2(e); kLazy in scores before the scale
};
// About how many parts `tiles` row tiles are cut into: with every tile rounded up, no more than `shares`.
__host__ __device__ inline int64_t tile_attn_parts(int shares, int tiles) {
  const int rest = shares - tiles, half = (shares + 1) / 2;
  return rest > half ? rest : half;
}
__host__ __device__ inline int64_t tile_slot_floats(int rows, int D) { return ((int64_t)rows * (D + 2) + 15) / 16 * 16; }
// Key tiles of a part, where all row tiles (`tiles`) have `sum` key tiles.  (64-bit divisions take hundreds of instructions; the
// sum is far below 2^53.)
__host__ __device__ inline int tile_attn_share(int shares, int step, int64_t sum, int tiles) {
  const double each = ceil((double)sum / (double)(int)tile_attn_parts(shares, tiles));
  return (int)fmin(fmax(each, (double)(kTileLeastKeys / step)), 2147483647.0);
}
// Parts of a row tile of nt key tiles.
__host__ __device__ inline int tile_parts(int nt, int share) { return nt > share ? (int)((uint32_t)(nt - 1) / (uint32_t)share) + 1 : 1; }

// Whether segments are taken in the order of their lengths: few ones with whole tiles, of a call without prefixes.  Prefixes come
// first, in their order: their partials lie in slots of their units' numbers, of which there are as many as prefixes can need.
constexpr int kByLength = 8;
__host__ __device__ inline bool tile_by_length(int num_groups, int shares, int segments) {
  return num_groups == 0 && shares == 0 && segments <= kByLength;
}
// The first unit of segment s of ns by falling length; sorted[][0], [1]: their key tiles and units; `before`: all units.
template <class Segments>
__host__ __device__ inline int tile_first_unit(const Segments& sorted, int ns, int s, int* before) {
  int at = 0;
  const int nt = sorted[s][0];
  for (int i = 0; i < ns; ++i) {
    const int other = sorted[i][0], units = sorted[i][1];
    at += other > nt || (other == nt && i < s) ? units : 0;
    *before += units;
  }
  return at;
}

// The most row tiles a head of sequences whose tokens come to total_tokens: each may end with a tile that is not full.
inline int64_t most_row_tiles(int64_t seqs, int64_t group, int64_t total_tokens, int64_t longest) {
  const int64_t all = (total_tokens * group + seqs * (kTileRows - 1)) / kTileRows;
  const int64_t each = (group * longest + kTileRows - 1) / kTileRows;
  return std::min(all, seqs * each);
}

struct TileLayout {
  int64_t units, prefix_units, groups_hdr, ws_prefix, ws_seq, total;   // offsets in bytes
  int shares, pitch;
  bool shared, merge;
};

// Units, and where their partials lie.  Prefixes count where sequences are longer than the least part (4 sequences of up to
// 265 keys behind 160 that they share: 11 us as they are, 17 with the prefix apart).  They run together with the sequences up
// to two workgroups a place that the chip has (kTileSlots), and all tiles are cut into parts then, else the prefixes' alone.
// Without prefixes tiles are cut where one a workgroup leaves half of the places free and there are keys enough for two parts.
inline TileLayout tile_layout(int64_t seqs, int64_t groups, int64_t hq, int64_t hkv, int64_t head_dim, int64_t total_tokens,
                              int64_t max_query_len, int64_t max_seq_len) {
  TileLayout l{};
  const int64_t group = hq / hkv;
  const bool is_long = max_seq_len > kTileLeastKeys;
  l.shared = groups > 0 && is_long;
  const int64_t pre = l.shared ? most_row_tiles(groups, group, total_tokens, total_tokens) : 0;
  const int64_t own = most_row_tiles(seqs, group, total_tokens, max_query_len);
  const int shares = (int)std::max<int64_t>(1, kTileSlots / hkv);
  l.merge = l.shared ? (pre + own) * hkv <= 2 * kTileSlots : is_long && own * hkv <= kTileSlots / 2;
  l.shares = l.shared || l.merge ? shares : 0;
  // (parts of prefixes are no more than their tiles and `shares`, whatever else is in the launch)
  l.prefix_units = l.shared ? pre + shares : 0;
  l.units = own + (l.merge ? pre + shares : 0);
  l.pitch = (int)std::min<int64_t>(kTileRows, group * max_query_len);
  int64_t off = 0;
  auto take = [&](int64_t bytes) {
    const int64_t at = off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  if (l.merge) take(l.units * kTileHdrInts * 4);
  l.groups_hdr = take(l.shared ? groups * 16 : 0);
  l.ws_prefix = take(l.prefix_units * hkv * tile_slot_floats(kTileRows, (int)head_dim) * 4);
  l.ws_seq = l.merge ? take(l.units * hkv * tile_slot_floats(l.pitch, (int)head_dim) * 4) : 0;
  l.total = std::max<int64_t>(off, 16);
  return l;
}

// Softmax weights of the cached keys, summed over the query rows of their KV head.
struct WeightParams {
  const void* k_cache;
  const int32_t* qsl;
  const int32_t* seq_lens;
  const int32_t* block_tables;
  const void* q;
  const float* lse;               // [T][hq]
  const int32_t* accepted;        // [num_seqs], or null: all of a sequence's tokens count
  const int32_t* first_keys;      // [num_seqs], or null: the keys in front of it are left as they are
  const float* weights_in;        // [num_blocks][hkv][block_size], or null: from 0
  float* weights;
  int num_blocks, hkv, block_size, head_dim, num_seqs, max_blocks, total_tokens, max_query_len, max_seq_len, hq, group;
  float scale_log2e;
};

// Eviction: which keys stay (one workgroup a sequence and head), then their rows' moves.
struct EvictParams {
  void* k_cache;
  void* v_cache;
  const float* weights;
  float* weights_out;
  const int32_t* seq_lens;
  const int32_t* block_tables;
  const int32_t* keep_lens;
  const int32_t* first_keys;      // or null
  int32_t* new_lens;
  int32_t* hdr;                   // [num_seqs][hkv][2]: keys that stay, the first that moves
  int32_t* list;                  // [num_seqs][hkv][pitch]: where each comes from
  int num_blocks, hkv, block_size, head_dim, num_seqs, max_blocks, max_seq_len, keep_last;
  int64_t pitch;                  // max_seq_len in whole batches of 128
};

// Of S keys: how many stay, and the keys [lo, hi) that are chosen among (those in front and behind stay anyhow).
struct EvictRange {
  int m, lo, hi;
};
__host__ __device__ inline EvictRange evict_range(int S, int keep, int first, int keep_last) {
  EvictRange r;
  r.m = keep < 0 ? 0 : (keep > S ? S : keep);
  r.lo = first < 0 ? 0 : (first > r.m ? r.m : first);
  r.hi = S - (keep_last < r.m - r.lo ? keep_last : r.m - r.lo);
  return r;
}
// The first key that is chosen among and not one of the `held` in registers.
__host__ __device__ inline int evict_rest(int held, int lo) { return held > lo ? held : lo; }

hipError_t launch_tile_attention(const TileAttnParams& p, hipStream_t s);
hipError_t launch_weights(const WeightParams& p, hipStream_t s);
hipError_t launch_evict(const EvictParams& p, hipStream_t s);

}  // namespace spexis
