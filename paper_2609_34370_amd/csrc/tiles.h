// Parameters and launches of the attention of many query rows, of the attention weights and of evictions by them.
#pragma once

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

hipError_t launch_tile_attention(const TileAttnParams& p, hipStream_t s);
hipError_t launch_weights(const WeightParams& p, hipStream_t s);
hipError_t launch_evict(const EvictParams& p, hipStream_t s);

}  // namespace spexis
