// Attention of many query rows at once over the paged cache: whole prompts (any number of new tokens a sequence), and
// batches whose sequences begin with a prefix that they share.
//
// Work decomposition.  A segment is a run of query tokens against a run of keys: a sequence against the keys that are its
// own, causally; and, where a group of sequences shares a prefix, all tokens of the group against that prefix, once.  With
// G query heads a KV head, a segment has G rows a token, in tiles of 128: row r is (token r / G, head r % G), so every row of
// a tile reads the same K and V.  A unit, one workgroup, is a tile against the keys that any of its rows sees, or, where there
// are too few tiles to fill the chip, against one of several equal parts of them.  Prefixes and parts leave fp32 partials
// (reference maximum, sum, unnormalised output) in the workspace.  With few units prefixes and sequences run together, and
// tile_merge_kernel joins what they leave; with many the prefixes run in a launch in front, and a unit that has all of a
// sequence's own keys joins the prefix's partials to its registers (512 sequences of 9 tokens, 28 query heads over 4, in 16
// groups: 219 us for 246, which had written and read 134 MB more; 64 sequences of 5 behind one prefix of 4096 keys: together
// 68 us, 75 one after the other).
//
// Each of the four waves owns 32 rows.  The 32 keys of a step (64 of 64-wide heads) pass through LDS, where all waves read
// them: fetched into registers two steps ahead, widened there from the 8-bit cache, and stored in the order in which a wave
// reads matrix operands, 1 KB a fragment, so that no two lanes meet in a bank.  With v_mfma_f32_32x32x16_bf16 (operand A: lane l holds
// row l%32, k-slice 8*(l/32)..+7; B: column l%32, same k-slice; C: lane l, value i holds row 8*(i/4) + 4*(l/32) + i%4,
// column l%32):
//   S^T[key][row] = K Q^T: lane l owns query row l%32, so a row's maximum is one over 32 values and one lane exchange;
//   O^T[d][row] += V^T P^T: the V layouts hold slots in the order in which the score tile leaves them, so P^T is the
//   lane's own values.
//
// Bound by the SIMDs' instructions: 16001 tokens of 32 query heads over 8 of 128 (2.1 TFLOP) take 1.99 to 2.10 ms on several cards,
// 1.00 to 1.05 PFLOP/s; the matrix cores are busy for 51% of the cycles, and for 52% vector instructions are active (maxima,
// exponentials, sums, the weights' roundings, staging): three waves a SIMD hide little of the one behind the other.  LDS is
// not the limit: busy for 39% of the cycles, 0.1% of them conflicts; 12 waves read up to 600 bytes a ns from it, and products
// with a read for each reach 2.1 PFLOP/s.  Prompts of 100 to 3500 tokens, eight together, 359 to 397 us, 0.82 to 0.91
// PFLOP/s; a large matrix product reaches 1.58.  Tried on the way (at 16001 tokens): 64 keys a step and two workgroups a CU, the
// same but for shared prefixes (65 us for 60); eight waves that take turns at the matrix cores, 1.94 ms for 2.03, prompts
// together 391 us for 372; 64 rows a wave, 2.30 ms, one wave a SIMD with nothing to run beside it; half or all of K loaded by
// every wave for itself, 2.32 and 2.30 ms; products spread among the exponentials by hand, or waves' priorities, no difference.
#include "attention.h"
#include "tiles.h"

namespace spexis {

namespace {

constexpr int kRows = kTileRows;

// Eight e4m3 codes times a power of two, as a matrix operand.
__device__ __forceinline__ u32x4 widen_codes(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
               __builtin_bit_cast(uint32_t, d)};
}

// Keys that sequence b shares with its group (a multiple of the block size), and the group.
__device__ __forceinline__ int prefix_of(const TileAttnParams& p, int b, int* group) {
  *group = -1;
  if (p.num_groups == 0) return 0;
  int lo = 0, hi = p.num_groups;   // the last group that starts at or before b
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.group_start[mid] <= b) lo = mid;
    else hi = mid;
  }
  const int first = p.group_start[lo], behind = p.group_start[lo + 1], len = p.prefix_lens[lo];   // together
  if (first > b || behind <= b) return 0;
  *group = lo;
  return clampi(len, 0, p.max_blocks * p.block_size) & ~(p.block_size - 1);
}

// Segment s: the groups' prefixes, then the sequences.  Clamped so that every address derived from it stays in its buffer.
struct Segment {
  int q0, rows;      // first query token, query rows a KV head
  int seq;           // the row of the block tables
  int base, end;     // keys [base, end)
  int last;          // token j sees the keys up to last + j (a prefix: all of them)
  int group;         // of a sequence with a shared prefix: its group, else -1
};

__device__ __forceinline__ Segment segment(const TileAttnParams& p, int s) {
  Segment g;
  if (s < p.num_groups) {
    const int b0 = clampi(p.group_start[s], 0, p.num_seqs), b1 = clampi(p.group_start[s + 1], b0, p.num_seqs);
    g.q0 = clampi(p.qsl[b0], 0, p.total_tokens);
    const int n = clampi(p.qsl[b1], g.q0, p.total_tokens) - g.q0;
    g.seq = min(b0, p.num_seqs - 1);
    g.base = 0;
    g.end = clampi(p.prefix_lens[s], 0, p.max_blocks * p.block_size) & ~(p.block_size - 1);
    g.rows = g.end > 0 ? n * p.group : 0;
    g.last = INT32_MAX / 2;
    g.group = -1;
    return g;
  }
  const int b = s - p.num_groups;
  const int q0 = p.qsl[b], q1 = p.qsl[b + 1], len = p.seq_lens[b], shared = prefix_of(p, b, &g.group);
  g.q0 = clampi(q0, 0, p.total_tokens);
  const int n = min(clampi(q1, g.q0, p.total_tokens) - g.q0, p.max_query_len);
  g.rows = n * p.group;
  g.seq = b;
  g.end = clampi(len, max(n, 1), p.max_blocks * p.block_size);
  g.last = g.end - n;
  g.base = min(shared, g.last & ~(p.block_size - 1));
  if (g.base == 0) g.group = -1;
  return g;
}

__device__ __forceinline__ int row_tiles(const Segment& g) { return (g.rows + kRows - 1) / kRows; }
__device__ __forceinline__ int key_tiles(const TileAttnParams& p, const Segment& g) { return (g.end - g.base + p.step - 1) / p.step; }
// The keys of a segment's row tile end in front of this one.
__device__ __forceinline__ int tile_end(const TileAttnParams& p, const Segment& g, int tile) {
  const int r = min(g.rows, (tile + 1) * kRows) - 1;
  return min((int64_t)g.end, (int64_t)g.last + r / p.group + 1);
}

struct Unit {
  Segment g;
  int seg, tile, part, parts, first;   // part of `parts` equal ones of the tile's keys; `first`: the unit of part 0
};

// The unit u of a head, of the launch's segments [seg_lo, seg_hi) (false: there are fewer).  All threads of the workgroup call
// it, a segment each at a time; the one whose segment has the unit hands it on.  Where units are parts of tiles, a part is about
// `share` key tiles: sum(ceil(nt / share)) units.  A few sequences with whole tiles are taken in the order of their
// lengths, so that what ends last is short (prompts of 100 to 3500 tokens, 32 + 8 heads: four 115 us for 122 by number, six 197 and 205, eight
// 352 to 435 and 361 to 435; of equal lengths 182 and 180; tile by tile over all of them 2% less, but 2% more in 8 bits: neighbours no
// longer read the same keys).  Beyond that the search for the order costs what it gives or more (12 and 16 prompts within 1%, 64 of 300
// tokens 143 for 116; in parts 16 steps of 5 tokens 27.3 for 25.6; 32 steps behind a prefix of 4096 42.0 for 38.1, 60 behind 512, 32 + 16
// heads, 123 and 115).  Steps of short sequences need no search (512 sequences behind 16 prefixes 192 us for 204).
__device__ __forceinline__ bool find_unit(const TileAttnParams& p, int u, Unit& o) {
  __shared__ int64_t sm_total[4];
  __shared__ int sm_rows[4], sm_scan[2][4], sm_sort[kByLength][2];
  __shared__ __attribute__((aligned(16))) int sm_unit[12];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ns = p.seg_hi - p.seg_lo;
  if (p.single) {   // a tile a segment: no search
    if (u >= ns) return false;
    o.g = segment(p, p.seg_lo + u);
    o.seg = p.seg_lo + u;
    o.tile = o.part = 0;
    o.parts = 1;
    o.first = u;
    __syncthreads();
    return o.g.rows > 0;
  }
  Segment g{};
  int tiles = 0, nt = 0;
  auto load = [&](int base) {
    const int s = p.seg_lo + base + tid;
    tiles = nt = 0;
    if (s < p.seg_hi) {
      g = segment(p, s);
      tiles = row_tiles(g);
      nt = key_tiles(p, g);
    }
  };
  int share = INT32_MAX;
  if (p.shares > 0) {
    int64_t sum = 0;   // key tiles of all row tiles; row tiles
    int rows = 0;
    for (int base = 0; base < ns; base += 256) {
      load(base);
      sum += (int64_t)tiles * nt;
      rows += tiles;
    }
    sum = (int64_t)wave_sum_u64((uint64_t)sum);
    rows = wave_sum_i32(rows);
    if (lane == 0) {
      sm_total[wave] = sum;
      sm_rows[wave] = rows;
    }
    __syncthreads();
    sum = sm_total[0] + sm_total[1] + sm_total[2] + sm_total[3];
    rows = sm_rows[0] + sm_rows[1] + sm_rows[2] + sm_rows[3];
    share = tile_attn_share(p.shares, p.step, sum, rows);
  }
  int before = 0, turn = 0;
  for (int base = 0; base < ns; base += 256, turn ^= 1) {
    if (p.shares == 0 || ns > 256) load(base);
    const int parts = tile_parts(nt, share), mine = tiles * parts;
    int at;
    if (tile_by_length(p.num_groups, p.shares, ns)) {   // the longest first: what ends last is short
      if (tid < ns) {
        sm_sort[tid][0] = nt;
        sm_sort[tid][1] = mine;
      }
      __syncthreads();
      at = tile_first_unit(sm_sort, ns, min(tid, ns - 1), &before);
    } else {
      const int incl = wave_incl_scan_i32(mine, lane);
      if (lane == 63) sm_scan[turn][wave] = incl;
      __syncthreads();
      at = before + incl - mine;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int x = sm_scan[turn][w];
        if (w < wave) at += x;
        before += x;
      }
    }
    if (u >= at && u < at + mine) {
      const int t = (int)((uint32_t)(u - at) / (uint32_t)parts);
      *reinterpret_cast<u32x4*>(sm_unit) = u32x4{(uint32_t)g.q0, (uint32_t)g.rows, (uint32_t)g.seq, (uint32_t)g.base};
      *reinterpret_cast<u32x4*>(sm_unit + 4) = u32x4{(uint32_t)g.end, (uint32_t)g.last, (uint32_t)g.group, (uint32_t)(p.seg_lo + base + tid)};
      *reinterpret_cast<u32x4*>(sm_unit + 8) = u32x4{(uint32_t)t, (uint32_t)(u - at - t * parts), (uint32_t)parts, (uint32_t)(at + t * parts)};
    }
    if (before > u) break;   // (the same for all threads)
  }
  if (before <= u) return false;
  __syncthreads();
  auto get = [&](int i) { return __builtin_amdgcn_readfirstlane(sm_unit[i]); };
  o.g = {get(0), get(1), get(2), get(3), get(4), get(5), get(6)};
  o.seg = get(7);
  o.tile = get(8);
  o.part = get(9);
  o.parts = get(10);
  o.first = get(11);
  return true;
}

// Where the partials of the prefix of row r of a sequence (first query token q0) lie: slots first .. first + n - 1, row `row` of
// each.  Headers that no unit wrote (inconsistent inputs) lead no farther than the workspace.
struct PrefixParts {
  int first, n, row;
};
__device__ __forceinline__ PrefixParts prefix_parts(const TileAttnParams& p, int group, int q0, int r) {
  const u32x4 g = *reinterpret_cast<const u32x4*>(p.groups_hdr + (int64_t)group * 4);   // first token, tiles, parts, first unit
  const int row = (int)min((int64_t)max(q0 - (int)g[0], 0) * p.group + r, (int64_t)p.total_tokens * p.group), tile = row / kRows;
  PrefixParts o;
  // units count tiles from the last
  o.first = (int)min(max((int64_t)(int)g[3] + ((int64_t)(int)g[1] - 1 - tile) * (int)g[2], (int64_t)0), (int64_t)p.prefix_units);
  o.n = clampi((int)g[2], 0, p.prefix_units - o.first);
  o.row = row % kRows;
  return o;
}

}  // namespace

template <int D, int BS, bool IN8>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3)))
void tile_attn_kernel(TileAttnParams p) {
  constexpr int KS = D / 16;              // k-steps of the score product
  constexpr int MT = D / 32;              // 32-wide head-dim tiles of the output
  constexpr int KT = tile_keys(D) / 32, kKeys = 32 * KT;   // tiles of 32 keys a step
  constexpr int NL = (IN8 ? D / 64 : D / 32) * KT / 2;   // 16-byte loads of K, and of V, a thread and step
  constexpr int kFrags = KT * KS;         // fragments of 1 KB of K, and of V (= 2 * KT * MT)
  __shared__ u32x4 sm[2][2][kFrags][kWave];   // [buffer][K, V]
  __shared__ int sm_odd[D];
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the heads alternate over the XCDs: with 8 of them each XCD's L2 holds one head's keys
  const int h = (int)blockIdx.x % p.hkv, u = (int)blockIdx.x / p.hkv;

  if (tid < D) sm_odd[tid] = INT32_MAX;
  Unit un{};
  const bool some = find_unit(p, u, un);
  const Segment g = un.g;
  // the tiles of a sequence that see most keys first
  const int tile = some ? row_tiles(g) - 1 - un.tile : 0;
  const bool is_prefix = some && un.seg < p.num_groups;
  // joins the prefix's partials itself: they were written by the launch before
  const bool whole = some && !is_prefix && un.parts == 1 && (g.group < 0 || p.seg_lo > 0);
  if (h == 0 && tid == 0) {   // what those who join the partials need to know
    if (is_prefix && un.tile == 0 && un.part == 0)
      *reinterpret_cast<u32x4*>(p.groups_hdr + (int64_t)un.seg * 4) =
          u32x4{(uint32_t)g.q0, (uint32_t)row_tiles(g), (uint32_t)un.parts, (uint32_t)un.first};
    if (p.merge) {
      int32_t* hdr = p.units_hdr + (int64_t)u * kTileHdrInts;
      const bool joins = some && !is_prefix && un.part == 0 && !whole;
      *reinterpret_cast<u32x4*>(hdr) =
          u32x4{joins ? 1u : 0u, (uint32_t)g.q0, (uint32_t)(joins ? g.rows - tile * kRows : 0), (uint32_t)tile};
      *reinterpret_cast<u32x4*>(hdr + 4) = u32x4{(uint32_t)un.parts, (uint32_t)un.first, (uint32_t)g.group, 0u};
    }
  }
  if (!some || (is_prefix && u >= p.prefix_units)) return;   // (the latter: groups that overlap)

  const int row0 = tile * kRows;
  const int sure0 = min((int64_t)g.end - 1, (int64_t)g.last + row0 / p.group);   // every row sees the keys up to this one
  const int end = tile_end(p, g, tile);                      // keys [g.base, end)
  const int nt = (end - g.base + kKeys - 1) / kKeys;
  const int k0 = un.parts == 1 ? 0 : (int)((int64_t)nt * un.part / un.parts), k1 = un.parts == 1 ? nt : (int)((int64_t)nt * (un.part + 1) / un.parts);

  // ---- staging: this thread's part of a step's keys, global memory -> registers -> LDS
  const uint8_t* kc = reinterpret_cast<const uint8_t*>(p.k_cache);
  const uint8_t* vc = reinterpret_cast<const uint8_t*>(p.v_cache);
  constexpr int64_t kHead = (int64_t)BS * D * (IN8 ? 1 : 2);   // bytes of one (block, head) chunk
  sint32* table = (sint32*)p.block_tables + (int64_t)g.seq * p.max_blocks;
  const int last_block = (g.end - 1) / BS;
  // K: wave w stages keys 32 kw + col, the k-steps from ks0 on (8 bits: two a load); V: the 16 keys of unit vw, the head-dim
  // tiles from mt0 on (8 bits: two a load)
  const int kw = KT == 2 ? wave & 1 : 0, ks0 = KT == 2 ? (wave >> 1) * (KS / 2) : wave * (KS / 4);
  const int vw = KT == 2 ? wave : wave & 1, mt0 = KT == 2 ? 0 : (wave >> 1) * (MT / 2);
  const int k_slot = col % BS, v_slot = (vw * 16) % BS;
  u32x4 kr[NL], vr[NL];
  float k_scale = 0.f, v_scale = 0.f;
  // Where a step's keys lie is looked up a step before they are loaded, and the answer not touched until then: the lookup's
  // latency would stand in front of every step.
  int kb0 = 0, kb1 = 0, vb = 0;
  auto block_of = [&](int key) { return table[min((int)((uint32_t)(g.base + key) / BS), last_block)]; };
  auto chunk_of = [&](int block) { return (int64_t)clampi(block, 0, p.num_blocks - 1) * p.hkv + h; };
  auto find_k = [&](int t) {
    kb0 = block_of(t * kKeys + kw * 32);
    kb1 = BS == 16 ? block_of(t * kKeys + kw * 32 + 16) : kb0;
  };
  auto find_v = [&](int t) { vb = block_of(t * kKeys + vw * 16); };
  // (steps behind the last find its last block: a valid one)
  auto load_k = [&](int t) {
    const int64_t c0 = chunk_of(kb0), c1 = BS == 16 ? chunk_of(kb1) : c0, c = BS == 16 && col >= 16 ? c1 : c0;
    if (IN8) {
      const uint8_t* a = kc + c * kHead + (k_slot / 16) * 16 * D + ((ks0 + half) * 16 + k_slot % 16) * 16;
#pragma unroll
      for (int i = 0; i < NL; ++i) kr[i] = ld16(a + i * 2 * 256);
      k_scale = p.scales[2 * c];
    } else {
      const uint8_t* a = kc + c * kHead + ((2 * ks0 + half) * BS + k_slot) * 16;
#pragma unroll
      for (int i = 0; i < NL; ++i) kr[i] = ld16(a + i * 2 * BS * 16);
    }
    find_k(t + 1);
  };
  auto load_v = [&](int t) {
    const int64_t c = chunk_of(vb);
    if (IN8) {
      const uint8_t* a = vc + c * kHead + (v_slot / 16) * 16 * D + mt0 / 2 * 1024 + (col * 2 + half) * 16;
#pragma unroll
      for (int i = 0; i < NL; ++i) vr[i] = ld16(a + i * 1024);
      v_scale = p.scales[2 * c + 1];
    } else {
      const uint8_t* a = vc + c * kHead + ((mt0 * 32 + col) * BS + v_slot + 8 * half) * 2;
#pragma unroll
      for (int i = 0; i < NL; ++i) vr[i] = ld16(a + i * 32 * BS * 2);
    }
    find_v(t + 1);
  };
  auto store_k = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      if (IN8) {
        u32x4* f = &sm[buf][0][kw * KS + ks0 + 2 * i + half][col];
        f[0] = widen_codes(kr[i][0], kr[i][1], k_scale);
        f[32] = widen_codes(kr[i][2], kr[i][3], k_scale);
      } else {
        sm[buf][0][kw * KS + ks0 + i][lane] = kr[i];
      }
    }
  };
  // A V that is not finite, of a key that some of the tile's rows do not see: 0 times it would reach them.  It becomes 0, and
  // sm_odd[d] the first such key of its element, from which on rows get a NaN there at the end.
  auto part_odd = [&](u32x4& v, int d, int key0) {
    uint32_t bad[4], any = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) any |= bad[w] = ((v[w] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
    if (__builtin_amdgcn_ballot_w64(any != 0) == 0) return;
#pragma unroll
    for (int w = 3; w >= 0; --w) {
      const int key = key0 + 8 * (w >> 1) + 4 * half + 2 * (w & 1);
      if (bad[w] >> 31) atomicMin(&sm_odd[d], key + 1);
      if (bad[w] & 0x8000u) atomicMin(&sm_odd[d], key);
      v[w] &= ~((bad[w] >> 15) * 0xFFFFu);
    }
  };
  auto store_v = [&](int buf, int t) {
    // 32-bit word w of a fragment holds this lane's keys 8 (w / 2) + 4 half + 2 (w % 2) and the next of unit `wave`
    const int over = g.end - (g.base + t * kKeys + vw * 16);   // keys of the unit in front of the sequence's end
    const bool edge = t * kKeys + g.base + kKeys - 1 > sure0;   // some row does not see all of the step's keys
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      u32x4 v[IN8 ? 2 : 1];
      if (IN8) {
        v[0] = widen_codes(vr[i][0], vr[i][1], v_scale);
        v[IN8 ? 1 : 0] = widen_codes(vr[i][2], vr[i][3], v_scale);
      } else {
        v[0] = vr[i];
      }
#pragma unroll
      for (int x = 0; x < (IN8 ? 2 : 1); ++x) {
        const int mt = mt0 + (IN8 ? 2 * i + x : i);
        if (edge) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {   // what lies behind the end may be anything
            const int key = 8 * (w >> 1) + 4 * half + 2 * (w & 1);
            v[x][w] &= (key < over ? 0x0000FFFFu : 0u) | (key + 1 < over ? 0xFFFF0000u : 0u);
          }
          part_odd(v[x], 32 * mt + col, g.base + t * kKeys + vw * 16);
        }
        sm[buf][1][vw * MT + mt][lane] = v[x];
      }
    }
  };

  if (k0 < k1) {
    find_k(k0);
    find_v(k0);
    load_k(k0);
    load_v(k0);
  }

  // ---- this wave's rows
  const int rw = row0 + wave * 32;
  const bool active = rw < g.rows;
  auto row_at = [&](int r) {   // of q and the outputs
    const int j = r / p.group;
    return (int64_t)(g.q0 + j) * p.hq + h * p.group + r - j * p.group;
  };
  int lim;   // the last key that the lane's row sees
  u32x4 qf[KS];
  {
    const int r = min(rw + col, g.rows - 1);   // rows behind the last repeat it
    lim = min((int64_t)g.end - 1, (int64_t)g.last + r / p.group);
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + row_at(r) * D + 8 * half;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = ld16(q + 16 * s) ^ p.q_sign;
  }
  // every row of the wave sees the keys up to this one
  const int sure = min((int64_t)g.end - 1, (int64_t)g.last + min(rw, g.rows - 1) / p.group);
  float m = kNegBig, l = 0.f;   // in units of a score before its scale
  f32x16 acc[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[mt][e] = 0.f;

  if (k0 < k1) {
    store_k(0);
    store_v(0, k0);
    if (k0 + 1 < k1) {
      load_k(k0 + 1);
      load_v(k0 + 1);
    }
  }
  for (int t = k0; t < k1; ++t) {
    const int buf = (t - k0) & 1;
    __syncthreads();
    if (t + 1 < k1) {
      store_k(buf ^ 1);
      store_v(buf ^ 1, t + 1);
    }
    if (t + 2 < k1) {
      load_k(t + 2);
      load_v(t + 2);
    }
    const int t0 = g.base + t * kKeys;
    f32x16 sc[KT];
    if (active) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[kt][e] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
          sc[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(sm[buf][0][kt * KS + s][lane]), as_bf16x8(qf[s]), sc[kt], 0, 0, 0);
      }
    }
    if (active) {
      if (t0 + kKeys - 1 > sure) {
        const int seen = lim - t0 - 4 * half;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (kt * 32 + (e >> 2) * 8 + (e & 3) > seen) sc[kt][e] = -INFINITY;
      }
      float mx = sc[0][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = kt == 0 ? 1 : 0; e < 16; ++e) mx = fmaxf(mx, sc[kt][e]);
      mx = halves_max(mx);
      // Lazy rescaling: the reference maximum moves only when a score exceeds it by more than 2^kLazy, so 2^(x - m)
      // stays <= 2^kLazy and the accumulators are rescaled rarely.
      if (__builtin_amdgcn_ballot_w64(mx > m + p.lazy) != 0) {
        const float mnew = fmaxf(m, mx), alpha = fast_exp2((m - mnew) * p.scale_log2e);
        m = mnew;
        l *= alpha;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[mt][e] *= alpha;
      }
      // (finite where a row has seen no key yet, whatever the scale: its scores are minus infinity and weigh 0)
      const float mc = fminf(-m * p.scale_log2e, 3.0e38f);
      u32x4 pw[2 * KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] = fast_exp2(fmaf(sc[kt][e], p.scale_log2e, mc));
          l += x[e];
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          pw[2 * kt][w] = pack_bf16x2(x[2 * w], x[2 * w + 1]);
          pw[2 * kt + 1][w] = pack_bf16x2(x[8 + 2 * w], x[8 + 2 * w + 1]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // (products moved in front hold more registers than three waves a SIMD have)
#pragma unroll
      for (int s2 = 0; s2 < 2 * KT; ++s2)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(sm[buf][1][s2 * MT + mt][lane]), as_bf16x8(pw[s2]), acc[mt], 0, 0, 0);
    }
  }

  // ---- outputs, through LDS (each wave its own quarter), so that a store instruction writes whole lines
  __syncthreads();
  if (!active) return;
  if (g.base + k1 * kKeys - 1 > sure0) {
    int first = sm_odd[lane];
    if (D == 128) first = min(first, sm_odd[D - kWave + lane]);
    if (__builtin_amdgcn_ballot_w64(first < INT32_MAX) != 0) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (lim >= sm_odd[32 * mt + 8 * (e >> 2) + 4 * half + (e & 3)]) acc[mt][e] = __builtin_nanf("");
    }
  }
  float lt = halves_sum(l);
  float mb = m * p.scale_log2e;   // in the base-2 domain
  if (whole && g.group >= 0) {    // the prefix's partials of the lane's row
    const PrefixParts parts = prefix_parts(p, g.group, g.q0, min(rw + col, g.rows - 1));
    for (int c = 0; c < parts.n; ++c) {
      const float* slot = p.ws_prefix + ((int64_t)(parts.first + c) * p.hkv + h) * tile_slot_floats(kRows, D);
      const float mc = slot[kRows * D + parts.row], lc = slot[kRows * (D + 1) + parts.row];
      f32x4 o[MT][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int a = 0; a < 4; ++a) o[mt][a] = *reinterpret_cast<const f32x4*>(slot + parts.row * D + 32 * mt + 8 * a + 4 * half);
      const float mn = fmaxf(mb, mc), x = fast_exp2(mb - mn), y = fast_exp2(mc - mn);
      lt = lt * x + lc * y;
      mb = mn;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[mt][e] = acc[mt][e] * x + o[mt][e >> 2][e & 3] * y;
    }
  }
  u32x4* const scr = &sm[0][0][0][0] + wave * kFrags * kWave;
  const int left = g.rows - rw;   // rows of this wave
  if (whole) {
    constexpr int kOc = D / 8;   // 16-byte chunks of an output row; chunk c of row col at chunk c ^ (col mod kOc)
    const float inv = 1.0f / lt;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const u32x2 w = {pack_bf16x2(acc[mt][4 * a] * inv, acc[mt][4 * a + 1] * inv),
                         pack_bf16x2(acc[mt][4 * a + 2] * inv, acc[mt][4 * a + 3] * inv)};
        reinterpret_cast<u32x2*>(scr)[(col * kOc + ((4 * mt + a) ^ (col & (kOc - 1)))) * 2 + half] = w;
      }
    wave_lds_fence();
#pragma unroll 1
    for (int i = lane; i < 32 * kOc; i += kWave) {
      const int row = i / kOc, c = i % kOc, rr = rw + row;
      if (row < left)
        st16(reinterpret_cast<uint16_t*>(p.out) + row_at(rr) * D + 8 * c, scr[row * kOc + (c ^ (row & (kOc - 1)))]);
    }
    if (p.lse && half == 0 && col < left) p.lse[row_at(rw + col)] = (mb + __builtin_amdgcn_logf(lt)) * kLn2;
  } else {
    // the partial: [pitch][D], then maxima (in the base-2 domain) and sums
    const int pitch = is_prefix ? kRows : p.pitch;
    float* slot = is_prefix ? p.ws_prefix + ((int64_t)u * p.hkv + h) * tile_slot_floats(kRows, D)
                            : p.ws_seq + ((int64_t)u * p.hkv + h) * tile_slot_floats(p.pitch, D);
    // in two halves of the head dim; chunk c of row col's half at chunk c ^ (col mod kHc)
    constexpr int kHc = D / 8;   // 16-byte chunks of half an fp32 row
#pragma unroll
    for (int hm = 0; hm < 2; ++hm) {
#pragma unroll
      for (int mt = hm * MT / 2; mt < (hm + 1) * MT / 2; ++mt)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int c = 8 * (mt - hm * MT / 2) + 2 * a + half;
          scr[col * kHc + (c ^ (col & (kHc - 1)))] =
              u32x4{__float_as_uint(acc[mt][4 * a]), __float_as_uint(acc[mt][4 * a + 1]), __float_as_uint(acc[mt][4 * a + 2]),
                    __float_as_uint(acc[mt][4 * a + 3])};
        }
      wave_lds_fence();
#pragma unroll 1
      for (int i = lane; i < 32 * kHc; i += kWave) {
        const int row = i / kHc, c = i % kHc;
        if (row < left)
          st16(slot + (int64_t)(wave * 32 + row) * D + hm * (D / 2) + 4 * c, scr[row * kHc + (c ^ (row & (kHc - 1)))]);
      }
      wave_lds_fence();   // the second half's writes follow these reads
    }
    if (half == 0 && col < left) {
      slot[(int64_t)pitch * D + wave * 32 + col] = mb;
      slot[(int64_t)pitch * (D + 1) + wave * 32 + col] = lt;
    }
  }
}

// Joins the parts of a sequence's tiles: workgroup (unit, head, 16 rows) for the first unit of a tile in parts; the others
// follow it, and the parts of the shared prefix are found by the group.
//   o = sum_c acc_c 2^(m_c - M) / sum_c l_c 2^(m_c - M),   M = max_c m_c
template <int D>
__global__ __launch_bounds__(16 * D / 8) void tile_merge_kernel(TileAttnParams p) {
  const int h = (int)blockIdx.x % p.hkv, u = (int)blockIdx.x / p.hkv;
  const int32_t* hdr = p.units_hdr + (int64_t)u * kTileHdrInts;
  const u32x4 h0 = *reinterpret_cast<const u32x4*>(hdr), h1 = *reinterpret_cast<const u32x4*>(hdr + 4);
  const int left = (int)h0[2], lr = (int)blockIdx.y * 16 + threadIdx.x / (D / 8), d = (threadIdx.x % (D / 8)) * 8;
  if (h0[0] != 1u || lr >= min(left, kRows)) return;
  const int q0 = (int)h0[1], r = (int)h0[3] * kRows + lr, parts = (int)h1[0], first = (int)h1[1], group = (int)h1[2];
  const int j = r / p.group;
  float M = kNegBig, den = 0.f;
  f32x4 o0 = {0.f, 0.f, 0.f, 0.f}, o1 = o0;
  auto add = [&](const float* slot, int pitch, int row) {
    const float mc = slot[(int64_t)pitch * D + row], lc = slot[(int64_t)pitch * (D + 1) + row];
    const f32x4 a0 = *reinterpret_cast<const f32x4*>(slot + (int64_t)row * D + d);
    const f32x4 a1 = *reinterpret_cast<const f32x4*>(slot + (int64_t)row * D + d + 4);
    const float mn = fmaxf(M, mc), x = fast_exp2(M - mn), e = fast_exp2(mc - mn);
    den = den * x + lc * e;
    o0 = o0 * x + a0 * e;
    o1 = o1 * x + a1 * e;
    M = mn;
  };
  for (int c = 0; c < parts && first + c < p.units; ++c)
    add(p.ws_seq + ((int64_t)(first + c) * p.hkv + h) * tile_slot_floats(p.pitch, D), p.pitch, lr);
  if (group >= 0) {
    const PrefixParts parts = prefix_parts(p, group, q0, r);
    for (int c = 0; c < parts.n; ++c)
      add(p.ws_prefix + ((int64_t)(parts.first + c) * p.hkv + h) * tile_slot_floats(kRows, D), kRows, parts.row);
  }
  const float inv = 1.0f / den;
  const int64_t row = (int64_t)(q0 + j) * p.hq + h * p.group + r % p.group;
  st16(reinterpret_cast<uint16_t*>(p.out) + row * D + d,
       u32x4{pack_bf16x2(o0[0] * inv, o0[1] * inv), pack_bf16x2(o0[2] * inv, o0[3] * inv), pack_bf16x2(o1[0] * inv, o1[1] * inv),
             pack_bf16x2(o1[2] * inv, o1[3] * inv)});
  if (p.lse && d == 0) p.lse[row] = (M + __builtin_amdgcn_logf(den)) * kLn2;
}

template <int D, int BS>
static hipError_t launch_units_t(const TileAttnParams& p, int units, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)units * p.hkv));
  if (p.scales) hipLaunchKernelGGL((tile_attn_kernel<D, BS, true>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((tile_attn_kernel<D, BS, false>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

template <int D, int BS>
static hipError_t launch_tiles_t(TileAttnParams p, hipStream_t s) {
  hipError_t e;
  if (p.num_groups > 0 && !p.merge) {   // the prefixes in front
    p.seg_hi = p.num_groups;
    e = launch_units_t<D, BS>(p, p.prefix_units, s);
    if (e != hipSuccess) return e;
    p.seg_lo = p.num_groups;
    p.shares = 0;
  }
  p.single = p.shares == 0 && (int64_t)p.group * p.max_query_len <= kRows && (int64_t)p.num_seqs * p.hkv < (1 << 24);
  p.seg_hi = p.num_groups + p.num_seqs;
  e = launch_units_t<D, BS>(p, p.single ? p.num_seqs : p.units, s);
  if (e != hipSuccess || !p.merge) return e;
  hipLaunchKernelGGL((tile_merge_kernel<D>), dim3((unsigned)((int64_t)p.units * p.hkv), (unsigned)((p.pitch + 15) / 16)),
                     dim3(16 * D / 8), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_tile_attention(const TileAttnParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.block_size == 16 ? launch_tiles_t<128, 16>(p, s) : launch_tiles_t<128, 32>(p, s);
  return p.block_size == 16 ? launch_tiles_t<64, 16>(p, s) : launch_tiles_t<64, 32>(p, s);
}

}  // namespace spexis
