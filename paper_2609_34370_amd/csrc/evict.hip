// Eviction from the paged cache: of every (sequence, KV head) the keys of least accumulated weight go, the others move
// together in their order.
//
// evict_choose_kernel, a workgroup a (sequence, head): the weights come into registers once; the last one that stays is found
// by its bits, from the highest in which the weights differ on, eight a pass (counts of a digit in LDS: whole numbers, so
// their order does not matter); then one scan gives every key its new place, in a list of where the rows come from.
// evict_move_kernel: the list's rows.  A key's new place is never behind its old one, so a workgroup that owns a slice of the
// head dim moves it in place, in rounds: what a round overwrites, no later one reads.
//
// Bound by memory for a batch: 64 sequences of 1024 to 4096 keys cut to about a half (8 KV heads of 128) take 22 us to choose
// and 235 to 250 to move: the lines of K hold keys that go beside those that stay, and V is read whole, so 1.08 GB (counted)
// where the kept rows alone are 724 MB, 4.4 TB/s.  For one sequence by latency: 16001 keys cut to a quarter take 27 us to choose, eight workgroups
// on their way through the passes, and 25 to move.  One wave a slice, without rounds, took 227 and 79.
#include "common.h"
#include "tiles.h"

namespace spexis {

namespace {

constexpr int kChoose = 1024, kWaves = kChoose / kWave;   // threads that choose
constexpr int kMove = 256;   // and that move a slice

// A weight's bits in the order of the values: -0 counts as 0, a NaN as less than any number; never 0 or 0xFFFFFFFF.
__device__ __forceinline__ uint32_t rank_bits(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  return w != w ? 1u : (u >> 31 ? ~u : u | 0x80000000u);
}

}  // namespace

// kHeld: keys of a thread in registers; longer sequences read the others again.
template <int kHeld>
__global__ __launch_bounds__(kChoose) __attribute__((amdgpu_waves_per_eu(kHeld == 4 ? 8 : 4)))
void evict_choose_kernel(EvictParams p) {
  __shared__ uint32_t sm_set[kWaves], sm_clear[kWaves];
  __shared__ int sm_hist[256], sm_pick[3], sm_more[kHeld][kWaves], sm_equal[kHeld][kWaves], sm_first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = (int)blockIdx.x / p.hkv, h = (int)blockIdx.x % p.hkv, bs = p.block_size;
  const int S = clampi(p.seq_lens[b], 0, (int)min((int64_t)p.max_blocks * bs, (int64_t)p.max_seq_len));
  const EvictRange range = evict_range(S, p.keep_lens[b], p.first_keys ? p.first_keys[b] : 0, p.keep_last);
  const int m = range.m, lo = range.lo, hi = range.hi;
  const int32_t* table = p.block_tables + (int64_t)b * p.max_blocks;
  const int shift = bs == 16 ? 4 : 5;
  auto block_of = [&](int t) { return clampi(table[t >> shift], 0, p.num_blocks - 1); };
  auto place = [&](int t) { return ((int64_t)block_of(t) * p.hkv + h) * bs + (t & (bs - 1)); };
  int32_t* hdr = p.hdr + (int64_t)blockIdx.x * 2;
  int32_t* list = p.list + (int64_t)blockIdx.x * p.pitch;
  if (m == S) {   // (the weights may still have to go to another array)
    if (p.weights_out != p.weights)
      for (int t = tid; t < m; t += kChoose) p.weights_out[place(t)] = p.weights[place(t)];
    if (tid == 0) {
      hdr[0] = m;
      hdr[1] = m;
    }
    return;
  }
  // The keys' ranks: those that stay anyhow above all, none behind the end.
  auto rank = [&](int t, float w) { return t >= S ? 0u : (t < lo || t >= hi ? 0xFFFFFFFFu : rank_bits(w)); };
  float held[kHeld];
  uint32_t key[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int t = i * kChoose + tid;
    held[i] = t < S ? p.weights[place(t)] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i) key[i] = rank(i * kChoose + tid, held[i]);
  const int rounds = min((S + kChoose - 1) / kChoose, kHeld);
  // f(rank) of the keys that are chosen among
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < rounds && key[i] - 1 < 0xFFFFFFFEu) f(key[i]);
    for (int t = evict_rest(kHeld * kChoose, lo) + tid; t < hi; t += kChoose) f(rank_bits(p.weights[place(t)]));
  };
  // `least`, the rank of the last one that stays, from the highest bit in which the ranks differ on, up to eight bits a pass;
  // `equal`, how many of those of this rank stay: the first ones.
  uint32_t least = 0xFFFFFFFEu;
  int equal = 0, want = m - lo - (S - hi);
  if (want > 0) {
    uint32_t set = 0, clear = 0;   // the bits that some have, and that some have not
    each([&](uint32_t k) {
      set |= k;
      clear |= ~k;
    });
    set = (uint32_t)wave_or((int)set);
    clear = (uint32_t)wave_or((int)clear);
    if (lane == 0) {
      sm_set[wave] = set;
      sm_clear[wave] = clear;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      set |= sm_set[w];
      clear |= sm_clear[w];
    }
    int shift = (set & clear) != 0 ? 32 - __builtin_clz(set & clear) : 0;   // ranks agree from this bit up
    uint32_t prefix = (uint32_t)((uint64_t)set >> shift);
    while (true) {
      if (shift == 0) {
        least = prefix;
        equal = want;
        break;
      }
      const int bits = min(shift, 8), at = shift - bits;
      if (tid < 256) sm_hist[tid] = 0;
      __syncthreads();
      each([&](uint32_t k) {
        if ((uint32_t)((uint64_t)k >> shift) == prefix) atomicAdd(&sm_hist[k >> at & ((1u << bits) - 1)], 1);
      });
      __syncthreads();
      if (wave == 0) {   // lane l: digits 255 - 4 l and down
        int c[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine += c[i] = sm_hist[255 - 4 * lane - i];
        int before = wave_incl_scan_i32(mine, lane) - mine;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < want && want <= before + c[i]) {
            sm_pick[0] = 255 - 4 * lane - i;
            sm_pick[1] = want - before;
            sm_pick[2] = c[i];
          }
          before += c[i];
        }
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)sm_pick[0];
      want = sm_pick[1];
      shift = at;
      if (want == sm_pick[2]) {   // all that begin like this stay
        least = prefix << shift;
        equal = INT32_MAX;
        break;
      }
    }
  }
  if (tid == 0) sm_first = m;
  // The keys in order: the new place of one is the number of those before it that stay.
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const uint64_t more = __builtin_amdgcn_ballot_w64(key[i] > least), same = __builtin_amdgcn_ballot_w64(key[i] == least);
    if (lane == 0) {
      sm_more[i][wave] = (int)__popcll(more);
      sm_equal[i][wave] = (int)__popcll(same);
    }
  }
  __syncthreads();
  if (wave < 2) {   // exclusive sums in place, of the one and the other; the whole sums
    int* a = wave == 0 ? &sm_more[0][0] : &sm_equal[0][0];
    constexpr int kEach = kHeld * kWaves / kWave;
    int v[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      v[i] = sum;
      sum += a[lane * kEach + i];
    }
    const int upto = wave_incl_scan_i32(sum, lane);
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < kEach; ++i) a[lane * kEach + i] = upto - sum + v[i];
    if (lane == 63) sm_pick[wave] = upto;
  }
  __syncthreads();
  const uint64_t below = (1ull << lane) - 1;
  int moves = m;   // the first new place that is not the old one
  auto put = [&](int dst, int t, float w) {
    list[dst] = t;
    p.weights_out[place(dst)] = w;   // (all weights that lie up to there are read)
    if (dst != t) moves = min(moves, dst);
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    if (i >= rounds) break;
    const bool more = key[i] > least, same = key[i] == least;
    const int before = sm_equal[i][wave] + (int)__popcll(__builtin_amdgcn_ballot_w64(same) & below);
    const int dst = sm_more[i][wave] + (int)__popcll(__builtin_amdgcn_ballot_w64(more) & below) + min(before, equal);
    if (more || (same && before < equal)) put(dst, i * kChoose + tid, held[i]);
  }
  if (S > kHeld * kChoose) {   // the others, read again, 1024 at a time
    int kept = sm_pick[0], equals = sm_pick[1];   // held ones of either kind
    __syncthreads();
    for (int t0 = kHeld * kChoose; t0 < S; t0 += kChoose) {
      const int t = t0 + tid;
      const float w = t < S ? p.weights[place(t)] : 0.f;
      const uint32_t k = rank(t, w);
      const uint64_t mo = __builtin_amdgcn_ballot_w64(k > least), sa = __builtin_amdgcn_ballot_w64(k == least);
      if (lane == 0) {
        sm_more[0][wave] = (int)__popcll(mo);
        sm_equal[0][wave] = (int)__popcll(sa);
      }
      __syncthreads();   // (and every weight of these 1024 is read)
      int all_m = 0, all_e = 0, dst = kept + (int)__popcll(mo & below), e = equals + (int)__popcll(sa & below);
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        if (v < wave) {
          dst += sm_more[0][v];
          e += sm_equal[0][v];
        }
        all_m += sm_more[0][v];
        all_e += sm_equal[0][v];
      }
      if ((mo >> lane & 1) || ((sa >> lane & 1) && e < equal)) put(dst + min(e, equal), t, w);
      kept += all_m;
      equals += all_e;
      __syncthreads();
    }
  }
  atomicMin(&sm_first, moves);
  __syncthreads();
  if (tid == 0) {
    hdr[0] = m;
    hdr[1] = sm_first;
  }
}

// A workgroup moves a slice of a (sequence, head): 8 of the head dim of K (16 bytes a row), or 4 rows of the head dim
// of V.  Rows go in rounds, in order: all of a round are read, the workgroup meets, then they are written.  The next round's
// may be on their way meanwhile: they lie where this one does not write.
//   K: 16 bytes a lane from each row's old place to its new one, kBatch a thread and round.
//   V holds a row's elements apart, two bytes each; gathered from memory by twos they took 51 cycles for each 64.  So a wave,
//   for 128 new places, streams the old blocks that they come from through LDS, 128 slots a group, and picks the elements there:
//   lane l makes of head-dim row l / 16 the 16 bytes of 8 slots.
template <int D, int BS>
__global__ __launch_bounds__(kMove) void evict_move_kernel(EvictParams p) {
  constexpr int W = kMove / kWave;
  constexpr int kSlices = D / 8, kAll = 3 * kSlices;   // kSlices of K, twice as many of V
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int item = (int)(blockIdx.x / kAll), slice = (int)(blockIdx.x % kAll);
  const int b = item / p.hkv, h = item % p.hkv;
  const int m = p.hdr[2 * (int64_t)item], first = p.hdr[2 * (int64_t)item + 1];
  if (slice == 0 && h == 0 && threadIdx.x == 0) p.new_lens[b] = m;
  if (first >= m) return;
  const int32_t* table = p.block_tables + (int64_t)b * p.max_blocks;
  const int32_t* list = p.list + (int64_t)item * p.pitch;
  auto chunk_of = [&](int block) { return ((int64_t)clampi(block, 0, p.num_blocks - 1) * p.hkv + h) * (BS * D); };
  auto from_list = [&](int i) { return clampi(list[i], 0, p.max_blocks * BS - 1); };   // (leads no farther than the table)
  if (slice < kSlices) {
    constexpr int kBatch = 4, kRound = 64 * W * kBatch;
    uint16_t* k = reinterpret_cast<uint16_t*>(p.k_cache) + slice * BS * 8;
    int r0 = (first & ~63) + (int)threadIdx.x;
    int src[kBatch], to[kBatch];   // old places; the new ones' blocks
    u32x4 v[kBatch];
    auto look_up = [&](int r) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) src[i] = from_list(min(max(r + 64 * W * i, first), m - 1));
    };
    auto read = [&](u32x4* v) {
      int block[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) block[i] = table[src[i] / BS];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) v[i] = ld16(k + chunk_of(block[i]) + (src[i] % BS) * 8);
    };
    look_up(r0);
    read(v);
    for (int left = m - (first & ~63); left > 0; left -= kRound, r0 += kRound) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) to[i] = table[min(r0 + 64 * W * i, m - 1) / BS];
      look_up(r0 + kRound);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the round's rows are here
      __syncthreads();
      u32x4 next[kBatch];
      if (left > kRound) read(next);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int t = r0 + 64 * W * i;
        if (t >= first && t < m) st16(k + chunk_of(to[i]) + (t % BS) * 8, v[i]);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) v[i] = next[i];
    }
  } else {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    __shared__ u32x4 sm_group[W][kWave];
    u32x4* const sm = sm_group[wave];
    uint16_t* v = reinterpret_cast<uint16_t*>(p.v_cache) + (slice - kSlices) * 4 * BS;
    // a group's bytes, 16 a lane: its blocks, of each 4 rows of BS slots
    constexpr int kLanes = BS / 2;   // lanes a block
    const int row = lane / 16, unit = (lane % 16) / 2, hf = lane % 2;
    // the lane's 8 new places of a batch: position hf * 8 + e of a unit of 16 holds slot 8 (e / 4) + 4 hf + e % 4
    auto place = [&](int t0, int e) { return t0 + unit * 16 + 8 * (e >> 2) + 4 * hf + (e & 3); };
    // A batch's old places (the list's pitch holds whole batches), of its groups the first block and the last.
    i32x4 s0, s1;
    int from = 0, until = 0;
    auto look_up = [&](int t0) {
      s0 = *reinterpret_cast<const i32x4*>(list + place(t0, 0));
      s1 = *reinterpret_cast<const i32x4*>(list + place(t0, 4));
      from = from_list(max(t0, first)) / BS;
      until = from_list(min(t0 + 127, m - 1)) / BS;
    };
    // The blocks of a window of groups come with one load; a lane's is handed to it.
    constexpr int kPer = 128 / BS, kWindow = 64 / kPer, kAhead = 3;   // (kAhead: groups on their way)
    int block0 = 0, last = 0, window = 0, blocks = 0, blocks_next = 0;
    u32x4 now, ahead[kAhead];
    auto load = [&](int g) {   // for g in order
      if (g / kWindow > window) blocks = table[min(block0 + ++window * 64 + lane, last)];
      const int block = __builtin_amdgcn_ds_bpermute(4 * (g % kWindow * kPer + lane / kLanes), blocks);
      return ld16(v + chunk_of(block) + (lane % kLanes) * 8);
    };
    auto look_further = [&]() { blocks_next = table[min(from + lane, until)]; };
    int src[8];   // from the first block on; -1: not of the batch
    auto begin = [&](int t0) {
      block0 = __builtin_amdgcn_readfirstlane(from);
      last = __builtin_amdgcn_readfirstlane(until);
      window = 0;
      blocks = blocks_next;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = place(t0, e);
        src[e] = t >= first && t < m ? (e < 4 ? s0[e & 3] : s1[e & 3]) - block0 * BS : -1;
      }
      now = load(0);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ahead[i] = load(min(1 + i, (last - block0) / kPer));
    };
    constexpr int kRound = 128 * W;
    int t0 = (first & ~127) + 128 * wave;
    if (t0 < m) {
      look_up(t0);
      look_further();
      begin(t0);
    }
    if (t0 + kRound < m) look_up(t0 + kRound);
    for (int left = m - (first & ~127); left > 0; left -= kRound, t0 += kRound) {
      u32x4 w = {0, 0, 0, 0};
      const int t = place(t0, 0);   // the lane's first place; its last is 11 on
      const int to = table[min(t, m - 1) / BS];
      if (t0 + kRound < m) look_further();
      if (t0 < m) {
        const int groups = (last - block0) / kPer;
        uint32_t x[8];
        int at[8];   // where in a group, and which (what is in other groups is read too, and left)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int s = src[e] & 127;
          at[e] = s / BS * (4 * BS) + row * BS + ((s % BS & ~12) | ((s >> 2 & 1) << 3) | ((s >> 3 & 1) << 2));
          x[e] = 0;
        }
        for (int g = 0; g <= groups; ++g) {
          wave_lds_fence();
          sm[lane] = now;
          wave_lds_fence();
          now = ahead[0];
#pragma unroll
          for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
          if (g + kAhead < groups) ahead[kAhead - 1] = load(g + 1 + kAhead);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] |= reinterpret_cast<const uint16_t*>(sm)[at[e]] & (src[e] >> 7 == g ? 0xFFFFu : 0u);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = x[2 * c] | x[2 * c + 1] << 16;
      }
      if (t0 + kRound < m) begin(t0 + kRound);
      if (t0 + 2 * kRound < m) look_up(t0 + 2 * kRound);
      __syncthreads();   // the round's elements are picked
      uint16_t* const at = v + chunk_of(to) + row * BS + (t % BS & 16) + 8 * hf;
      if (t >= first && t + 11 < m) {
        st16(at, w);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int place_e = place(t0, e);
          if (place_e >= first && place_e < m) at[e] = (uint16_t)(w[e >> 1] >> 16 * (e & 1));
        }
      }
    }
  }
}

template <int D, int BS>
static hipError_t launch_move_t(const EvictParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.num_seqs * p.hkv * (3 * (D / 8))));
  hipLaunchKernelGGL((evict_move_kernel<D, BS>), grid, dim3(kMove), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  const dim3 items((unsigned)((int64_t)p.num_seqs * p.hkv));
  if (p.max_seq_len <= 4 * kChoose) hipLaunchKernelGGL((evict_choose_kernel<4>), items, dim3(kChoose), 0, s, p);
  else hipLaunchKernelGGL((evict_choose_kernel<16>), items, dim3(kChoose), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.head_dim == 128) return p.block_size == 16 ? launch_move_t<128, 16>(p, s) : launch_move_t<128, 32>(p, s);
  return p.block_size == 16 ? launch_move_t<64, 16>(p, s) : launch_move_t<64, 32>(p, s);
}

}  // namespace spexis
