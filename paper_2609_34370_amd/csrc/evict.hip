// Eviction from the paged cache: of every (sequence, KV head) the keys of least accumulated weight go, the others move
// together in their order.
//
// evict_choose_kernel, a workgroup a (sequence, head): the weights come into registers once; the last one that stays is found
// by its bits, from the highest in which the weights differ on, eight a pass (counts of a digit in LDS: whole numbers, so
// their order does not matter); then one scan gives every key its new place, in a list of where the rows come from.
// evict_move_kernel: the list's rows.  A key's new place is never behind its old one, so a wave that owns a slice of the
// head dim moves it in place: what a step overwrites, no later one reads.
#include "common.h"
#include "tiles.h"

namespace spexis {

namespace {

constexpr int kChoose = 1024, kWaves = kChoose / kWave;

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
  __shared__ int sm_hist[256], sm_wave[kWaves], sm_pick[3], sm_more[kHeld][kWaves], sm_equal[kHeld][kWaves], sm_first;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = (int)blockIdx.x / p.hkv, h = (int)blockIdx.x % p.hkv, bs = p.block_size;
  const int S = clampi(p.seq_lens[b], 0, (int)min((int64_t)p.max_blocks * bs, (int64_t)p.max_seq_len));
  const int m = clampi(p.keep_lens[b], 0, S);
  const int f = p.first_keys ? clampi(p.first_keys[b], 0, m) : 0;
  const int last = min(p.keep_last, m - f);
  const int lo = f, hi = S - last;   // the keys that are chosen among
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
    for (int t = kHeld * kChoose + tid; t < hi; t += kChoose) f(rank_bits(p.weights[place(t)]));
  };
  // `least`, the rank of the last one that stays, from the highest bit in which the ranks differ on, up to eight bits a pass;
  // `equal`, how many of those of this rank stay: the first ones.
  uint32_t least = 0xFFFFFFFEu;
  int equal = 0, want = m - f - last;
  if (want > 0) {
    const uint32_t one = rank_bits(p.weights[place(lo)]);
    uint32_t differ = 0;
    each([&](uint32_t k) { differ |= k ^ one; });
    differ = (uint32_t)wave_or((int)differ);
    if (lane == 0) sm_wave[wave] = (int)differ;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) differ |= (uint32_t)sm_wave[w];
    int shift = 32 - __builtin_clz(differ | 1);   // ranks agree from this bit up
    if (differ == 0) shift = 0;
    uint32_t prefix = (uint32_t)((uint64_t)one >> shift);
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

// Wave s of a (sequence, head): slice s of K (8 of the head dim: 16 bytes a row), or of V (4 rows of the head dim).
//   K: 16 bytes a lane from each row's old place to its new one, kBatch times 64 rows read, then written.
//   V holds a row's elements apart, two bytes each; gathered from memory by twos they took 51 cycles for each 64.  So the wave
//   streams the old blocks whole through LDS, 128 slots a group, and picks the elements there: lane l makes of head-dim row
//   l / 16 and 128 new places the 16 bytes of 8 slots.
template <int D, int BS>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  constexpr int kSlices = D / 8;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int per = 3 * kSlices / 4;   // kSlices of K, twice as many of V
  const int item = (int)(blockIdx.x / per), slice = (int)(blockIdx.x % per) * 4 + wave;
  const int b = item / p.hkv, h = item % p.hkv;
  const int m = p.hdr[2 * (int64_t)item], first = p.hdr[2 * (int64_t)item + 1];
  if (slice == 0 && h == 0 && lane == 0) p.new_lens[b] = m;
  if (first >= m) return;
  const int32_t* table = p.block_tables + (int64_t)b * p.max_blocks;
  auto chunk = [&](int t) { return ((int64_t)clampi(table[t / BS], 0, p.num_blocks - 1) * p.hkv + h) * (BS * D); };
  if (slice < kSlices) {
    constexpr int kBatch = 4;
    const int32_t* list = p.list + (int64_t)item * p.pitch;
    uint16_t* k = reinterpret_cast<uint16_t*>(p.k_cache) + slice * BS * 8;
    auto from = [&](int t) { return list[min(max(t, first), m - 1)]; };
    int src[kBatch];
    int t0 = first & ~63;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) src[i] = from(t0 + 64 * i + lane);
    for (; t0 < m; t0 += 64 * kBatch) {
      u32x4 v[kBatch];
      int64_t at[kBatch], to[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) at[i] = chunk(src[i]) + (src[i] % BS) * 8;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) v[i] = ld16(k + at[i]);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        to[i] = chunk(min(t0 + 64 * i + lane, m - 1));
        src[i] = from(t0 + 64 * (kBatch + i) + lane);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int t = t0 + 64 * i + lane;
        if (t >= first && t < m) st16(k + to[i] + (t % BS) * 8, v[i]);
      }
    }
  } else {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    __shared__ u32x4 sm_group[4][kWave];
    u32x4* const sm = sm_group[wave];
    const int32_t* list = p.list + (int64_t)item * p.pitch;
    uint16_t* v = reinterpret_cast<uint16_t*>(p.v_cache) + (slice - kSlices) * 4 * BS;
    // a group's bytes, 16 a lane: its blocks, of each 4 rows of BS slots
    constexpr int kLanes = BS / 2;   // lanes a block
    const int row = lane / 16, unit = (lane % 16) / 2, hf = lane % 2;
    const int last = list[m - 1], last_group = last >> 7;
    // The blocks of a window of groups come with one load, a window ahead; a lane's is handed to it.  (No farther than the
    // last key that stays.)
    constexpr int kPer = 128 / BS, kWindow = 64 / kPer;
    auto look_up = [&](int w) { return table[min(w * 64 + lane, last / BS)]; };
    int window = (list[first] >> 7) / kWindow, blocks = look_up(window), blocks_next = look_up(window + 1);
    auto load = [&](int g) {   // for g in order
      g = min(g, last_group);
      if (g / kWindow > window) {
        ++window;
        blocks = blocks_next;
        blocks_next = look_up(window + 1);
      }
      const int block = __builtin_amdgcn_ds_bpermute(4 * (g % kWindow * kPer + lane / kLanes), blocks);
      return ld16(v + ((int64_t)clampi(block, 0, p.num_blocks - 1) * p.hkv + h) * (BS * D) + (lane % kLanes) * 8);
    };
    // the lane's 8 new places of a batch: position hf * 8 + e of a unit of 16 holds slot 8 (e / 4) + 4 hf + e % 4
    auto place = [&](int t0, int e) { return t0 + unit * 16 + 8 * (e >> 2) + 4 * hf + (e & 3); };
    int t0 = first & ~127, g = list[first] >> 7;
    i32x4 s0 = *reinterpret_cast<const i32x4*>(list + place(t0, 0)), s1 = *reinterpret_cast<const i32x4*>(list + place(t0, 4));
    constexpr int kAhead = 3;   // groups on their way
    u32x4 ahead[kAhead];
    const u32x4 now = load(g);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = load(g + 1 + i);
    sm[lane] = now;
    wave_lds_fence();
    for (; t0 < m; t0 += 128) {
      int src[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = place(t0, e);
        src[e] = t >= first && t < m ? (e < 4 ? s0[e & 3] : s1[e & 3]) : -1;
      }
      const int until = t0 + 128 <= m ? __builtin_amdgcn_readlane(src[7], 15) >> 7 : last_group;
      const int64_t to_chunk = chunk(min(place(t0, 0), m - 1));
      if (t0 + 128 < m) {   // the list's pitch holds whole batches
        s0 = *reinterpret_cast<const i32x4*>(list + place(t0 + 128, 0));
        s1 = *reinterpret_cast<const i32x4*>(list + place(t0 + 128, 4));
      }
      uint32_t x[8];
      int at[8];   // where in a group, and which (what is in other groups is read too, and left)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int s = src[e] & 127;
        at[e] = s / BS * (4 * BS) + row * BS + ((s % BS & ~12) | ((s >> 2 & 1) << 3) | ((s >> 3 & 1) << 2));
        x[e] = 0;
      }
      while (true) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[e] |= reinterpret_cast<const uint16_t*>(sm)[at[e]] & (src[e] >> 7 == g ? 0xFFFFu : 0u);
        if (g >= until) break;
        wave_lds_fence();
        sm[lane] = ahead[0];
        wave_lds_fence();
        ++g;
#pragma unroll
        for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
        ahead[kAhead - 1] = load(g + kAhead);
      }
      const int t = place(t0, 0);   // the chunk's first slot; its last is 11 on
      uint16_t* to = v + to_chunk + row * BS + (t % BS & 16) + 8 * hf;
      if (t >= first && t + 11 < m) {
        u32x4 w;
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = x[2 * c] | x[2 * c + 1] << 16;
        st16(to, w);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (src[e] >= 0) to[e] = (uint16_t)x[e];
      }
    }
  }
}

template <int D>
static hipError_t launch_move_t(const EvictParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.num_seqs * p.hkv * (3 * (D / 8) / 4)));
  if (p.block_size == 16) hipLaunchKernelGGL((evict_move_kernel<D, 16>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((evict_move_kernel<D, 32>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  const dim3 items((unsigned)((int64_t)p.num_seqs * p.hkv));
  if (p.max_seq_len <= 4 * kChoose) hipLaunchKernelGGL((evict_choose_kernel<4>), items, dim3(kChoose), 0, s, p);
  else hipLaunchKernelGGL((evict_choose_kernel<16>), items, dim3(kChoose), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return p.head_dim == 128 ? launch_move_t<128>(p, s) : launch_move_t<64>(p, s);
}

}  // namespace spexis
