// Eviction from the paged cache: of every (sequence, KV head) the keys of least accumulated weight go, the others move
// together in their order.
//
// evict_choose_kernel, a workgroup a (sequence, head): the weight of the last key that stays, by its bits from the top, eight
// a pass over the weights (counts of a digit in LDS: whole numbers, so their order does not matter); then the keys in order,
// each with its new place, into a list.  evict_move_kernel: the list's rows.  A key's new place is never behind its old one,
// so a wave that owns a slice of the head dim moves it in place, 64 rows a step: what a step overwrites, no later one reads.
#include "common.h"
#include "kernels.h"

namespace spexis {

namespace {

constexpr int kChoose = 1024;

// Bits in the order of the values: -0 counts as 0, a NaN as less than any number.
__device__ __forceinline__ uint32_t rank_bits(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  return w != w ? 0u : (u >> 31 ? ~u : u | 0x80000000u);
}

}  // namespace

__global__ __launch_bounds__(kChoose) void evict_choose_kernel(EvictParams p) {
  __shared__ int sm_hist[256], sm_keep[kChoose / 64], sm_equal[kChoose / 64], sm_pick[2], sm_first;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = (int)blockIdx.x / p.hkv, h = (int)blockIdx.x % p.hkv, bs = p.block_size;
  const int S = clampi(p.seq_lens[b], 0, (int)min((int64_t)p.max_blocks * bs, (int64_t)p.max_seq_len));
  const int m = clampi(p.keep_lens[b], 0, S);
  const int f = p.first_keys ? clampi(p.first_keys[b], 0, m) : 0;
  const int last = min(p.keep_last, m - f);
  const int lo = f, hi = S - last;   // the keys that are chosen among
  const int32_t* table = p.block_tables + (int64_t)b * p.max_blocks;
  auto place = [&](int t) {
    return ((int64_t)clampi(table[t / bs], 0, p.num_blocks - 1) * p.hkv + h) * bs + t % bs;
  };
  int32_t* hdr = p.hdr + (int64_t)blockIdx.x * 2;
  int32_t* list = p.list + (int64_t)blockIdx.x * p.max_seq_len;
  if (m == S) {   // (the weights may still have to go to another array)
    if (p.weights_out != p.weights)
      for (int t = tid; t < m; t += kChoose) p.weights_out[place(t)] = p.weights[place(t)];
    if (tid == 0) {
      hdr[0] = m;
      hdr[1] = m;
    }
    return;
  }
  // the `want`-th largest of the middle: its bits digit by digit, and how many of those equal to it stay
  uint32_t prefix = 0;
  int want = m - f - last;
  if (tid == 0) sm_first = m;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) sm_hist[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kChoose) {
        const uint32_t u = rank_bits(p.weights[place(t)]);
        if (shift == 24 || (u >> (shift + 8)) == prefix) atomicAdd(&sm_hist[u >> shift & 255], 1);
      }
      __syncthreads();
      if (wave == 0) {
        // lane l: digits 255 - 4l and down
        int c[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine += c[i] = sm_hist[255 - 4 * lane - i];
        int at = wave_incl_scan_i32(mine, lane) - mine;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (at < want && want <= at + c[i]) {
            sm_pick[0] = 255 - 4 * lane - i;
            sm_pick[1] = want - at;
          }
          at += c[i];
        }
      }
      __syncthreads();
      prefix = prefix << 8 | (uint32_t)sm_pick[0];
      want = sm_pick[1];
    }
  }
  const bool any = m - f - last > 0;
  // the keys in order
  int kept = 0, equals = 0;
  for (int t0 = 0; t0 < S; t0 += kChoose) {
    const int t = t0 + tid;
    const bool in = t < S, always = in && (t < lo || t >= hi);
    float w = 0.f;
    int64_t at = 0;
    if (in) {
      at = place(t);
      w = p.weights[at];
    }
    const uint32_t u = rank_bits(w);
    const bool equal = in && !always && any && u == prefix;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(equal);
    if (lane == 0) sm_equal[wave] = (int)__popcll(eq);
    __syncthreads();
    int e = equals + (int)__popcll(eq & ((1ull << lane) - 1)), all_e = 0, all_k = 0;
#pragma unroll
    for (int i = 0; i < kChoose / 64; ++i) {
      if (i < wave) e += sm_equal[i];
      all_e += sm_equal[i];
    }
    const bool stays = always || (in && any && u > prefix) || (equal && e < want);
    const uint64_t ks = __builtin_amdgcn_ballot_w64(stays);
    if (lane == 0) sm_keep[wave] = (int)__popcll(ks);
    __syncthreads();
    int dst = kept + (int)__popcll(ks & ((1ull << lane) - 1));
#pragma unroll
    for (int i = 0; i < kChoose / 64; ++i) {
      if (i < wave) dst += sm_keep[i];
      all_k += sm_keep[i];
    }
    if (stays) {
      list[dst] = t;
      p.weights_out[place(dst)] = w;   // every weight of these steps is read
      if (dst != t) atomicMin(&sm_first, dst);
    }
    kept += all_k;
    equals += all_e;
  }
  __syncthreads();
  if (tid == 0) {
    hdr[0] = m;
    hdr[1] = sm_first;
  }
}

// Wave s of a (sequence, head): slice s of K (8 of the head dim: 16 bytes a row), or of V (8 rows of the head dim, of which
// a lane takes one and 8 slots).
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictParams p) {
  constexpr int kSlices = D / 8;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int per = 2 * kSlices / 4;
  const int item = (int)(blockIdx.x / per), slice = (int)(blockIdx.x % per) * 4 + wave, bs = p.block_size;
  const int b = item / p.hkv, h = item % p.hkv;
  const int m = p.hdr[2 * (int64_t)item], first = p.hdr[2 * (int64_t)item + 1];
  if (slice == 0 && h == 0 && lane == 0) p.new_lens[b] = m;
  if (first >= m) return;
  const int32_t* list = p.list + (int64_t)item * p.max_seq_len;
  const int32_t* table = p.block_tables + (int64_t)b * p.max_blocks;
  auto chunk = [&](int t) { return ((int64_t)clampi(table[t / bs], 0, p.num_blocks - 1) * p.hkv + h) * bs * D; };
  if (slice < kSlices) {
    uint16_t* k = reinterpret_cast<uint16_t*>(p.k_cache) + slice * bs * 8;
    for (int t0 = first & ~63; t0 < m; t0 += 64) {
      const int t = t0 + lane, src = list[min(max(t, first), m - 1)];
      const u32x4 v = ld16(k + chunk(src) + (src % bs) * 8);
      if (t >= first && t < m) st16(k + chunk(t) + (t % bs) * 8, v);
    }
  } else {
    // lane: head-dim row lane / 8, and of the 64 rows' 8 chunks of 8 slots chunk lane % 8
    uint16_t* v = reinterpret_cast<uint16_t*>(p.v_cache) + ((slice - kSlices) * 8 + lane / 8) * bs;
    const int unit = (lane % 8) / 2, hf = lane % 2;
    for (int t0 = first & ~63; t0 < m; t0 += 64) {
      uint16_t x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {   // position hf * 8 + e holds slot 8 (e / 4) + 4 hf + e % 4 of its 16
        const int t = t0 + unit * 16 + 8 * (e >> 2) + 4 * hf + (e & 3), src = list[min(max(t, first), m - 1)], s = src % bs;
        x[e] = v[chunk(src) + ((s & ~12) | ((s >> 2 & 1) << 3) | ((s >> 3 & 1) << 2))];
      }
      const int t = t0 + unit * 16 + 4 * hf;   // the chunk's first slot; its last is 11 on
      if (t >= m) continue;
      uint16_t* to = v + chunk(t) + (t % bs & 16) + 8 * hf;
      if (t >= first && t + 11 < m) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = x[2 * i] | (uint32_t)x[2 * i + 1] << 16;
        st16(to, w);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int at = t + 8 * (e >> 2) + (e & 3);
          if (at >= first && at < m) to[e] = x[e];
        }
      }
    }
  }
}

hipError_t launch_evict(const EvictParams& p, hipStream_t s) {
  const int64_t items = (int64_t)p.num_seqs * p.hkv;
  hipLaunchKernelGGL(evict_choose_kernel, dim3((unsigned)items), dim3(kChoose), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(items * (2 * (p.head_dim / 8) / 4)));
  if (p.head_dim == 128) hipLaunchKernelGGL((evict_move_kernel<128>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((evict_move_kernel<64>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace spexis
