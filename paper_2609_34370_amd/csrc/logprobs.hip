// Log probabilities of given tokens under softmax(logits / T), with the entropy and the top alternatives of
// their rows.
//   w_v = (x_v - max x) c, c = log2(e) / T;  Z = sum 2^w;  U = sum 2^w w
//   log p(v) = (x_v - max x) / T - ln Z;   H = ln Z - ln2 U / Z
//   (both terms of H are at least 0, as is ln Z: no cancellation)
// Bound by reading the logits once: 4608 rows of 152064 fp32 with 5 alternatives 413 us, 6.8 TB/s, what a large read
// reaches.  221 rows of 128256 (64 sequences' emitted tokens) with 20 alternatives 34 us, 3.3 TB/s: four rounds of loads a
// workgroup, of which the first has to find a threshold and to sort (with none 24 us), and 4.8 us of merge.  bf16 rows are
// bound by instructions, as many a logit on half the bytes: 266 us, 5.3 TB/s, and 31 us.
//
// Work split.  A workgroup takes one part of one item's row, its four waves every fourth chunk of 2048 logits (in
// registers, the next one in flight).  Every lane keeps a running maximum, Z and U of its own: no exchange
// until the end.  With one part per row the workgroup writes the outputs; with more, a second launch combines them.
//
// Top alternatives, by (logit, lower index first): a wave's candidates wait in LDS as 64-bit keys, the logit's order in
// the upper half and the index's complement in the lower, so that no two are equal and every order of work gives the
// same list.  A logit becomes a candidate when it reaches the threshold; when more than 64 wait they are
// sorted (one key a lane) and cut to n, and the threshold rises just above the n-th.  A wave meets its indices in
// ascending order, chunk by chunk and group by group, so a later logit that equals the n-th loses to it.  Before
// that the threshold is the n-th largest of the workgroup's 256 lanes' maxima so far (at least n logits reach it,
// few more do), found again after 1, 4, 16 ... chunks while
// at least as many are to come (a search costs about one chunk's work).
// 600 rows of 128256 with 20 alternatives take 59 us; masked but for four logits, or of one value, 64 to 66; ascending,
// where every logit is a candidate, 761.
#include "common.h"
#include "kernels.h"

namespace spexis {

constexpr int kLpElems = 32;                    // logits of a chunk per lane
constexpr int kLpGroup = 8;                     // of them between two looks at the candidates' count
constexpr int kLpKeep = 64;                     // candidates that wait without being sorted
constexpr int kLpCap = kLpKeep + kLpGroup * kWave;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2 = 0.693147180559945309f;

__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);   // -0 counts as 0
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// The value of lane l ^ J, in lane moves that need no LDS.
template <int J>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int lane) {
  if constexpr (J == 1) return dpp_u32<kDppQuadXor1, 0xF>(v, v);
  if constexpr (J == 2) return dpp_u32<kDppQuadXor2, 0xF>(v, v);
  if constexpr (J == 4) {   // l ^ 7 in each half of a row, then l ^ 3 in each quad
    const uint32_t m = dpp_u32<0x141, 0xF>(v, v);
    return dpp_u32<0x1B, 0xF>(m, m);
  }
  if constexpr (J == 8) return dpp_u32<0x128, 0xF>(v, v);   // a row of 16 rotated by 8
  if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane & 16 ? r[0] : r[1];
  }
  if constexpr (J == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane & 32 ? r[0] : r[1];
  }
}
template <int J>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int lane) {
  return (uint64_t)lane_xor<J>((uint32_t)(v >> 32), lane) << 32 | lane_xor<J>((uint32_t)v, lane);
}
// Bitonic network over the lanes of a wave; lane 0 ends with the largest key.  A step exchanges with lane l ^ J
// inside sorted runs of N lanes, descending where bit N of the lane is clear.
template <int N, int J, typename K>
__device__ __forceinline__ K sort_step(K k, int lane) {
  const K o = lane_xor<J>(k, lane);
  return (((lane & J) == 0) == ((lane & N) == 0)) == (o > k) ? o : k;
}
template <int N, int J, typename K>
__device__ __forceinline__ K sort_run(K k, int lane) {   // a bitonic run of N lanes sorted
  k = sort_step<N, J>(k, lane);
  if constexpr (J > 1) k = sort_run<N, J / 2>(k, lane);
  return k;
}
template <typename K>
__device__ __forceinline__ K wave_sort_desc(K k, int lane) {
  k = sort_run<2, 1>(k, lane);
  k = sort_run<4, 2>(k, lane);
  k = sort_run<8, 4>(k, lane);
  k = sort_run<16, 8>(k, lane);
  k = sort_run<32, 16>(k, lane);
  return sort_run<64, 32>(k, lane);
}

__device__ __forceinline__ uint64_t max_u64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
  SPEXIS_DPP_REDUCE(v, dpp_u64_move, max_u64)
  return readlane_u64(v, kWave - 1);
}

// A wave's candidates: `keys` in LDS, of which `count` wait; `cut` is the least logit that still becomes one.
struct Candidates {
  uint64_t* keys;
  int count, sorted;   // the first `sorted` are in order
  float cut;
};
__device__ __forceinline__ void push(Candidates& c, bool mine, uint64_t key) {
  const uint64_t hit = __builtin_amdgcn_ballot_w64(mine);
  const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
  if (mine) c.keys[c.count + before] = key;
  c.count += (int)__popcll(hit);
}
// Sorts what waits and keeps the n largest.
__device__ __forceinline__ void compact(Candidates& c, int n, int lane) {
  if (c.count == c.sorted) return;
  wave_lds_fence();
  uint64_t best = 0;
#pragma unroll 1
  for (int b = 0; b < c.count; b += kWave) {
    const uint64_t k = b + lane < c.count ? c.keys[b + lane] : 0;
    if (__builtin_amdgcn_ballot_w64(k > readlane_u64(best, n - 1)) == 0) continue;
    const uint64_t s = wave_sort_desc(k, lane);
    if (b == 0) {
      best = s;
    } else {   // the larger of each and its mirror image in the other: the 64 largest, a bitonic run
      const uint64_t r = ((uint64_t)(uint32_t)__shfl((int)(uint32_t)(s >> 32), kWave - 1 - lane) << 32) |
                         (uint32_t)__shfl((int)(uint32_t)s, kWave - 1 - lane);
      best = sort_run<64, 32>(best > r ? best : r, lane);
    }
  }
  wave_lds_fence();
  if (lane < n) c.keys[lane] = best;
  wave_lds_fence();
  c.count = c.sorted = min(c.count, n);
  if (c.count == n) {
    c.cut = value_of((uint32_t)(readlane_u64(best, n - 1) >> 32) + 1u);   // just above the n-th
  }
}

// Running maximum m (a logit), Z and U of the logits seen, relative to m.
struct RowStats {
  float m, z, u;
};
__device__ __forceinline__ RowStats rebase(RowStats s, float m, float c) {
  const float d = (s.m - m) * c, a = fast_exp2(d);
  // a = 0: nothing is left of U (and d may be infinite); a NaN in Z stays
  return {m, s.z * a, a > 0.f ? a * (s.u + d * s.z) : 0.f};
}
__device__ __forceinline__ RowStats wave_combine(RowStats s, float c) {
  const RowStats r = rebase(s, wave_max(s.m), c);
  return {r.m, wave_sum(r.z), wave_sum(r.u)};
}

// Writes an item's outputs, one wave.  none: it has no token; x: the token's logit; best: its keys, the n largest in descending order over the lanes.
__device__ __forceinline__ void write_item(const LogprobParams& p, int item, bool none, float x, RowStats s, uint64_t best,
                                           int found, int lane) {
  const float nan = __builtin_nanf("");
  const bool bad = !none && !(s.z > 0.f);   // a NaN, +inf, or nothing above -inf
  const float lz = kLn2 * __builtin_log2f(s.z);
  // (not by way of w, which overflows for a masked logit of the type's lowest value)
  auto logp = [&](float x) { return bad ? nan : (x - s.m) * p.inv_t - lz; };
  if (lane < p.top) {
    const bool has = !none && !bad && lane < found;
    const int64_t at = (int64_t)item * p.top + lane;
    p.top_ids[at] = has ? (int32_t)~(uint32_t)best : -1;
    p.top_logprobs[at] = has ? logp(value_of((uint32_t)(best >> 32))) : bad ? nan : -__builtin_inff();
  }
  if (lane == 0) {
    p.logprob[item] = none ? 0.f : logp(x);
    if (p.entropy != nullptr) p.entropy[item] = none ? 0.f : bad ? nan : lz - kLn2 * (s.u / s.z);
  }
}

template <typename E>
__device__ __forceinline__ float logit_at(const E* row, int v) {
  if constexpr (sizeof(E) == 2) return __uint_as_float((uint32_t)row[v] << 16);
  else return row[v];
}

// An item's row (null: the item has no token) and its token's logit.
template <typename E>
__device__ __forceinline__ const E* item_row(const LogprobParams& p, int item, float& logit) {
  const int tok = p.tokens[item], r = p.row_ids != nullptr ? p.row_ids[item] : item;
  if (tok < 0 || tok >= p.V || r < 0 || r >= p.rows) return nullptr;
  const E* row = reinterpret_cast<const E*>(p.logits) + (int64_t)r * p.stride;
  logit = logit_at(row, tok);
  return row;
}

template <typename E, bool kTop>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobParams p) {
  constexpr int kVec = 16 / (int)sizeof(E), kLoads = kLpElems / kVec, kChunkVecs = kLoads * kWave;
  __shared__ uint64_t sm_keys[4][kTop ? kLpCap : 1];
  __shared__ uint32_t sm_most[4][kWave / 2];
  __shared__ RowStats sm_stats[4];
  __shared__ int sm_count[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int item = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  float logit;
  const E* row = item_row<E>(p, item, logit);
  if (row == nullptr) {
    if (p.parts == 1 && wave == 0) write_item(p, item, true, 0.f, {0.f, 1.f, 0.f}, 0, 0, lane);
    return;
  }
  // The row as 16-byte vectors; element e of vector v is logit v * kVec + e - skip.
  const int skip = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(E));
  const E* base = row - skip;
  const int vecs = (p.V + skip + kVec - 1) / kVec, chunks = (vecs + kChunkVecs - 1) / kChunkVecs;
  const int c0 = (int)((int64_t)chunks * part / p.parts), c1 = (int)((int64_t)chunks * (part + 1) / p.parts);

  u32x4 raw[kLoads];
  auto load = [&](int chunk) {
    const int v0 = chunk * kChunkVecs;
    if ((v0 > 0 || skip == 0) && (v0 + kChunkVecs) * kVec - skip <= p.V) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base) + v0 + i * kWave + lane);
      return;
    }
    // the row's first and last chunk: logits one by one, -inf outside the row
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const int at = (v0 + i * kWave + lane) * kVec + e - skip;
        if constexpr (sizeof(E) == 2) {
          const uint32_t x = at >= 0 && at < p.V ? (uint32_t)row[at] : 0xFF80u;
          raw[i][e / 2] = e % 2 ? raw[i][e / 2] | (x << 16) : x;
        } else {
          raw[i][e] = at >= 0 && at < p.V ? __float_as_uint(row[at]) : 0xFF800000u;
        }
      }
  };

  RowStats s = {kLowest, 0.f, 0.f};
  Candidates cand = {sm_keys[wave], 0, 0, -__builtin_inff()};
  float lane_most = -__builtin_inff();   // the lane's maximum so far
  // The threshold of the whole workgroup: the n-th largest (n <= 32) of its 256 lanes' maxima.
  auto agree = [&]() {
    const uint32_t mine = wave_sort_desc(order_of(lane_most), lane);
    __syncthreads();   // the last round's reads
    if (lane < kWave / 2) sm_most[wave][lane] = mine;
    __syncthreads();
    // two pairs of descending halves, each as one bitonic run; the second ends in ascending order
    const int at = lane < kWave / 2 ? lane : kWave - 1 - lane, up = lane < kWave / 2 ? 0 : 1;
    const uint32_t a = sort_run<64, 32>(sm_most[up][at], lane), b = ~sort_run<64, 32>(~sm_most[2 + up][at], lane);
    const uint32_t all = sort_run<64, 32>(a > b ? a : b, lane);
    cand.cut = fmaxf(cand.cut, value_of((uint32_t)__builtin_amdgcn_readlane((int)all, p.top - 1)));
  };
  int chunk = c0 + wave;
  if (chunk < c1) load(chunk);
  const int rounds = (c1 - c0 + 3) / 4;   // the same for the four waves
  for (int round = 0, next = 0; round < rounds; ++round, chunk += 4) {
    const bool some = chunk < c1;
    float x[kLpElems];
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (sizeof(E) == 2) x[i * kVec + e] = __uint_as_float(e % 2 ? raw[i][e / 2] & 0xFFFF0000u : raw[i][e / 2] << 16);
        else x[i * kVec + e] = __uint_as_float(raw[i][e]);
      }
    if (chunk + 4 < c1) load(chunk + 4);
    float group[kLpElems / kLpGroup], most = -__builtin_inff();
#pragma unroll
    for (int g = 0; g < kLpElems / kLpGroup; ++g) {
      group[g] = x[g * kLpGroup];
#pragma unroll
      for (int j = 1; j < kLpGroup; ++j) group[g] = fmaxf(group[g], x[g * kLpGroup + j]);
      most = fmaxf(most, group[g]);
    }
    if constexpr (kTop) {
      if (some) lane_most = fmaxf(lane_most, most);
      if (round == next) {   // after 1, 4, 16 ... rounds, the later times only where as many follow
        agree();
        next = 4 * next + 3;
        if (2 * (next + 1) > rounds) next = rounds;
      }
    }
    if (!some) continue;
    if (most > s.m) s = rebase(s, most, p.c);
#pragma unroll
    for (int j = 0; j < kLpElems; ++j) {
      const float w = (x[j] - s.m) * p.c, e = fast_exp2(w);
      s.z += e;
      s.u += e * fmaxf(w, kLowest);   // 0 * -inf would be NaN
    }
    if constexpr (kTop) {
      if (__builtin_amdgcn_ballot_w64(most >= cand.cut) != 0) {
        const int at = chunk * kChunkVecs * kVec - skip;
        int done = 0;   // groups that were searched
#pragma unroll
        for (int g = 0; g < kLpElems / kLpGroup; ++g) {
          if (cand.count > kLpKeep) continue;
          done = g + 1;
          if (__builtin_amdgcn_ballot_w64(group[g] >= cand.cut) == 0) continue;
#pragma unroll
          for (int j = g * kLpGroup; j < (g + 1) * kLpGroup; ++j) {
            if (__builtin_amdgcn_ballot_w64(x[j] >= cand.cut) == 0) continue;
            const int id = at + (j / kVec * kWave + lane) * kVec + j % kVec;
            // (outside the row lies -inf)
            push(cand, x[j] >= cand.cut && id >= 0 && id < p.V, (uint64_t)order_of(x[j]) << 32 | ~(uint32_t)id);
          }
        }
        // Many at once (sorted rows, ties): what is left of the chunk is read again, group by group, between sorts.
        // One place for the sort, outside the code that holds the chunk in registers.
        while (cand.count > kLpKeep) {
          compact(cand, p.top, lane);
          for (; done < kLpElems / kLpGroup && cand.count <= kLpKeep; ++done)
#pragma unroll 1
            for (int j = done * kLpGroup; j < (done + 1) * kLpGroup; ++j) {
              const int id = at + (j / kVec * kWave + lane) * kVec + j % kVec;
              float y = -__builtin_inff();
              if (id >= 0 && id < p.V) y = logit_at(row, id);
              push(cand, y >= cand.cut && id >= 0 && id < p.V, (uint64_t)order_of(y) << 32 | ~(uint32_t)id);
            }
        }
      }
    }
  }

  // ---- the four waves' together
  s = wave_combine(s, p.c);
  if (lane == 0) {
    sm_stats[wave] = s;
    sm_count[wave] = cand.count;
  }
  __syncthreads();
  if (wave != 0) return;
  s = wave_combine(lane < 4 ? sm_stats[lane] : RowStats{kLowest, 0.f, 0.f}, p.c);
  uint64_t best = 0;
  if constexpr (kTop) {
    static_assert(4 * kLpKeep <= kLpCap, "every wave's candidates fit into the first one's buffer");
    for (int w = 1; w < 4; ++w) {
      if (lane < sm_count[w]) cand.keys[cand.count + lane] = sm_keys[w][lane];   // at most kLpKeep
      cand.count += sm_count[w];
    }
    compact(cand, p.top, lane);
    best = lane < cand.count ? cand.keys[lane] : 0;
  }
  if (p.parts == 1) {
    write_item(p, item, false, logit, s, best, cand.count, lane);
    return;
  }
  if (lane == 0) reinterpret_cast<f32x4*>(p.part_stats)[blockIdx.x] = f32x4{s.m, s.z, s.u, 0.f};
  if (kTop && lane < p.top) p.part_keys[(int64_t)blockIdx.x * p.top + lane] = best;
}

// The parts of every item, one wave an item.
template <typename E, bool kTop>
__global__ __launch_bounds__(256) void logprobs_merge_kernel(LogprobParams p) {
  __shared__ uint64_t sm_keys[4][kTop ? kLpCap : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int item = blockIdx.x * 4 + wave;
  if (item >= p.items) return;
  float logit;
  const E* row = item_row<E>(p, item, logit);
  if (row == nullptr) return write_item(p, item, true, 0.f, {0.f, 1.f, 0.f}, 0, 0, lane);
  RowStats s = {kLowest, 0.f, 0.f};
  if (lane < p.parts) {   // at most a wave's lanes
    const f32x4 v = reinterpret_cast<const f32x4*>(p.part_stats)[(int64_t)item * p.parts + lane];
    s = {v[0], v[1], v[2]};
  }
  s = wave_combine(s, p.c);
  uint64_t best = 0;
  Candidates cand = {sm_keys[wave], 0, 0, 0.f};
  if constexpr (kTop) {
    const uint64_t* keys = p.part_keys + (int64_t)item * p.parts * p.top;
    // the largest of the parts' n-th keys: n keys reach it, so what is below it is not asked for
    const uint64_t least = wave_max_u64(lane < p.parts ? keys[lane * p.top + p.top - 1] : 0);   // 0: none
    const int total = p.parts * p.top;
    constexpr int kAhead = 8;
    static_assert(kLpKeep + kAhead * kWave <= kLpCap, "a round's candidates fit");
    for (int b0 = 0; b0 < total; b0 += kAhead * kWave) {
      uint64_t k[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) k[i] = b0 + i * kWave + lane < total ? keys[b0 + i * kWave + lane] : 0;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) push(cand, k[i] != 0 && k[i] >= least, k[i]);
      if (cand.count > kLpKeep) compact(cand, p.top, lane);
    }
    compact(cand, p.top, lane);
    best = lane < cand.count ? cand.keys[lane] : 0;
  }
  write_item(p, item, false, logit, s, best, cand.count, lane);
}

template <typename E, bool kTop>
static hipError_t launch_logprobs_t(const LogprobParams& p, hipStream_t s) {
  hipLaunchKernelGGL((logprobs_kernel<E, kTop>), dim3((unsigned)(p.items * p.parts)), dim3(256), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  hipLaunchKernelGGL((logprobs_merge_kernel<E, kTop>), dim3((unsigned)((p.items + 3) / 4)), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_logprobs(const LogprobParams& p, hipStream_t s) {
  if (p.in16) return p.top > 0 ? launch_logprobs_t<uint16_t, true>(p, s) : launch_logprobs_t<uint16_t, false>(p, s);
  return p.top > 0 ? launch_logprobs_t<float, true>(p, s) : launch_logprobs_t<float, false>(p, s);
}

}  // namespace spexis
