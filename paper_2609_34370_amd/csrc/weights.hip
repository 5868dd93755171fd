// The softmax weight that every cached key gets from a step's query rows, summed over the rows of its KV head: what an
// eviction goes by.  With the row's lse (the logarithm of its sum of exponentials, from the attention call) a weight is
// exp(scale <q, k> - lse): one pass over K, no statistics.
//
// A wave owns 32 keys of one (sequence, KV head): their K in registers, in the layout's order the A operand of
// S^T[key][row] = K Q^T (v_mfma_f32_32x32x16_bf16), against the rows 32 at a time, which the four waves of a workgroup share
// through LDS (each fetching them for itself, as many bytes as K, took 98 instead of 88 us at the step below, 58 instead of 26
// at the prompts).  Lane l then holds row l%32 and keys 8*(i/4) + 4*(l/32) + i%4: it adds its weights up over the row tiles,
// and one reduction over the lanes at the end gives the sums, always in the same order.
//
// Bound by the bytes of K for a step's rows: 64 sequences of 1024 to 4096 keys (32 query heads over 8 of 128, up to 5 tokens;
// 363 MB) take 73 to 88 us on four cards, 4.1 to 5.0 TB/s.  With many rows by a workgroup's start and its chain of row
// tiles: 64 tokens of 28 heads over 6 prompts of 2001 to 8000 keys (4 KV heads; 14.3 GFLOP) 25 to 27 us, vector instructions active
// for 42% of the cycles, the matrix cores 18%, LDS 14%.  Two key tiles a wave, which halve the reads of q, took 108 and 39 us with three instead of five waves a SIMD; rows fetched two tiles ahead 79 and 29.
#include "attention.h"
#include "tiles.h"

namespace spexis {

constexpr int kWeightKeys = 128;   // keys of a workgroup: 32 a wave

template <int D, int BS>
__global__ __launch_bounds__(256)
void weights_kernel(WeightParams p, int chunks) {
  constexpr int KS = D / 16;   // k-steps
  __shared__ u32x4 sm_q[2][KS][kWave];   // a tile of rows, as operands
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int h = (int)(blockIdx.x % (uint32_t)p.hkv);
  const int x = (int)(blockIdx.x / (uint32_t)p.hkv), b = x / chunks, key0 = (x % chunks) * kWeightKeys, k0 = key0 + wave * 32;
  sint32 *qsl = (sint32*)p.qsl, *lens = (sint32*)p.seq_lens, *acc_len = (sint32*)p.accepted;
  const int q0 = clampi(qsl[b], 0, p.total_tokens), len = lens[b];
  int n = min(clampi(qsl[b + 1], q0, p.total_tokens) - q0, p.max_query_len);
  if (p.accepted) n = clampi(acc_len[b] + 1, 0, n);
  const int S = clampi(len, n, (int)min((int64_t)p.max_blocks * BS, (int64_t)p.max_seq_len));
  const int first = p.first_keys ? clampi(((sint32*)p.first_keys)[b], 0, S) : 0;
  if (key0 >= S || key0 + kWeightKeys <= first) return;
  const int L = S - n, R = n * p.group;
  sint32* table = (sint32*)p.block_tables + (int64_t)b * p.max_blocks;
  const int last = (S - 1) / BS;
  // the chunks of 16 keys (those behind the end repeat the last block: their sums are not written)
  constexpr int kPer = 32 / BS;   // blocks a tile
  int64_t chunk[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    chunk[i] = (int64_t)clampi(table[min(k0 / BS + i, last)], 0, p.num_blocks - 1) * p.hkv + h;
  // what a masked key's score becomes: minus infinity once it is scaled
  const float no_score = p.scale_log2e < 0.f ? INFINITY : -INFINITY;
  u32x4 kf[KS];
  const int64_t mine = col >= 16 ? chunk[kPer - 1] : chunk[0];
  const uint16_t* kp = reinterpret_cast<const uint16_t*>(p.k_cache) + mine * BS * D + (half * BS + col % BS) * 8;
#pragma unroll
  for (int s = 0; s < KS; ++s) kf[s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + s * 2 * BS * 8));
  float acc[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  // Rows from the first token that sees a key of the workgroup on, 32 at a time: each wave fetches a quarter of their q for all,
  // one tile ahead.
  constexpr int kMine = KS / 4;
  u32x4 q[kMine];
  float sum = 0.f, sum_next = 0.f;   // log2 of the row's sum of exponentials; infinite where there is no row: no weight
  int lim = 0, lim_next = 0;         // the last key that the lane's row sees
  auto load = [&](int r0) {
    const int r = min(r0 + col, R - 1), j = r / p.group;
    const int64_t row = (int64_t)(q0 + j) * p.hq + h * p.group + r - j * p.group;
    const uint16_t* a = reinterpret_cast<const uint16_t*>(p.q) + row * D + 8 * half + 16 * kMine * wave;
    sum_next = r0 + col < R ? p.lse[row] : INFINITY;
    lim_next = L + j;
#pragma unroll
    for (int i = 0; i < kMine; ++i) q[i] = ld16(a + 16 * i);
  };
  int r0 = max(key0 - L, 0) * p.group;
  if (r0 < R) load(r0);
  for (int buf = 0; r0 < R; r0 += 32, buf ^= 1) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) sm_q[buf][kMine * wave + i][lane] = q[i];
    sum = sum_next * kLog2E;
    lim = lim_next;
    __syncthreads();   // (the other buffer's readers are past it too when this one is written again)
    if (r0 + 32 < R) load(r0 + 32);
    // the rows from r0 on see the keys up to this one
    const int sure = L + r0 / p.group;
    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[s]), as_bf16x8(sm_q[buf][s][lane]), sc, 0, 0, 0);
    if (k0 + 31 > sure) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (k0 + (e >> 2) * 8 + 4 * half + (e & 3) > lim) sc[e] = no_score;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += fast_exp2(fmaf(sc[e], p.scale_log2e, -sum));
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {   // lanes 31 and 63 end with the sums over the rows
    float v = acc[e];
    v += dpp_sum_move<kDppRowShr + 1, 0xF>(v);
    v += dpp_sum_move<kDppRowShr + 2, 0xF>(v);
    v += dpp_sum_move<kDppRowShr + 4, 0xF>(v);
    v += dpp_sum_move<kDppRowShr + 8, 0xF>(v);
    v += dpp_sum_move<kDppRowBcast15, 0xA>(v);
    acc[e] = v;
  }
  if (col != 31) return;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int key = k0 + 8 * a + 4 * half;
    const int64_t at = (a >= 2 ? chunk[kPer - 1] : chunk[0]) * BS + key % BS;
    if (key >= first && key + 3 < S) {
      f32x4 v = {acc[4 * a], acc[4 * a + 1], acc[4 * a + 2], acc[4 * a + 3]};
      if (p.weights_in && key < L) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(p.weights_in + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += key + e < L ? w[e] : 0.f;
      }
      *reinterpret_cast<f32x4*>(p.weights + at) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key + e >= first && key + e < S) p.weights[at + e] = acc[4 * a + e] + (p.weights_in && key + e < L ? p.weights_in[at + e] : 0.f);
    }
  }
}

template <int D>
static hipError_t launch_weights_t(const WeightParams& p, hipStream_t s) {
  const int chunks = (p.max_seq_len + kWeightKeys - 1) / kWeightKeys;
  const dim3 grid((unsigned)((int64_t)p.num_seqs * chunks * p.hkv));
  if (p.block_size == 16) hipLaunchKernelGGL((weights_kernel<D, 16>), grid, dim3(256), 0, s, p, chunks);
  else hipLaunchKernelGGL((weights_kernel<D, 32>), grid, dim3(256), 0, s, p, chunks);
  return hipGetLastError();
}

hipError_t launch_weights(const WeightParams& p, hipStream_t s) {
  return p.head_dim == 128 ? launch_weights_t<128>(p, s) : launch_weights_t<64>(p, s);
}

}  // namespace spexis
