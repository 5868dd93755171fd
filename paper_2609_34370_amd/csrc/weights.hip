// The softmax weight that every cached key gets from a step's query rows, summed over the rows of its KV head: what an
// eviction goes by.  With the row's lse (the logarithm of its sum of exponentials, from the attention call) a weight is
// exp(scale <q, k> - lse): one pass over K, no statistics.
//
// A wave owns 32 keys of one (sequence, KV head): their K in registers, in the layout's order the A operand of
// S^T[key][row] = K Q^T (v_mfma_f32_32x32x16_bf16), against the rows 32 at a time.  Lane l then holds row l%32 and keys
// 8*(i/4) + 4*(l/32) + i%4: it adds its weights up over the row tiles, and one reduction over the lanes at the end gives the
// sums, always in the same order.
#include "attention.h"

namespace spexis {

template <int D, int BS>
__global__ __launch_bounds__(256) void weights_kernel(WeightParams p, int chunks) {
  constexpr int KS = D / 16;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int h = (int)(blockIdx.x % (uint32_t)p.hkv);
  const int x = (int)(blockIdx.x / (uint32_t)p.hkv), b = x / chunks, k0 = (x % chunks) * 128 + wave * 32;
  const int q0 = clampi(p.qsl[b], 0, p.total_tokens);
  int n = min(clampi(p.qsl[b + 1], q0, p.total_tokens) - q0, p.max_query_len);
  if (p.accepted) n = clampi(p.accepted[b] + 1, 0, n);
  const int S = clampi(p.seq_lens[b], n, (int)min((int64_t)p.max_blocks * BS, (int64_t)p.max_seq_len));
  if (k0 >= S) return;
  const int L = S - n, R = n * p.group;
  sint32* table = (sint32*)p.block_tables + (int64_t)b * p.max_blocks;
  const int last = (S - 1) / BS;
  const int64_t ca = (int64_t)clampi(table[k0 / BS], 0, p.num_blocks - 1) * p.hkv + h;
  const int64_t cb = BS == 32 ? ca : (int64_t)clampi(table[min(k0 / BS + 1, last)], 0, p.num_blocks - 1) * p.hkv + h;
  const uint16_t* kp = reinterpret_cast<const uint16_t*>(p.k_cache) + (BS == 16 && col >= 16 ? cb : ca) * BS * D +
                       (half * BS + col % BS) * 8;
  u32x4 kf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) kf[s] = ld16(kp + s * 2 * BS * 8);
  float acc[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  // rows from the first token that sees key k0 on
  for (int r0 = max(k0 - L, 0) * p.group; r0 < R; r0 += 32) {
    const int r = min(r0 + col, R - 1), j = r / p.group;
    const int64_t row = (int64_t)(q0 + j) * p.hq + h * p.group + r % p.group;
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + row * D + 8 * half;
    const float sum = p.lse[row] * kLog2E;
    const int lim = r0 + col < R ? L + j : -1;   // the last key that the lane's row sees
    u32x4 qf[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = ld16(q + 16 * s);
    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[s]), as_bf16x8(qf[s]), sc, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float w = fast_exp2(fmaf(sc[e], p.scale_log2e, -sum));
      acc[e] += k0 + (e >> 2) * 8 + 4 * half + (e & 3) <= lim ? w : 0.f;
    }
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
    const int64_t at = (BS == 16 && a >= 2 ? cb : ca) * BS + key % BS;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (key + e < S) p.weights[at + e] = acc[4 * a + e] + (p.weights_in && key + e < L ? p.weights_in[at + e] : 0.f);
  }
}

template <int D>
static hipError_t launch_weights_t(const WeightParams& p, hipStream_t s) {
  const int chunks = (p.max_seq_len + 127) / 128;
  const dim3 grid((unsigned)((int64_t)p.num_seqs * chunks * p.hkv));
  if (p.block_size == 16) hipLaunchKernelGGL((weights_kernel<D, 16>), grid, dim3(256), 0, s, p, chunks);
  else hipLaunchKernelGGL((weights_kernel<D, 32>), grid, dim3(256), 0, s, p, chunks);
  return hipGetLastError();
}

hipError_t launch_weights(const WeightParams& p, hipStream_t s) {
  return p.head_dim == 128 ? launch_weights_t<128>(p, s) : launch_weights_t<64>(p, s);
}

}  // namespace spexis
