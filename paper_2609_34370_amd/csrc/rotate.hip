// The rotating appends: the rotary position embedding of a step's q and k, and its new K/V rows into the
// paged cache, in one launch -- into the bf16 cache of spexis_append_kv, or into a cache held in 8 bits
// (e4m3 codes, one power-of-two scale per block of tokens, KV head and pool).
//
// A pair (x_a, x_b) of frequency i turns by the angle whose cosine c and sine s the table holds:
//   y_a = x_a c - x_b s,   y_b = x_b c + x_a s.
// Memory bound: every row is read once and written once, about three operations an element.
//
// Work split.  A wave takes one (block of tokens, KV head) that gets new rows, or one query token with all
// its heads; the waves of a workgroup share nothing.  A block belongs to one wave because the scale of an
// 8-bit block needs all its rows, and because V is stored 8 slots to a 16-byte piece: the wave rewrites the
// pieces it touches whole, so no two waves write into one piece.
// Which block: sequence b gets the indices from start(b) = floor(qsl[b] / bs) + 2 b.  n new tokens touch at most
// floor(n / bs) + 2 blocks, which start(b+1) - start(b) is never below, so the launch needs no length
// on the host and no scan: wave-wide search for the last b with start(b) <= index, two probes for 4096 sequences.
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace spexis {

// The last b in [0, n) with f(b) <= x, for f not falling and f(0) <= x (an f that falls gives some b in range).
template <typename F>
__device__ __forceinline__ int wave_search(int n, int x, int lane, F f) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const uint64_t hit = __builtin_amdgcn_ballot_w64(at < hi && f(at) <= x);
    lo += max((int)__popcll(hit) - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int seq_start(const RotateParams& p, int b) { return clampi(p.qsl[b], 0, p.total_tokens); }

// The two 8-element chunks that one task takes of a row, a and b, and how they turn.  Halves: element i pairs
// with i + rot/2, so the chunks are 8t.. and rot/2 + 8t..; pairs: (2i, 2i+1), chunks 16t.. and 16t+8...
// Either way the task's frequencies are 8t .. 8t+7.  Past the rotated part: two chunks that are copied.
struct Task {
  int a, b, freq;
  bool turns;
};
__device__ __forceinline__ Task row_task(const RotateParams& p, int t) {
  if (16 * t >= p.rot || p.cos_sin == nullptr) return {16 * t, 16 * t + 8, 0, false};
  return p.style == 0 ? Task{8 * t, p.rot / 2 + 8 * t, 8 * t, true} : Task{16 * t, 16 * t + 8, 8 * t, true};
}

struct Angles {
  float c[8], s[8];
};
__device__ __forceinline__ Angles load_angles(const RotateParams& p, const Task& t, int pos) {
  Angles g;
  const float* row = p.cos_sin + (int64_t)clampi(pos, 0, p.max_position - 1) * p.rot + t.freq;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 c = *reinterpret_cast<const f32x4*>(row + 4 * i), s = *reinterpret_cast<const f32x4*>(row + p.rot / 2 + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      g.c[4 * i + e] = c[e];
      g.s[4 * i + e] = s[e];
    }
  }
  return g;
}

__device__ __forceinline__ void widen(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 narrow(const float (&x)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  return v;
}

// One pair.  T double: a bf16 times an fp32 has 32 significant bits, so the sum is rounded once in 64 bits and
// once to 32; what an 8-bit code is rounded from is then the same in any order of evaluation.  T float: before
// a rounding to bf16, whose half step is 2^15 times larger.
template <typename T>
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const T x = a, y = b, cc = c, ss = s;
  a = (float)(x * cc - y * ss);
  b = (float)(y * cc + x * ss);
}
template <typename T>
__device__ __forceinline__ void turn_task(const RotateParams& p, const Task& t, const Angles& g, float (&x)[8], float (&y)[8]) {
  if (!t.turns) return;
  if (p.style == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn<T>(x[i], y[i], g.c[i], g.s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn<T>(x[2 * i], x[2 * i + 1], g.c[i], g.s[i]);
      turn<T>(y[2 * i], y[2 * i + 1], g.c[4 + i], g.s[4 + i]);
    }
  }
}

// q of one token, every head: the lanes are (head, task), so the token's angles are loaded once.
template <int D>
__device__ __forceinline__ void rotate_query(const RotateParams& p, int tok, int lane) {
  constexpr int kTasks = D / 16, kHeads = kWave / kTasks;
  const int t = lane % kTasks;
  const Task task = row_task(p, t);
  int pos = 0;
  if (p.positions != nullptr) {
    pos = p.positions[tok];
  } else {
    const int b = wave_search(p.num_seqs, tok, lane, [&](int i) { return seq_start(p, i); });
    const int q1 = clampi(p.qsl[b + 1], 0, p.total_tokens);
    pos = p.seq_lens[b] - (q1 - tok);
  }
  Angles g;
  if (task.turns) g = load_angles(p, task, pos);
  const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + (int64_t)tok * p.hq * D;
  uint16_t* o = reinterpret_cast<uint16_t*>(p.q_out) + (int64_t)tok * p.hq * D;
#pragma unroll 4
  for (int h = lane / kTasks; h < p.hq; h += kHeads) {
    float x[8], y[8];
    widen(ld16(q + h * D + task.a), x);
    widen(ld16(q + h * D + task.b), y);
    turn_task<float>(p, task, g, x, y);
    st16(o + h * D + task.a, narrow(x));
    st16(o + h * D + task.b, narrow(y));
  }
}

// Two values of at most 448 to e4m3 codes, to nearest even.  The format has no infinity: what is not finite
// becomes the NaN 0x7f (put in by hand: the conversion would give a NaN of either sign).
__device__ __forceinline__ uint32_t pack_e4m3x2(float x, float y) {
  const bool bx = !(fabsf(x) < __builtin_inff()), by = !(fabsf(y) < __builtin_inff());
  const uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bx ? 0.f : x, by ? 0.f : y, 0, false) & 0xFFFFu;
  return w | (bx ? 0x7Fu : 0u) | (by ? 0x7F00u : 0u);
}
__device__ __forceinline__ u32x2 pack_e4m3x8(const float (&x)[8], float mul) {
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = pack_e4m3x2(x[4 * i] * mul, x[4 * i + 1] * mul) | (pack_e4m3x2(x[4 * i + 2] * mul, x[4 * i + 3] * mul) << 16);
  return w;
}
// Four codes whose scale changes by the factor r.
__device__ __forceinline__ uint32_t rescale_e4m3x4(uint32_t w, float r) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return pack_e4m3x2(lo[0] * r, lo[1] * r) | (pack_e4m3x2(hi[0] * r, hi[1] * r) << 16);
}

// The exponent of the least power of two, from 2^-100, by which `most` is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ int least_exp(float most) {
  const uint32_t u = __float_as_uint(most);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, -100);
}
__device__ __forceinline__ float exp_float(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The largest finite magnitude of 16 values, at least m.
__device__ __forceinline__ float most_finite(const float (&x)[8], const float (&y)[8], float m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]), b = fabsf(y[i]);
    m = fmaxf(m, a < __builtin_inff() ? a : 0.f);
    m = fmaxf(m, b < __builtin_inff() ? b : 0.f);
  }
  return m;
}

// The new rows of one (block of tokens, KV head).
template <int D, int BS, bool k8>
__device__ __forceinline__ void append_block(const RotateParams& p, int index, int h, int lane, u32x4* lds) {
  constexpr int kTasks = D / 16, kMine = BS * kTasks / kWave;   // tasks of a row; of a lane, at most
  constexpr int kUnits = BS / 16;
  const int b = wave_search(p.num_seqs, index, lane, [&](int i) { return seq_start(p, i) / BS + 2 * i; });
  const int q0 = seq_start(p, b), q1 = clampi(p.qsl[b + 1], q0, p.total_tokens);
  const int cap = p.max_blocks * BS;
  const int n = min(q1 - q0, cap), S = clampi(p.seq_lens[b], n, cap), L = S - n;
  const int t = L / BS + (index - (q0 / BS + 2 * b));
  if (n == 0 || t < L / BS || t > (S - 1) / BS) return;
  const int lo = max(L, t * BS), m = min(S, (t + 1) * BS) - lo;   // first new position, new rows
  const int first = lo - t * BS;                                  // its slot: the block holds that many rows
  const int blk = clampi(p.block_tables[(int64_t)b * p.max_blocks + t], 0, p.num_blocks - 1);
  const int64_t at = (int64_t)blk * p.hkv + h;
  const int tok0 = q0 + (lo - L);

  // ---- the new rows: tasks k = row * kTasks + t, the lane's at lane, lane + 64, ...
  const uint16_t* nk = reinterpret_cast<const uint16_t*>(p.new_k);
  const uint16_t* nv = reinterpret_cast<const uint16_t*>(p.new_v);
  const Task task = row_task(p, lane % kTasks);   // 64 is a multiple of kTasks: the same for all of them
  float kx[kMine][8], ky[kMine][8];
  u32x4 va[kMine], vb[kMine];
  float kmost = 0.f, vmost = 0.f;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int r = (lane + kWave * i) / kTasks;
    if (r >= m) continue;
    const int64_t row = ((int64_t)(tok0 + r) * p.hkv + h) * D;
    const u32x4 a = ld16(nk + row + task.a), c = ld16(nk + row + task.b);
    va[i] = ld16(nv + row + 16 * (lane % kTasks));
    vb[i] = ld16(nv + row + 16 * (lane % kTasks) + 8);
    widen(a, kx[i]);
    widen(c, ky[i]);
    if (task.turns) {
      const Angles g = load_angles(p, task, p.positions != nullptr ? p.positions[tok0 + r] : lo + r);
      turn_task<std::conditional_t<k8, double, float>>(p, task, g, kx[i], ky[i]);
    }
    if constexpr (k8) {
      kmost = most_finite(kx[i], ky[i], kmost);
      float x[8], y[8];
      widen(va[i], x);
      widen(vb[i], y);
      vmost = most_finite(x, y, vmost);
    }
  }

  // ---- the scales: never lowered while the block holds earlier rows, whose codes would overflow
  float kratio = 1.f, vratio = 1.f, kmul = 1.f, vmul = 1.f;
  if constexpr (k8) {
    float* sp = p.scales + 2 * at;
    float ks = exp_float(least_exp(wave_max(kmost))), vs = exp_float(least_exp(wave_max(vmost)));
    if (first > 0) {
      const float ko = sp[0], vo = sp[1];
      ks = fmaxf(ks, ko);
      vs = fmaxf(vs, vo);
      kratio = ko / ks;
      vratio = vo / vs;
    }
    if (lane == 0) *reinterpret_cast<f32x2*>(sp) = f32x2{ks, vs};
    kmul = 1.f / ks;   // exact: a power of two
    vmul = 1.f / vs;
  }

  // ---- K: 8 dims of a slot are contiguous (16 in the 8-bit cache)
  if constexpr (k8) {
    uint8_t* kc = reinterpret_cast<uint8_t*>(p.k_cache) + at * (BS * D);
    auto chunk = [&](int slot, int d) { return kc + ((slot / 16 * (D / 16) + d / 16) * 16 + slot % 16) * 16 + d % 16; };
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int r = (lane + kWave * i) / kTasks;
      if (r >= m) continue;
      *reinterpret_cast<u32x2*>(chunk(first + r, task.a)) = pack_e4m3x8(kx[i], kmul);
      *reinterpret_cast<u32x2*>(chunk(first + r, task.b)) = pack_e4m3x8(ky[i], kmul);
    }
    if (kratio != 1.f)
      for (int k = lane; k < first * kTasks; k += kWave) {
        u32x4* g = reinterpret_cast<u32x4*>(chunk(k / kTasks, 16 * (k % kTasks)));
        u32x4 w = *g;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = rescale_e4m3x4(w[e], kratio);
        *g = w;
      }
  } else {
    uint16_t* kc = reinterpret_cast<uint16_t*>(p.k_cache) + at * (BS * D);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int r = (lane + kWave * i) / kTasks;
      if (r >= m) continue;
      st16(kc + (task.a / 8 * BS + first + r) * 8, narrow(kx[i]));
      st16(kc + (task.b / 8 * BS + first + r) * 8, narrow(ky[i]));
    }
  }

  // ---- V: transposed through LDS, then the touched units' 16-byte pieces
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int k = lane + kWave * i;
    if (k / kTasks >= m) continue;
    if constexpr (k8) {
      float x[8], y[8];
      widen(va[i], x);
      widen(vb[i], y);
      const u32x2 a = pack_e4m3x8(x, vmul), c = pack_e4m3x8(y, vmul);
      lds[k] = u32x4{a[0], a[1], c[0], c[1]};
    } else {
      lds[2 * k] = va[i];
      lds[2 * k + 1] = vb[i];
    }
  }
  wave_lds_fence();
  // Piece (unit, part, half): the 8 slots (i / 4) * 8 + half * 4 + i % 4 of a unit of 16, of one dim (bf16) or of
  // dims d and d + 32 (8 bits).
  constexpr int kPieces = k8 ? D : 2 * D;   // of a unit
  for (int c = lane; c < kUnits * kPieces; c += kWave) {
    const int u = c / kPieces, part = c % kPieces, half = part & 1;
    const int s0 = u * 16 + half * 4;
    // slots s0 .. s0+3 and s0+8 .. s0+11
    const int l = first, e = first + m;
    const bool some = (s0 < e && s0 + 4 > l) || (s0 + 8 < e && s0 + 12 > l);
    const bool all = s0 >= l && s0 + 12 <= e;
    const bool again = k8 && vratio != 1.f && s0 < first;
    if (!some && !again) continue;
    u32x4* g;
    int d;
    if constexpr (k8) {
      d = part / 64 * 64 + part % 64 / 2;
      g = reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(p.v_cache) + at * (BS * D) + (u * D + part) * 16);
    } else {
      d = part / 2;
      g = reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(p.v_cache) + at * (BS * D) + d * BS + u * 16 + half * 8);
    }
    u32x4 w = {0u, 0u, 0u, 0u};
    if (!all) w = *g;
    if constexpr (k8) {
      const uint8_t* rows = reinterpret_cast<const uint8_t*>(lds);
#pragma unroll
      for (int j = 0; j < 2; ++j)       // dim d + 32 j: words 2j, 2j+1
#pragma unroll
        for (int q = 0; q < 2; ++q) {   // slots s0 + 8 q ..
          uint32_t x = w[2 * j + q];
          if (vratio != 1.f) {
            const uint32_t y = rescale_e4m3x4(x, vratio);
#pragma unroll
            for (int i = 0; i < 4; ++i)   // only rows the sequence holds
              if (s0 + 8 * q + i < first) x = (x & ~(0xFFu << (8 * i))) | (y & (0xFFu << (8 * i)));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = s0 + 8 * q + i - first;
            if (r >= 0 && r < m) x = (x & ~(0xFFu << (8 * i))) | ((uint32_t)rows[r * D + d + 32 * j] << (8 * i));
          }
          w[2 * j + q] = x;
        }
    } else {
      const uint16_t* rows = reinterpret_cast<const uint16_t*>(lds);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = s0 + (i >> 2) * 8 + (i & 3) - first;
        if (r < 0 || r >= m) continue;
        const uint32_t v = rows[r * D + d];
        w[i >> 1] = (i & 1) ? ((w[i >> 1] & 0x0000FFFFu) | (v << 16)) : ((w[i >> 1] & 0xFFFF0000u) | v);
      }
    }
    *g = w;
  }
}

template <int D, int BS, bool k8>
__global__ __launch_bounds__(256) void rotate_append_kernel(RotateParams p) {
  __shared__ u32x4 lds[4][BS * D * (k8 ? 1 : 2) / 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int w = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + wave);   // below 2^31 (host)
  if (w < p.append_waves) {
    append_block<D, BS, k8>(p, w / p.hkv, w % p.hkv, lane, lds[wave]);
  } else if (w - p.append_waves < p.query_waves) {
    rotate_query<D>(p, w - p.append_waves, lane);
  }
}

template <int D, int BS, bool k8>
static hipError_t launch_rotate_t(const RotateParams& p, hipStream_t s) {
  const unsigned wgs = ((unsigned)p.append_waves + (unsigned)p.query_waves + 3) / 4;
  hipLaunchKernelGGL((rotate_append_kernel<D, BS, k8>), dim3(wgs), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <bool k8>
static hipError_t launch_rotate_k(const RotateParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.block_size == 16 ? launch_rotate_t<128, 16, k8>(p, s) : launch_rotate_t<128, 32, k8>(p, s);
  return p.block_size == 16 ? launch_rotate_t<64, 16, k8>(p, s) : launch_rotate_t<64, 32, k8>(p, s);
}

hipError_t launch_rotate_append(RotateParams p, hipStream_t s) {
  p.append_waves = (int)rotate_append_waves(p.total_tokens, p.block_size, p.num_seqs, p.hkv);
  p.query_waves = p.q != nullptr ? p.total_tokens : 0;
  return p.scales != nullptr ? launch_rotate_k<true>(p, s) : launch_rotate_k<false>(p, s);
}

}  // namespace spexis
