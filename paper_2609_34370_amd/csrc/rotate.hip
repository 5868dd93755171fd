// The rotating appends: the rotary position embedding of a step's q and k, and its new K/V rows into the
// paged cache, in one launch -- into the bf16 cache of spexis_append_kv, or into a cache held in 8 bits
// (e4m3 codes, one power-of-two scale per block of tokens, KV head and pool).
//
// A pair (x_a, x_b) of frequency i turns by the angle whose cosine c and sine s the table holds:
//   y_a = x_a c - x_b s,   y_b = x_b c + x_a s.
// Memory bound: every row is read once and written once, about three operations an element.
//
// Work split.  A workgroup takes one (block of tokens, KV head) that gets new rows, or a wave one query token with all
// its heads.  A block belongs to one workgroup because the scale of an 8-bit block needs all its rows, and
// because V is stored 8 slots to a 16-byte piece, which is rewritten whole: no two workgroups write into one piece.
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

// q of one token, every head, one wave: the lanes are (head, task), so the token's angles are loaded once; the rows are
// in flight while the position is looked up.
template <int D>
__device__ __forceinline__ void rotate_query(const RotateParams& p, int tok, int lane) {
  constexpr int kTasks = D / 16, kHeads = kWave / kTasks, kAhead = 4;
  const Task task = row_task(p, lane % kTasks);
  const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + (int64_t)tok * p.hq * D;
  uint16_t* o = reinterpret_cast<uint16_t*>(p.q_out) + (int64_t)tok * p.hq * D;
  u32x4 a[kAhead], b[kAhead];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = min(h0 + i * kHeads, p.hq - 1);
      a[i] = ld16(q + h * D + task.a);
      b[i] = ld16(q + h * D + task.b);
    }
  };
  load(lane / kTasks);
  int pos = 0;
  if (p.positions != nullptr) {
    pos = p.positions[tok];
  } else {
    const int s = wave_search(p.num_seqs, tok, lane, [&](int i) { return seq_start(p, i); });
    pos = p.seq_lens[s] - (clampi(p.qsl[s + 1], 0, p.total_tokens) - tok);
  }
  Angles g;
  if (task.turns) g = load_angles(p, task, pos);
  for (int h0 = lane / kTasks; h0 < p.hq; h0 += kAhead * kHeads) {
    if (h0 != lane / kTasks) load(h0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * kHeads;
      if (h >= p.hq) break;
      float x[8], y[8];
      widen(a[i], x);
      widen(b[i], y);
      turn_task<float>(p, task, g, x, y);
      st16(o + h * D + task.a, narrow(x));
      st16(o + h * D + task.b, narrow(y));
    }
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

// A thread takes one task of K and of V of a block's rows: a workgroup is a (block of tokens, KV head).
template <int D, int BS>
constexpr int kThreads = BS * D / 16;

// The new rows of one (block of tokens, KV head).
template <int D, int BS, bool k8>
__device__ __forceinline__ void append_block(const RotateParams& p, int index, int h, int thread) {
  constexpr int kTasks = D / 16, kWaves = kThreads<D, BS> / kWave;
  const int lane = thread & 63, wave = thread >> 6;
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

  // ---- every load: the thread's part of a new row, its token's angles, the V piece that it will write, the scales
  const int r = thread / kTasks;
  const bool row = r < m;
  const Task task = row_task(p, thread % kTasks);
  u32x4 ka, kb, va, vb;
  Angles g;
  if (row) {
    const int tok = q0 + (lo - L) + r;
    const int64_t k = ((int64_t)tok * p.hkv + h) * D;
    const uint16_t* nk = reinterpret_cast<const uint16_t*>(p.new_k) + k;
    const uint16_t* nv = reinterpret_cast<const uint16_t*>(p.new_v) + k;
    ka = ld16(nk + task.a);
    kb = ld16(nk + task.b);
    va = ld16(nv + 16 * (thread % kTasks));
    vb = ld16(nv + 16 * (thread % kTasks) + 8);
    if (task.turns) g = load_angles(p, task, p.positions != nullptr ? p.positions[tok] : lo + r);
  }
  // Piece (unit, part, half): the 8 slots (i / 4) * 8 + half * 4 + i % 4 of a unit of 16, of one dim (bf16) or of
  // dims d and d + 32 (8 bits).
  constexpr int kPieces = k8 ? 1 : 2, kUnitPieces = k8 ? D : 2 * D;   // of a thread, of a unit
  u32x4 piece[kPieces];
  u32x4* place[kPieces];
  int slot[kPieces], dim[kPieces];   // the piece's first slot, and dim
  bool some[kPieces];                // new rows lie in it
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int c = thread + i * kThreads<D, BS>, u = c / kUnitPieces, part = c % kUnitPieces;
    const int s0 = slot[i] = u * 16 + (part & 1) * 4;   // slots s0 .. s0+3 and s0+8 .. s0+11
    dim[i] = k8 ? part / 64 * 64 + part % 64 / 2 : part / 2;
    place[i] = reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(p.v_cache) + at * (BS * D * (k8 ? 1 : 2)) +
                                        (k8 ? (u * D + part) * 16 : dim[i] * BS * 2 + u * 32 + (part & 1) * 16));
    some[i] = (s0 < first + m && s0 + 4 > first) || (s0 + 8 < first + m && s0 + 12 > first);
    piece[i] = u32x4{0u, 0u, 0u, 0u};
    if (some[i] && !(s0 >= first && s0 + 12 <= first + m)) piece[i] = *place[i];
  }
  float* sp = k8 ? p.scales + 2 * at : nullptr;
  f32x2 before = {0.f, 0.f};
  if (k8 && first > 0) before = *reinterpret_cast<const f32x2*>(sp);

  __shared__ u32x4 rows[BS * D * (k8 ? 1 : 2) / 16];   // V's new rows, as they will lie in the cache
  float kx[8], ky[8];
  if (row) {
    widen(ka, kx);
    widen(kb, ky);
    turn_task<std::conditional_t<k8, double, float>>(p, task, g, kx, ky);
  }
  float kratio = 1.f, vratio = 1.f;
  if constexpr (k8) {
    float vx[8], vy[8], kmost = 0.f, vmost = 0.f;
    if (row) {
      widen(va, vx);
      widen(vb, vy);
      kmost = most_finite(kx, ky, kmost);
      vmost = most_finite(vx, vy, vmost);
    }
    kmost = wave_max(kmost);
    vmost = wave_max(vmost);
    if constexpr (kWaves > 1) {
      __shared__ f32x2 most[kWaves];
      if (lane == 0) most[wave] = f32x2{kmost, vmost};
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        kmost = fmaxf(kmost, most[w][0]);
        vmost = fmaxf(vmost, most[w][1]);
      }
    }
    // the scales: never lowered while the block holds earlier rows, whose codes would overflow
    float ks = exp_float(least_exp(kmost)), vs = exp_float(least_exp(vmost));
    if (first > 0) {
      ks = fmaxf(ks, before[0]);
      vs = fmaxf(vs, before[1]);
      kratio = before[0] / ks;
      vratio = before[1] / vs;
    }
    if (thread == 0) *reinterpret_cast<f32x2*>(sp) = f32x2{ks, vs};
    // K: 16 dims of a slot are contiguous
    uint8_t* kc = reinterpret_cast<uint8_t*>(p.k_cache) + at * (BS * D);
    auto chunk = [&](int slot, int d) { return kc + ((slot / 16 * (D / 16) + d / 16) * 16 + slot % 16) * 16 + d % 16; };
    if (row) {
      const float kmul = 1.f / ks, vmul = 1.f / vs;   // exact: powers of two
      *reinterpret_cast<u32x2*>(chunk(first + r, task.a)) = pack_e4m3x8(kx, kmul);
      *reinterpret_cast<u32x2*>(chunk(first + r, task.b)) = pack_e4m3x8(ky, kmul);
      const u32x2 a = pack_e4m3x8(vx, vmul), c = pack_e4m3x8(vy, vmul);
      rows[thread] = u32x4{a[0], a[1], c[0], c[1]};
    }
    if (kratio != 1.f && r < first) {
      u32x4* o = reinterpret_cast<u32x4*>(chunk(r, 16 * (thread % kTasks)));
      u32x4 w = *o;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = rescale_e4m3x4(w[e], kratio);
      *o = w;
    }
  } else if (row) {
    uint16_t* kc = reinterpret_cast<uint16_t*>(p.k_cache) + at * (BS * D);   // 8 dims of a slot are contiguous
    st16(kc + (task.a / 8 * BS + first + r) * 8, narrow(kx));
    st16(kc + (task.b / 8 * BS + first + r) * 8, narrow(ky));
    rows[2 * thread] = va;
    rows[2 * thread + 1] = vb;
  }
  __syncthreads();

  // ---- V: each piece with its new slots put in
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const bool again = k8 && vratio != 1.f && slot[i] < first;   // it holds earlier rows of another scale
    if (!some[i] && !again) continue;
    u32x4 w = piece[i];
    if (!some[i]) w = *place[i];
    if constexpr (k8) {
      const uint8_t* in = reinterpret_cast<const uint8_t*>(rows) + dim[i];
#pragma unroll
      for (int j = 0; j < 2; ++j)       // dim, dim + 32: words 2j, 2j+1
#pragma unroll
        for (int q = 0; q < 2; ++q) {   // slots + 8 q ..
          uint32_t x = w[2 * j + q];
          if (vratio != 1.f) {
            const uint32_t y = rescale_e4m3x4(x, vratio);
#pragma unroll
            for (int e = 0; e < 4; ++e)   // only rows the sequence holds
              if (slot[i] + 8 * q + e < first) x = (x & ~(0xFFu << (8 * e))) | (y & (0xFFu << (8 * e)));
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = slot[i] + 8 * q + e - first;
            if (k >= 0 && k < m) x = (x & ~(0xFFu << (8 * e))) | ((uint32_t)in[k * D + 32 * j] << (8 * e));
          }
          w[2 * j + q] = x;
        }
    } else {
      const uint16_t* in = reinterpret_cast<const uint16_t*>(rows) + dim[i];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int k = slot[i] + (e >> 2) * 8 + (e & 3) - first;
        if (k < 0 || k >= m) continue;
        const uint32_t v = in[k * D];
        w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0x0000FFFFu) | (v << 16)) : ((w[e >> 1] & 0xFFFF0000u) | v);
      }
    }
    *place[i] = w;
  }
}

template <int D, int BS, bool k8>
__global__ __launch_bounds__((kThreads<D, BS>)) void rotate_append_kernel(RotateParams p) {
  const int w = blockIdx.x;
  if (w < p.append_groups) return append_block<D, BS, k8>(p, w / p.hkv, w % p.hkv, threadIdx.x);
  constexpr int kWaves = kThreads<D, BS> / kWave;
  const int tok = __builtin_amdgcn_readfirstlane((w - p.append_groups) * kWaves + (int)(threadIdx.x >> 6));
  if (tok < p.total_tokens) rotate_query<D>(p, tok, threadIdx.x & 63);
}

template <int D, int BS, bool k8>
static hipError_t launch_rotate_t(const RotateParams& p, hipStream_t s) {
  constexpr int kWaves = kThreads<D, BS> / kWave;
  const unsigned queries = p.q != nullptr ? ((unsigned)p.total_tokens + kWaves - 1) / kWaves : 0;
  hipLaunchKernelGGL((rotate_append_kernel<D, BS, k8>), dim3((unsigned)p.append_groups + queries), dim3(kThreads<D, BS>), 0,
                     s, p);
  return hipGetLastError();
}
template <bool k8>
static hipError_t launch_rotate_k(const RotateParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.block_size == 16 ? launch_rotate_t<128, 16, k8>(p, s) : launch_rotate_t<128, 32, k8>(p, s);
  return p.block_size == 16 ? launch_rotate_t<64, 16, k8>(p, s) : launch_rotate_t<64, 32, k8>(p, s);
}

hipError_t launch_rotate_append(RotateParams p, hipStream_t s) {
  p.append_groups = (int)rotate_append_groups(p.total_tokens, p.block_size, p.num_seqs, p.hkv);
  return p.scales != nullptr ? launch_rotate_k<true>(p, s) : launch_rotate_k<false>(p, s);
}

}  // namespace spexis
