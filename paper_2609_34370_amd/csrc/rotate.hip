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
// floor(n / bs) + 2 blocks, which start(b+1) - start(b) is never below, so no scan over the lengths is needed: a
// wave-wide search for the last b with start(b) <= index, two probes for 4096 sequences.  Where the sequences are of
// about one length (a step's drafts), every one gets the blocks of the longest, without the search.
//
// Measured (reads and writes of 5.3 TB/s are what a large copy reaches): q and keys of 14420 prompt tokens (28 + 4 heads
// of 128) into the bf16 cache 48.5 us, 5.5 TB/s with what the last-level cache holds; of 15060 (32 + 8) into the 8-bit
// cache 58 us, 5.9 TB/s; a step of 512 sequences of 9 rows in 8 bits 19.5 us, 4.2 TB/s.  A step of 64 sequences is a
// launch and two dependent loads, 5.6 us.  (Figures below: the whole call in a replayed graph, on three sets of buffers in
// turn.)
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
  // widened here, pair by pair (no instruction; the compiler would widen a whole task first, 64 more registers)
  if constexpr (sizeof(T) == 8) asm volatile("" : "+v"(a), "+v"(b), "+v"(c), "+v"(s));
  const T x = a, y = b, cc = c, ss = s;
  a = (float)(x * cc - y * ss);
  b = (float)(y * cc + x * ss);
}
// A task's elements as pairs (x[i], y[i]), and back.  Halves: x is chunk a, y chunk b; pairs: x the even elements, y the
// odd ones.
__device__ __forceinline__ void to_pairs(const RotateParams& p, u32x4 a, u32x4 b, float (&x)[8], float (&y)[8]) {
  if (p.style == 0) {
    widen(a, x);
    widen(b, y);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = i < 4 ? a[i] : b[i - 4];
    x[i] = __uint_as_float(w << 16);
    y[i] = __uint_as_float(w & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void from_pairs(const RotateParams& p, float (&x)[8], float (&y)[8]) {
  if (p.style == 0) return;
  const float a[8] = {x[0], y[0], x[1], y[1], x[2], y[2], x[3], y[3]}, b[8] = {x[4], y[4], x[5], y[5], x[6], y[6], x[7], y[7]};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = a[i];
    y[i] = b[i];
  }
}
// Chunks a and b turned: x and y are theirs.
template <typename T>
__device__ __forceinline__ void turn_task(const RotateParams& p, const Task& t, const Angles& g, u32x4 a, u32x4 b, float (&x)[8],
                                          float (&y)[8]) {
  to_pairs(p, a, b, x, y);
  if (t.turns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn<T>(x[i], y[i], g.c[i], g.s[i]);
  }
  from_pairs(p, x, y);
}

// q of one token, every head, one wave: the lanes are (head, task), so the token's angles are loaded once; the rows are
// in flight while the position is looked up.
template <int D, bool kStream>
__device__ __forceinline__ void rotate_query(const RotateParams& p, int index, int lane) {
  constexpr int kTasks = D / 16, kHeads = kWave / kTasks, kAhead = 2;
  const Task task = row_task(p, lane % kTasks);
  int tok = index, s = 0, q1 = 0;
  if (p.seq_tokens > 0) {   // token index % seq_tokens of sequence index / seq_tokens
    s = index / p.seq_tokens;
    q1 = clampi(p.qsl[s + 1], 0, p.total_tokens);
    tok = seq_start(p, s) + index % p.seq_tokens;
    if (tok >= q1) return;
  } else if (tok >= clampi(p.qsl[p.num_seqs], 0, p.total_tokens)) {
    return;   // a row behind the last sequence: left as it is
  }
  const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + (int64_t)tok * p.hq * D;
  uint16_t* o = reinterpret_cast<uint16_t*>(p.q_out) + (int64_t)tok * p.hq * D;
  u32x4 a[kAhead], b[kAhead];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = min(h0 + i * kHeads, p.hq - 1);
      const u32x4* pa = reinterpret_cast<const u32x4*>(q + h * D + task.a);
      const u32x4* pb = reinterpret_cast<const u32x4*>(q + h * D + task.b);
      a[i] = kStream ? __builtin_nontemporal_load(pa) : *pa;
      b[i] = kStream ? __builtin_nontemporal_load(pb) : *pb;
    }
  };
  load(lane / kTasks);
  int pos = 0;
  if (p.positions != nullptr) {
    pos = p.positions[tok];
  } else {
    if (p.seq_tokens == 0) {
      s = wave_search(p.num_seqs, tok, lane, [&](int i) { return seq_start(p, i); });
      q1 = clampi(p.qsl[s + 1], 0, p.total_tokens);
    }
    pos = p.seq_lens[s] - (q1 - tok);
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
      turn_task<float>(p, task, g, a[i], b[i], x, y);
      // written once, read by a later launch (512 sequences of 9 rows, 8 bits, 19.8 us, plain stores 23.3; 14420 prompt
      // tokens, bf16, 49.7 and 52.7)
      __builtin_nontemporal_store(narrow(x), reinterpret_cast<u32x4*>(o + h * D + task.a));
      __builtin_nontemporal_store(narrow(y), reinterpret_cast<u32x4*>(o + h * D + task.b));
    }
  }
}

// Four values of at most 448 to e4m3 codes, to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ u32x2 pack_e4m3x8(const float (&x)[8], float mul) {
  return u32x2{pack_e4m3x4(x[0] * mul, x[1] * mul, x[2] * mul, x[3] * mul),
               pack_e4m3x4(x[4] * mul, x[5] * mul, x[6] * mul, x[7] * mul)};
}
// Four codes whose scale changes by the factor r; a NaN becomes 0x7f.
__device__ __forceinline__ uint32_t rescale_e4m3x4(uint32_t w, float r) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const uint32_t nan = ((((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xFFu;
  return (pack_e4m3x4(lo[0] * r, lo[1] * r, hi[0] * r, hi[1] * r) & ~nan) | (nan & 0x7F7F7F7Fu);
}
// The largest magnitude that is stored, 240 * 2^120: values beyond it (the largest bf16 is 255 * 2^120) would round up
// to the code of 256, and 256 * 2^120 is infinity in bf16, where the attention widens codes.
constexpr uint32_t kMostBits = 0x7F700000u;
__device__ __forceinline__ void limit_finite(float (&x)[8]) {
  const float most = __uint_as_float(kMostBits);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (fabsf(x[e]) < __builtin_inff()) x[e] = fminf(fmaxf(x[e], -most), most);
}
// The format has no infinity: what is not finite is stored as the NaN 0x7f, written over the conversion's result.
__device__ __forceinline__ void store_nans(const float (&x)[8], uint8_t* codes, int step) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (!(fabsf(x[e]) < __builtin_inff())) codes[e * step] = 0x7F;
}

// The exponent of the least power of two, from 2^-100, by which `most` is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ int least_exp(uint32_t u) {   // most's bits
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, -100);
}
__device__ __forceinline__ float exp_float(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

constexpr uint32_t kInf = 0x7F800000u;
// The largest magnitude of 16 values as bits, from kInf up if one is not finite; and the largest of the finite ones.
__device__ __forceinline__ uint32_t most_bits(const float (&x)[8], const float (&y)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, max(__float_as_uint(x[i]) & 0x7FFFFFFFu, __float_as_uint(y[i]) & 0x7FFFFFFFu));
  return m;
}
__device__ __forceinline__ uint32_t most_finite_bits(const float (&x)[8], const float (&y)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu, b = __float_as_uint(y[i]) & 0x7FFFFFFFu;
    m = max(m, max(a < kInf ? a : 0u, b < kInf ? b : 0u));
  }
  return m;
}
// The same of one wave's 16 bf16 values a lane, without widening them: the largest 15-bit pattern.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t most_bits_bf16(u32x4 a, u32x4 b) {
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, a[i] & 0x7FFF7FFFu));
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, b[i] & 0x7FFF7FFFu));
  }
  return (uint32_t)max(m[0], m[1]) << 16;
}

// Ones in the bytes of the values (of kBytes each) k with lo <= k < hi, of a word that holds values 0 ...
template <int kBytes>
__device__ __forceinline__ uint32_t value_mask(int lo, int hi) {
  constexpr int kValues = 4 / kBytes;
  auto below = [](int n) { return n <= 0 ? 0u : n >= kValues ? 0xFFFFFFFFu : (1u << (8 * kBytes * n)) - 1u; };
  return below(hi) & ~below(lo);
}

// A workgroup is a (block of tokens, KV head); a thread takes one task of K and of V.
template <int D, int BS>
constexpr int kThreads = BS * D / 16;

// The new rows of one (block of tokens, KV head).
template <int D, int BS, bool k8>
__device__ __forceinline__ void append_block(const RotateParams& p, int index, int h, int thread) {
  constexpr int kTasks = D / 16, kWaves = kThreads<D, BS> / kWave;
  const int lane = thread & 63, wave = thread >> 6;
  const int b = p.seq_blocks > 0 ? rotate_block(index, p.num_seqs).seq
                                 : wave_search(p.num_seqs, index, lane, [&](int i) { return seq_start(p, i) / BS + 2 * i; });
  const int q0 = seq_start(p, b), q1 = clampi(p.qsl[b + 1], q0, p.total_tokens);
  const int cap = p.max_blocks * BS;
  const int n = min(min(q1 - q0, p.max_query_len), cap), S = clampi(p.seq_lens[b], n, cap), L = S - n;
  const int t = L / BS + (p.seq_blocks > 0 ? rotate_block(index, p.num_seqs).nth : index - (q0 / BS + 2 * b));
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

  // V's new rows as they will lie in the cache: piece c at image[c], the thread's 16 dims at places 32 bytes apart
  constexpr int kBytes = k8 ? 1 : 2;
  __shared__ u32x4 image[BS * D * kBytes / 16];
  const int at_slot = first + r, us = at_slot & 15, pos = (us >> 3) * 4 + (us & 3), t16 = thread % kTasks;
  uint8_t* mine = reinterpret_cast<uint8_t*>(image) +
                  (k8 ? (at_slot >> 4) * 16 * D + ((t16 >> 2) * 32 + (t16 & 1) * 16) * 32 + (t16 >> 1 & 1) * 8
                      : (at_slot >> 4) * 32 * D + t16 * 16 * 32) +
                  (us >> 2 & 1) * 16 + pos * kBytes;
  float kx[8], ky[8];
  if (row) turn_task<std::conditional_t<k8, double, float>>(p, task, g, ka, kb, kx, ky);
  float kratio = 1.f, vratio = 1.f;
  if constexpr (k8) {
    uint32_t kmost = row ? most_bits(kx, ky) : 0u, vmost = row ? most_bits_bf16(va, vb) : 0u;
    const bool usual = __builtin_amdgcn_ballot_w64(kmost > kMostBits || vmost > kMostBits) == 0;   // the wave's values
    if (!usual && row) {
      limit_finite(kx);
      limit_finite(ky);
      float vx[8], vy[8];
      widen(va, vx);
      widen(vb, vy);
      kmost = most_finite_bits(kx, ky);
      vmost = most_finite_bits(vx, vy);
    }
    kmost = __float_as_uint(wave_max(__uint_as_float(kmost)));
    vmost = __float_as_uint(wave_max(__uint_as_float(vmost)));
    if constexpr (kWaves > 1) {
      __shared__ u32x2 most[kWaves];
      if (lane == 0) most[wave] = u32x2{kmost, vmost};
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        kmost = max(kmost, most[w][0]);
        vmost = max(vmost, most[w][1]);
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
      *reinterpret_cast<u32x2*>(chunk(at_slot, task.a)) = pack_e4m3x8(kx, kmul);
      *reinterpret_cast<u32x2*>(chunk(at_slot, task.b)) = pack_e4m3x8(ky, kmul);
      if (!usual) {
        store_nans(kx, chunk(at_slot, task.a), 1);
        store_nans(ky, chunk(at_slot, task.b), 1);
      }
      auto values = [&](u32x4 v, uint8_t* to) {
        float x[8];
        widen(v, x);
        if (!usual) limit_finite(x);
        const u32x2 c = pack_e4m3x8(x, vmul);
#pragma unroll
        for (int e = 0; e < 8; ++e) to[32 * e] = (uint8_t)(c[e / 4] >> (8 * (e % 4)));
        if (!usual) store_nans(x, to, 32);
      };
      values(va, mine);
      values(vb, mine + 8 * 32);
    }
    if (kratio != 1.f && r < first) {
      u32x4* o = reinterpret_cast<u32x4*>(chunk(r, 16 * t16));
      u32x4 w = *o;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = rescale_e4m3x4(w[e], kratio);
      *o = w;
    }
  } else if (row) {
    uint16_t* kc = reinterpret_cast<uint16_t*>(p.k_cache) + at * (BS * D);   // 8 dims of a slot are contiguous
    st16(kc + (task.a / 8 * BS + at_slot) * 8, narrow(kx));
    st16(kc + (task.b / 8 * BS + at_slot) * 8, narrow(ky));
#pragma unroll
    for (int e = 0; e < 16; ++e)
      *reinterpret_cast<uint16_t*>(mine + 32 * e) = (uint16_t)((e < 8 ? va[e / 2] : vb[e / 2 - 4]) >> (16 * (e % 2)));
  }
  __syncthreads();

  // ---- V: each piece with its new slots put in
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const bool again = k8 && vratio != 1.f && slot[i] < first;   // it holds earlier rows of another scale
    if (!some[i] && !again) continue;
    u32x4 w = piece[i];
    if (k8 && !some[i]) w = *place[i];
    const u32x4 in = image[thread + i * kThreads<D, BS>];
    if constexpr (k8) {
      // words q and q + 2: slots + 8 q .. + 8 q + 3 of dim and of dim + 32
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int s0 = slot[i] + 8 * q;
        if (vratio != 1.f) {
          const uint32_t held = value_mask<1>(0, first - s0);   // only rows the sequence holds
          w[q] = (w[q] & ~held) | (rescale_e4m3x4(w[q], vratio) & held);
          w[q + 2] = (w[q + 2] & ~held) | (rescale_e4m3x4(w[q + 2], vratio) & held);
        }
        const uint32_t fresh = value_mask<1>(first - s0, first + m - s0);
        w[q] = (w[q] & ~fresh) | (in[q] & fresh);
        w[q + 2] = (w[q + 2] & ~fresh) | (in[q + 2] & fresh);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {   // slots s0, s0 + 1
        const int s0 = slot[i] + q / 2 * 8 + q % 2 * 2;
        const uint32_t fresh = value_mask<2>(first - s0, first + m - s0);
        w[q] = (w[q] & ~fresh) | (in[q] & fresh);
      }
    }
    // whole lines of new slots in the 8-bit cache: 15060 prompt tokens 58.8 us, plain stores 62.1 (bf16, where a piece is
    // part of a line: 14420 49.7, streamed 52.8)
    if constexpr (k8) __builtin_nontemporal_store(w, place[i]);
    else *place[i] = w;
  }
}

// 8 bits, 128-wide heads: appends and queries alternate: appends compute and wait for one load after the other, queries keep
// the memory busy meanwhile (28 + 4 heads: 512 sequences of 9 rows 19.8 us, appends first 22.7; 15060 prompt tokens, 32 + 8
// heads, 58.8 and 61.1; below 50 MB the order decides less and rather for appends first: 512 of 5 17.9 and 17.3, 64 of 5 5.8
// and 5.4, 128 of 5 7.9 and 6.9).  Appends of 64-wide heads are one wave each and as short as the queries: first (512 of 9,
// 8 + 2 heads, 7.5 us, alternating 11.6; 14420 prompt tokens 12.0 and 15.2).  bf16 appends are as bound by memory as queries
// and come first, too (512 of 5 18.9 us, alternating 22.2; 128 of 5 7.3 and 8.9; but 14420 prompt tokens 49.7 and 46.2).
template <int D, bool k8>
constexpr bool kAlternate = k8 && D == 128;

template <int D, int BS, bool k8>
__global__ __launch_bounds__((kThreads<D, BS>)) void rotate_append_kernel(RotateParams p) {
  constexpr int kWaves = kThreads<D, BS> / kWave;
  const RotatePlace place = rotate_place(blockIdx.x, kAlternate<D, k8> ? p.mix : 0, p.append_groups);
  if (place.append) {
    if (place.index < p.append_groups) append_block<D, BS, k8>(p, place.index / p.hkv, place.index % p.hkv, threadIdx.x);
    return;
  }
  const int query = __builtin_amdgcn_readfirstlane(place.index * kWaves + (int)(threadIdx.x >> 6));
  if (query >= p.queries) return;
  if (p.stream_q) rotate_query<D, true>(p, query, threadIdx.x & 63);
  else rotate_query<D, false>(p, query, threadIdx.x & 63);
}

template <int D, int BS, bool k8>
static hipError_t launch_rotate_t(RotateParams p, hipStream_t s) {
  constexpr int kWaves = kThreads<D, BS> / kWave;
  const int64_t queries = ((int64_t)p.queries + kWaves - 1) / kWaves;
  const int64_t groups = rotate_groups(p.append_groups, queries, kAlternate<D, k8>, &p.mix);
  hipLaunchKernelGGL((rotate_append_kernel<D, BS, k8>), dim3((unsigned)groups), dim3(kThreads<D, BS>), 0, s, p);
  return hipGetLastError();
}
template <bool k8>
static hipError_t launch_rotate_k(const RotateParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.block_size == 16 ? launch_rotate_t<128, 16, k8>(p, s) : launch_rotate_t<128, 32, k8>(p, s);
  return p.block_size == 16 ? launch_rotate_t<64, 16, k8>(p, s) : launch_rotate_t<64, 32, k8>(p, s);
}

hipError_t launch_rotate_append(RotateParams p, hipStream_t s) {
  const int64_t B = p.num_seqs, T = p.total_tokens, bs = p.block_size, n = p.max_query_len;
  // Sequences of about one length need no search: the longest one's blocks for each, where that is no more (512 sequences
  // of 9 rows, 8 bits, 19.8 us, by search 22.4; of one 11.7 and 15.5; of 5, bf16, 18.9 and 20.4), and its tokens where at
  // most half of the waves find none in a step (512 of 1 to 9, 8 bits, 17.4 us, by search 20.6; of 9, 64-wide, bf16, 7.2 and
  // 8.3), a fifth among prompts, whose search costs less (8 of 100 to 1000 20.8 us, by search 19.3).
  const int64_t blocks = B * ((n + bs - 2) / bs + 1), all = T / bs + 2 * B;
  p.seq_blocks = blocks <= all ? (int)((n + bs - 2) / bs + 1) : 0;
  p.append_groups = (int)((blocks <= all ? blocks : all) * p.hkv);
  const bool step = n <= 64 && T <= 1 << 20 && (int64_t)p.append_groups * p.head_dim * bs / 16 <= 1 << 30;   // far from a launch's limit
  p.seq_tokens = (step ? 5 : 8) * B * n <= 10 * T ? (int)n : 0;
  // q beyond 64 MB does not come from the caches: loads that leave the rest in them (prompts, 103 MB of q, 8 bits, the
  // call 45.9 us, plain loads 51.9); below that, it may (21 MB: 20.3, streamed 26.0)
  p.stream_q = T * p.hq * p.head_dim * 2 > (int64_t)1 << 26;
  p.queries = p.q == nullptr ? 0 : p.seq_tokens > 0 ? (int)(B * n) : (int)T;
  return p.scales != nullptr ? launch_rotate_k<true>(p, s) : launch_rotate_k<false>(p, s);
}

}  // namespace spexis
