// What the attention over the bf16 cache and the one over the 8-bit cache share: the stream of 32-key tiles, its
// shares, and the lane exchanges of the online softmax.
#pragma once

#include "common.h"
#include "kernels.h"

namespace spexis {

// Lane l and lane l ^ 32 combined, in one cross-half lane swap (v_permlane32_swap): the swap of a
// value with itself leaves the lower half's value in the first result and the upper half's in the
// second, in every lane.
__device__ __forceinline__ float halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

constexpr float kNegBig = -1.0e30f;   // finite "minus infinity" of the running maxima

// acc[mt] *= alpha (alpha per lane: the lane's query row), in place on the registers that hold the
// accumulators.  Written out because otherwise the compiler keeps a second copy of every
// accumulator in vector registers, refreshed by one v_accvgpr_read per accumulator on every tile,
// for the rare tiles that take this path.  The hazard checks do not look inside inline assembly:
// the leading s_nops give an accumulator's last MFMA its 18+ wait states before the first read
// (this is its own basic block, so no MFMA is scheduled in between), the trailing one covers the
// last write before the next MFMA reads it as its C operand.
template <int MT>
__device__ __forceinline__ void scale_acc(f32x16 (&acc)[MT], float alpha) {
  asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7");
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = acc[mt][e], t;
      asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1"
                   : "+a"(v), "=&v"(t)
                   : "v"(alpha));
      acc[mt][e] = v;
    }
  asm volatile("s_nop 4");
}
constexpr float kLazy = 8.0f;         // base-2 headroom before the running maximum moves
constexpr int kWaitVmcnt0 = 0x0F70;   // s_waitcnt operand: vmcnt(0), expcnt and lgkmcnt not waited

// Read-only view of an int32 array: loads through it at wave-uniform addresses become scalar
// loads, counted apart from the vector loads of the tiles.
typedef const __attribute__((address_space(4))) int32_t sint32;

struct SeqGeo {
  int q0, n, S, nt;   // first query token, query tokens, keys, 32-key tiles (0: no query)
};

// Geometry of sequence b, clamped so that every address derived from it stays in its buffer.
template <typename Ptr>
__device__ __forceinline__ SeqGeo seq_geo(const AttnParams& p, Ptr qsl, Ptr seq_lens, int b) {
  SeqGeo g;
  g.q0 = clampi(qsl[b], 0, p.total_tokens);
  const int q1 = clampi(qsl[b + 1], g.q0, p.total_tokens);
  g.n = min(q1 - g.q0, p.rmax / p.group);
  g.S = clampi(seq_lens[b], max(g.n, 1), p.max_blocks * p.block_size);
  g.nt = g.n >= 1 ? (g.S + 31) >> 5 : 0;
  return g;
}

// Position in a head's tile stream: sequence, tile of the sequence, and the sequence's size.
struct Cursor {
  int b, t, nt, S;
};

__device__ __forceinline__ void advance(const AttnParams& p, Cursor& c) {
  if (++c.t < c.nt) return;
  c.t = 0;
  SeqGeo g;
  do {
    if (c.b + 1 >= p.num_seqs) return;   // never past the stream's end; stay on a valid item
    ++c.b;
    g = seq_geo(p, (sint32*)p.qsl, (sint32*)p.seq_lens, c.b);
  } while (g.nt == 0);
  c.nt = g.nt;
  c.S = g.S;
}

// Share geometry of a head's tile stream: shares pair up, shares 2j and 2j+1 covering tiles
// [2jP, 2(j+1)P), the first (the wave on an even XCD) P + dlt of them and the second P - dlt.
// dlt = 0 gives equal shares of P.
__device__ __forceinline__ int share_delta(int P, int skew) { return (int)(((int64_t)P * skew) >> 10); }
__device__ __forceinline__ int64_t share_first(int s, int P, int dlt) {
  return (int64_t)(s >> 1) * 2 * P + (s & 1) * (P + dlt);
}
__device__ __forceinline__ int share_size(int s, int P, int dlt) { return (s & 1) ? P - dlt : P + dlt; }
__device__ __forceinline__ int share_of(int g, int P, int dlt) {
  const int j = g / (2 * P);
  return 2 * j + (g - 2 * P * j >= P + dlt ? 1 : 0);
}

// A share of a head's stream of positions: [g0, g0 + cnt), where it starts, and the geometry it was cut by.  A position is
// a tile, or one of the `tail` positions behind every sequence's last tile, which stand for what an item costs besides
// its tiles; the share starts at a tile.
struct Share {
  int P, dlt, g0, cnt, tail;   // the positions of a share (paired: P + dlt and P - dlt)
  Cursor start;
};

// Share `share` of a head (the same for all of a wave's lanes); false where it holds no tile.  tail: what an
// item costs, in tiles.
__device__ __forceinline__ bool find_share(const AttnParams& p, int share, int lane, Share& o, int tail) {
  int total, P, b0 = 0, f0 = 0;   // P: the positions of a share
  Cursor start;
  if (p.num_seqs <= kWave) {
    // one pass: lane b holds sequence b's geometry; the share start is read from the lanes
    const SeqGeo gl = lane < p.num_seqs ? seq_geo(p, p.qsl, p.seq_lens, lane) : SeqGeo{0, 0, 0, 0};
    const uint64_t some = __builtin_amdgcn_ballot_w64(gl.nt > 0);   // the sequences with tiles, and those before a lane's
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0));
    const int scan = wave_incl_scan_i32(gl.nt, lane), tiles = __builtin_amdgcn_readlane(scan, kWave - 1);
    const int size = gl.nt > 0 ? gl.nt + tail : 0, incl = scan + tail * (before + (gl.nt > 0 ? 1 : 0));
    total = tiles + tail * (int)__popcll(some);   // < 2^31 (host)
    P = attn_share_positions(p.least, tiles, (int)__popcll(some), tail, p.nshares);
    if (share_first(share, P, share_delta(P, p.skew)) >= total) return false;
    const int g0 = (int)share_first(share, P, share_delta(P, p.skew));
    const uint64_t hit = __builtin_amdgcn_ballot_w64(incl > g0);
    if (hit == 0) return false;
    const int l0 = __builtin_ctzll(hit);
    b0 = l0;
    f0 = __builtin_amdgcn_readlane(incl - size, l0);
    start.b = b0;
    start.nt = __builtin_amdgcn_readlane(gl.nt, l0);
    start.S = __builtin_amdgcn_readlane(gl.S, l0);
    start.t = g0 - f0;
  } else {
    // 512 sequences at a time, eight a lane whose loads are in flight together (the bf16 kernel against a search of 64 at a
    // time: 512 sequences of 20 to 200 keys 17.5 us for 19.8, 64-wide, 74.3 for 76.9, 128-wide; from 65 to 150 the same)
    constexpr int kAhead = 8;
    int nt[kAhead];
    const auto sizes = [&](int base) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int b = base + k * kWave + lane;
        nt[k] = seq_geo(p, p.qsl, p.seq_lens, min(b, p.num_seqs - 1)).nt;
        if (b >= p.num_seqs) nt[k] = 0;
      }
    };
    int per_lane = 0, items = 0;
    for (int base = 0; base < p.num_seqs; base += kAhead * kWave) {
      sizes(base);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        per_lane += nt[k];
        items += (int)__popcll(__builtin_amdgcn_ballot_w64(nt[k] > 0));
      }
    }
    const int tiles = __builtin_amdgcn_readfirstlane(wave_sum_i32(per_lane));
    total = tiles + tail * items;   // < 2^31 (host)
    P = attn_share_positions(p.least, tiles, items, tail, p.nshares);
    if (share_first(share, P, share_delta(P, p.skew)) >= total) return false;
    const int g0 = (int)share_first(share, P, share_delta(P, p.skew));
    // the sequence holding position g0, and the stream index of its first tile
    int before = 0;
    bool found = false;
    for (int base = 0; base < p.num_seqs && !found; base += kAhead * kWave) {
      if (p.num_seqs > kAhead * kWave) sizes(base);   // else they are still there
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (found) continue;
        const int size = nt[k] > 0 ? nt[k] + tail : 0, incl = wave_incl_scan_i32(size, lane);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(before + incl > g0);
        if (hit != 0) {
          const int l0 = __builtin_ctzll(hit);
          b0 = base + k * kWave + l0;
          f0 = before + __builtin_amdgcn_readlane(incl - size, l0);
          found = true;
        } else {
          before += __builtin_amdgcn_readlane(incl, kWave - 1);
        }
      }
    }
    b0 = __builtin_amdgcn_readfirstlane(b0);
    f0 = __builtin_amdgcn_readfirstlane(f0);
    const SeqGeo g = seq_geo(p, (sint32*)p.qsl, (sint32*)p.seq_lens, b0);
    if (g.nt == 0 || g0 < f0 || g0 - f0 >= g.nt + tail) return false;   // inputs changed under us
    start.b = b0;
    start.nt = g.nt;
    start.S = g.S;
    start.t = g0 - f0;
  }
  const int dlt = share_delta(P, p.skew);
  int g0 = (int)share_first(share, P, dlt), cnt = min(share_size(share, P, dlt), total - g0);
  if (tail > 0 && start.t >= start.nt) {   // it starts behind a sequence's tiles: with the next one
    const int skip = start.nt + tail - start.t;
    if (skip >= cnt) return false;
    g0 += skip;
    cnt -= skip;
    start.t = start.nt - 1;
    advance(p, start);
  }
  o = {P, dlt, g0, cnt, tail, start};
  return true;
}

}  // namespace spexis
