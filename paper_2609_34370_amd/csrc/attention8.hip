// Verification attention over the cache held in 8 bits: attention.hip's work split (a head's 32-key tiles cut into
// shares, one wave a share, partials merged), on tiles of half the bytes, in which shares an item costs more than its tiles.
//
// A tile is 32 keys: two units of 16 slots, which in blocks of 16 are two blocks.  Codes come from HBM straight into
// registers, 16 bytes a lane, and are widened there to the bf16 operands of v_mfma_f32_32x32x16_bf16 by
// v_cvt_scalef32_pk_bf16_fp8, two at a time, which also applies the block's scale (a power of two: no rounding).
//   S^T[key][row] = K Q^T: lane l holds key l%32 and, of 32 dims, the 16 from 16 (l/32) on: its 16 bytes feed two
//     products, each of 8 dims of the lower and 8 of the upper half; Q's registers hold the same dims.
//   O^T[d][row] += V^T P^T: 16 bytes hold 8 slots of dims d and d + 32, the slots in the order in which a lane of the
//     score tile holds keys, so they feed the products of two head-dim tiles.
//
// Bound by the cache's bytes up to 32 query rows a head: 64 sequences of 1024 to 4096 keys (32 query heads over 8 of 128,
// 5 tokens; 357 MB) take 62 to 65 us (two cards), 5.5 to 5.8 TB/s, and 7.8 us of merge behind them.  With 33 to 64 rows by
// one wave's chain: 512 sequences of 512 to 2048 keys (63 rows, 762 MB) 154 to 158 us, 4.9 TB/s, and 18.4 us of merge.  There
// a wave lives 302 thousand cycles, 3600 for each of its 84 tiles, at about 2.1 GHz: 352 vector instructions a tile (32
// exponentials, 64 conversions of codes and 16 of weights among them) and 32 matrix products, which are busy for 28% of the
// time; for 57% of it an instruction issues, for 28% the wave waits for loads, for 15% for earlier results.  One sequence of
// 16384 keys: 13 to 15 us for 32 MB, a chain of share search, block ids, codes and products, whose partials (7.1 MB) are
// written and read again, and 6.9 us of merge.
// One wave a SIMD holds everything in registers; two (half the registers each, twice the shares and partials) took 78
// and 197 us a call where one took 71 and 180.  Three tiles in flight took 72 us instead of 71 (one row tile; two have no
// registers for a third).
#include "attention.h"

namespace spexis {

// Eight e4m3 codes times a power of two, as a matrix operand.
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return as_bf16x8(u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                         __builtin_bit_cast(uint32_t, d)});
}

// An accumulator where an item ends.  Written out because otherwise the compiler reads every accumulator into a vector
// register on every tile, for the few tiles that end an item.  The hazard checks do not look inside inline assembly:
// settle_acc(), in a basic block without an MFMA, gives an accumulator's last MFMA its 18 wait states.
__device__ __forceinline__ void settle_acc() { asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7"); }
__device__ __forceinline__ float read_acc(float a) {
  float t;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(t) : "a"(a));
  return t;
}

template <int D, int BS, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1)))
void verify_attn8_kernel(AttnParams p) {
  constexpr int KS = D / 16;   // k-steps of the score product
  constexpr int KL = D / 32;   // 16-byte loads of K: two k-steps each
  constexpr int VP = D / 64;   // pairs of head-dim tiles: a 16-byte load of V holds both
  constexpr int MT = D / 32;   // 32-wide head-dim tiles of the output
  constexpr int DEPTH = 2;     // tiles in flight
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  // Wave qw -> (share s, head h); wid = s * hkv + h names its partial slots and header.  Paired shares (skew > 0): wave
  // qw = 8m + 4 par + r takes u = 4m + r: share 2 (u / hkv) + par of head u % hkv, so the two shares of a pair run on
  // XCDs of opposite parity, and the waves of a workgroup take neighbouring heads of one share.
  const int qw = (int)blockIdx.x * 4 + wave;
  int share, h;
  if (p.skew > 0) {
    const int u = ((qw >> 3) << 2) | (qw & 3);
    share = 2 * (u / p.hkv) + ((qw >> 2) & 1);
    h = u % p.hkv;
  } else {
    share = qw / p.hkv;
    h = qw % p.hkv;
  }
  const int wid = share * p.hkv + h;
  const int64_t slot_f = attn_slot_floats(p.rmax, D);
  float* slots = p.ws + (int64_t)wid * 2 * slot_f;
  int32_t* hdr = reinterpret_cast<int32_t*>(p.ws + (int64_t)p.nwaves * 2 * slot_f) + (int64_t)wid * kAttnHdrInts;
  Share sh;   // this wave's share [g0, g0 + cnt) of head h's tile stream
  if (share >= p.nshares || !find_share(p, share, lane, sh, p.item_cost)) {
    if (lane == 0) *reinterpret_cast<u32x4*>(hdr) = u32x4{0u, 0u, 0u, 0u};
    return;
  }
  const int cnt = sh.cnt;

  // ---- loading: the tile being issued (lc, its block ids) and the next one (nc), one step ahead
  const uint8_t* kc = reinterpret_cast<const uint8_t*>(p.k_cache);
  const uint8_t* vc = reinterpret_cast<const uint8_t*>(p.v_cache);
  constexpr int64_t kHead = (int64_t)BS * D;   // bytes of one (block, head) chunk
  // Physical blocks of a tile: keys 0..15 and 16..31 (one block when BS = 32).  The second id repeats the first past
  // the sequence end; those keys are masked.
  auto tile_blocks = [&](const Cursor& c, int& ka, int& kb) {
    sint32* row = (sint32*)p.block_tables + (int64_t)c.b * p.max_blocks;
    if (BS == 16) {
      ka = clampi(row[2 * c.t], 0, p.num_blocks - 1);
      kb = clampi(row[min(2 * c.t + 1, (c.S - 1) >> 4)], 0, p.num_blocks - 1);
    } else {
      ka = kb = clampi(row[c.t], 0, p.num_blocks - 1);
    }
  };
  // An item's tiles are loaded in whole groups of DEPTH, so that every item begins in slot 0: past its last tile the
  // positions of a group load that tile again (a cache hit).
  struct Pos {
    Cursor c;
    int end, more, left;   // the item's tiles end, its loads after this one, the share's positions after those tiles
  };
  auto padded = [](int tiles) { return (tiles + DEPTH - 1) / DEPTH * DEPTH; };
  auto step = [&](Pos& x) {
    if (x.more > 0) {
      --x.more;
      if (x.c.t + 1 < x.end) ++x.c.t;
    } else if (x.left > sh.tail) {
      x.left -= sh.tail;
      x.c.t = x.c.nt - 1;
      advance(p, x.c);
      x.end = min(x.c.nt, x.left);
      x.left -= x.end;
      x.more = padded(x.end) - 1;
    }
  };
  Pos now;   // the position being issued and (next) the one after it, whose block ids are on their way
  now.c = sh.start;
  now.end = min(now.c.nt, now.c.t + cnt);
  now.left = cnt - (now.end - now.c.t);
  now.more = padded(now.end - now.c.t) - 1;
  Pos next = now;
  int la, lb, na, nb;
  step(next);
  tile_blocks(now.c, la, lb);
  tile_blocks(next.c, na, nb);

  struct Buf {
    u32x4 k[KL];
    u32x4 v[2][VP];   // [unit]
    f32x2 s;          // the scales of K and V of the unit of lane col's key
  };
  Buf buf[DEPTH];
  // Loads are issued unconditionally -- past the share's end they re-read its last tile -- so the count of
  // outstanding loads is the same on every path and waits stay partial.  The scales come by vector loads like the
  // tiles: a wait for a scalar load waits for every scalar load.
  auto get = [](const uint8_t* a) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a)); };
  auto load_tile = [&](Buf& B) {
    const int64_t ca = (int64_t)la * p.hkv + h, cb = (int64_t)lb * p.hkv + h;
    const int64_t ck = BS == 16 && col >= 16 ? cb : ca;   // lane col's key lies in unit col / 16
    const uint8_t* kp = kc + ck * kHead + (BS == 32 && col >= 16 ? 16 * D : 0) + (half * 16 + (col & 15)) * 16;
    B.s = reinterpret_cast<const f32x2*>(p.scales)[ck];
#pragma unroll
    for (int j = 0; j < KL; ++j) B.k[j] = get(kp + j * 512);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t* vp = vc + (BS == 16 && u == 1 ? cb : ca) * kHead + (BS == 32 ? u * 16 * D : 0) + (col * 2 + half) * 16;
#pragma unroll
      for (int i2 = 0; i2 < VP; ++i2) B.v[u][i2] = get(vp + i2 * 1024);
    }
    // to the next position
    now = next;
    la = na;
    lb = nb;
    step(next);
    tile_blocks(next.c, na, nb);
  };

  // ---- the item being computed and its online-softmax state
  // r / group for a row r < 64: (r * magic) >> 16 is exact, since r * (magic - 65536 / group) < 64 <= 65536 / group
  const int magic = (65536 + p.group - 1) / p.group;
  Cursor pc = sh.start;
  int q0 = 0, L = 0, R = 0, lim[NT];
  float m[NT], l[NT];
  f32x16 acc[NT][MT];
  // Q, the score product's B operand: with two row tiles, row tile 0 in this wave's part of LDS and row tile 1 in
  // registers; one row tile in registers.
  constexpr bool kQinLds = NT == 2;
  u32x4 qr[KS];
  // Each wave's KS KB of LDS: Q's row tile 0 while an item runs (two row tiles), and the scratch through which an
  // item's results are transposed at its end, so that a store instruction writes whole lines of consecutive rows.
  __shared__ u32x4 sm_q[4][KS][kWave];
  u32x4* const scr = &sm_q[wave][0][0];
  // The partial of the share's first item (its later part, which ends inside the share) waits in this wave's LDS, its
  // maxima and sums in registers, and goes to memory when the wave ends: stores in the middle of a share cost more than
  // their bytes.  Its 16-byte chunks c of row r lie at c ^ (r mod chunks): lanes hold one chunk of 32 rows.
  constexpr int kChunks = D / 4;
  __shared__ f32x4 sm_stash[4][NT * 32 * kChunks];
  float st_m[NT], st_l[NT];
  int stash_rows = 0;

  // A tile at the causal edge whose V holds NaN codes: a weight of 0 times NaN would reach the rows that do not see
  // the key.  So the codes become 0, and the rows that do see them get their NaN by two products whose factors are
  // finite: 448 * 2^118 times 2^127 overflows to infinity, and infinity minus infinity is NaN.
  auto part_nans = [&](Buf& B) {
    uint32_t some = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i2 = 0; i2 < VP; ++i2)
#pragma unroll
        for (int w = 0; w < 4; ++w) some |= ((B.v[u][i2][w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    if (__builtin_amdgcn_ballot_w64(some != 0) == 0) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        u32x4 sees;   // bf16 2^127 (0x7F00) for the keys that the lane's row sees
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int key = pc.t * 32 + 16 * u + (w >> 1) * 8 + 4 * half + 2 * (w & 1);
          sees[w] = (key <= lim[nt] ? 0x7F00u : 0u) | (key + 1 <= lim[nt] ? 0x7F000000u : 0u);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t c[2];
#pragma unroll
          for (int w = 0; w < 2; ++w)   // the code of 448 where a NaN lies
            c[w] = ((((B.v[u][mt / 2][2 * (mt % 2) + w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 0x7Eu;
          const bf16x8 big = widen8(c[0], c[1], 0x1p118f);
          acc[nt][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(big, as_bf16x8(sees), acc[nt][mt], 0, 0, 0);
          acc[nt][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(big, as_bf16x8(sees | 0x80008000u), acc[nt][mt], 0, 0, 0);
        }
      }
#pragma unroll
      for (int i2 = 0; i2 < VP; ++i2)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t nan = ((B.v[u][i2][w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
          B.v[u][i2][w] &= ~((nan >> 7) * 0xFFu);
        }
    }
  };

  // Tile pc.t of the item (not live: the position only pads the item's last group), then the load of the slot's next
  // position.
  auto process = [&](Buf& B, bool live) {
    const int t0 = pc.t * 32, S = pc.S;
    const bool need_mask = t0 + 31 > L;   // causal edge (keys >= S are past every row's limit)
    float vs[2];
    f32x16 sc[NT];
    if (live) {
      if (t0 + 32 > S) {
        // the tile runs past the sequence: zero V rows of keys >= S (they may hold anything)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            // words w and w + 2 hold the same four keys, of two head-dim tiles
            const int kbase = t0 + 16 * u + 8 * w + 4 * half;
            uint32_t keep = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) keep |= kbase + e < S ? 0xFFu << (8 * e) : 0u;
#pragma unroll
            for (int i2 = 0; i2 < VP; ++i2) {
              B.v[u][i2][w] &= keep;
              B.v[u][i2][w + 2] &= keep;
            }
          }
      }
      if (need_mask) part_nans(B);
      vs[0] = readlane_f32(B.s[1], 0);
      vs[1] = readlane_f32(B.s[1], 16);
      // both row tiles' scores first: the second's products run under the first's softmax
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[nt][e] = 0.f;
      bf16x8 kop[KS];
#pragma unroll
      for (int j = 0; j < KL; ++j) {
        kop[2 * j] = widen8(B.k[j][0], B.k[j][1], B.s[0]);
        kop[2 * j + 1] = widen8(B.k[j][2], B.k[j][3], B.s[0]);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int s = 0; s < KS; ++s)
          sc[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              kop[s], as_bf16x8(kQinLds && nt == 0 ? sm_q[wave][s][lane] : qr[s]), sc[nt], 0, 0, 0);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = sc[nt][e] * p.scale_log2e;
        if (need_mask) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = t0 + (e >> 2) * 8 + 4 * half + (e & 3);
            if (key > lim[nt]) x[e] = -INFINITY;
          }
        }
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
        mx = halves_max(mx);
        // Lazy rescaling: the reference maximum moves only when a score exceeds it by more than 2^kLazy, so 2^(x - m)
        // stays <= 2^kLazy and the accumulators are rescaled rarely.
        if (__builtin_amdgcn_ballot_w64(mx > m[nt] + kLazy) != 0) {
          const float mold = m[nt], mnew = fmaxf(mold, mx), alpha = fast_exp2(mold - mnew);
          m[nt] = mnew;
          l[nt] *= alpha;
          // a row still at kNegBig has added nothing yet: the first tile of an item scales nothing
          if (__builtin_amdgcn_ballot_w64(mold > kNegBig) != 0) scale_acc<MT>(acc[nt], alpha);
        }
        float ps = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[e] = fast_exp2(x[e] - m[nt]);
          ps += x[e];
        }
        l[nt] += ps;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          u32x4 pw;
#pragma unroll
          for (int w = 0; w < 4; ++w) pw[w] = pack_bf16x2(x[8 * u + 2 * w], x[8 * u + 2 * w + 1]);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            acc[nt][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                widen8(B.v[u][mt / 2][2 * (mt % 2)], B.v[u][mt / 2][2 * (mt % 2) + 1], vs[u]), as_bf16x8(pw), acc[nt][mt], 0,
                0, 0);
        }
      }
      ++pc.t;
    }
    load_tile(B);
  };

  // An item that this wave computed whole: normalised, bf16, row by row.  Chunk c of row col at chunk c ^ (col mod kOc)
  // of the scratch row.
  auto write_whole = [&]() {
    constexpr int kOc = D / 8;   // 16-byte chunks of an output row
    uint16_t* out = reinterpret_cast<uint16_t*>(p.out) + ((int64_t)q0 * p.hq + h * p.group) * D;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float inv = 1.0f / halves_sum(l[nt]);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const u32x2 w = {pack_bf16x2(read_acc(acc[nt][mt][4 * a]) * inv, read_acc(acc[nt][mt][4 * a + 1]) * inv),
                           pack_bf16x2(read_acc(acc[nt][mt][4 * a + 2]) * inv, read_acc(acc[nt][mt][4 * a + 3]) * inv)};
          const int c = 4 * mt + a;
          reinterpret_cast<u32x2*>(scr)[(col * kOc + (c ^ (col & (kOc - 1)))) * 2 + half] = w;
        }
      wave_lds_fence();
#pragma unroll 4
      for (int x = 0; x < 32 * kOc / kWave; ++x) {
        const int row = (x * kWave + lane) / kOc, c = lane % kOc, r = nt * 32 + row;
        const u32x4 v = scr[row * kOc + (c ^ (row & (kOc - 1)))];
        // row r is (token j, head g) with r = j * G + g: at (j * Hq + g) * D
        const int j = (r * magic) >> 16;
        if (r < R)
          __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(out + ((int64_t)j * (p.hq - p.group) + r) * D + 8 * c));
      }
      wave_lds_fence();   // the next row tile's writes follow these reads
    }
  };
  auto put4 = [](float* a, u32x4 v) {
    // two row tiles: large partials, streamed; one: the merge reads them from the caches
    if (NT == 2) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a));
    else *reinterpret_cast<u32x4*>(a) = v;
  };

  int done = 0;             // positions of the share that are done
  int at = 0, ran = 0;      // the item's first one, and its tiles in the share
  Cursor item = sh.start;   // the item, at its first tile in the share
  bool head = false;        // the share's last item is finished by a later share
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load_tile(buf[d]);
  for (;;) {
    // ---- between two items.  With one row tile the next one's Q is in flight while the last one's results are written
    // (two row tiles: there are no registers for it).
    const bool more = done < cnt;
    SeqGeo g = {0, 1, 0, 0};
    u32x4 qn[NT][KS];
    auto load_q = [&]() {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        // padding rows repeat a real row
        const int r = nt * 32 + col, rr = r < p.group * g.n ? r : p.group * g.n - 1, j = (rr * magic) >> 16;
        const uint16_t* qrow = reinterpret_cast<const uint16_t*>(p.q) +
                               ((int64_t)(g.q0 + j) * p.hq + h * p.group + rr - j * p.group) * D + 16 * half;
#pragma unroll
        for (int s = 0; s < KS; ++s) qn[nt][s] = ld16(qrow + s / 2 * 32 + s % 2 * 8);
      }
    };
    if (more) {
      g = seq_geo(p, (sint32*)p.qsl, (sint32*)p.seq_lens, pc.b);
      if (NT == 1) load_q();
    }
    if (ran > 0) {
      const bool starts_before = at == 0 && item.t != 0, ends_after = item.t + ran < item.nt;
      settle_acc();
      if (starts_before) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int lr = nt * 32 + col;
          if (lr < R) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int a = 0; a < 4; ++a)
                sm_stash[wave][lr * kChunks + ((8 * mt + 2 * a + half) ^ (lr & (kChunks - 1)))] =
                    f32x4{read_acc(acc[nt][mt][4 * a]), read_acc(acc[nt][mt][4 * a + 1]), read_acc(acc[nt][mt][4 * a + 2]),
                          read_acc(acc[nt][mt][4 * a + 3])};
          }
          st_m[nt] = m[nt];
          st_l[nt] = halves_sum(l[nt]);
        }
        stash_rows = R;
      } else if (!ends_after) {
        write_whole();
      } else {
        head = true;   // its partial stays in the accumulators
      }
    }
    if (!more) break;
    item = pc;
    at = done;
    q0 = g.q0;
    L = pc.S - g.n;
    R = p.group * g.n;
    if (NT == 2) load_q();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 32 + col, rr = r < R ? r : R - 1;
      lim[nt] = L + ((rr * magic) >> 16);   // keys 0 .. L + j are visible
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if (kQinLds && nt == 0) sm_q[wave][s][lane] = qn[nt][s];
        else qr[s] = qn[nt][s];
      }
      m[nt] = kNegBig;
      l[nt] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[nt][mt][e] = 0.f;
    }
    // Everything in flight has arrived past this point (Q was issued last): entering the loop here changes none of its
    // wait counts.
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    ran = min(cnt - done, pc.nt - pc.t);
    for (int t = 0; t < ran; t += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        process(buf[d], t + d < ran);
      }
    }
    done += ran;
    if (pc.t == pc.nt) {
      done += sh.tail;
      if (done < cnt) {
        pc.t = pc.nt - 1;
        advance(p, pc);
      }
    }
  }

  // ---- the share's last item, if a later share finishes it: its partial to slot 1, half of the head dimension at a time
  if (head) {
    constexpr int kHc = D / 8;   // 16-byte chunks of half an fp32 row
    float* slot1 = slots + slot_f;
    settle_acc();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float lt = halves_sum(l[nt]);
      const int lr = nt * 32 + col;
#pragma unroll
      for (int hm = 0; hm < 2; ++hm) {
#pragma unroll
        for (int mt = hm * MT / 2; mt < (hm + 1) * MT / 2; ++mt)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const int c = 8 * (mt - hm * MT / 2) + 2 * a + half;
            scr[col * kHc + (c ^ (col & (kHc - 1)))] =
                u32x4{__float_as_uint(read_acc(acc[nt][mt][4 * a])), __float_as_uint(read_acc(acc[nt][mt][4 * a + 1])),
                      __float_as_uint(read_acc(acc[nt][mt][4 * a + 2])), __float_as_uint(read_acc(acc[nt][mt][4 * a + 3]))};
          }
        wave_lds_fence();
#pragma unroll 4
        for (int x = 0; x < 32 * kHc / kWave; ++x) {
          const int row = (x * kWave + lane) / kHc, c = lane % kHc, r = nt * 32 + row;
          const u32x4 v = scr[row * kHc + (c ^ (row & (kHc - 1)))];
          if (r < R) put4(slot1 + (int64_t)r * D + hm * (D / 2) + 4 * c, v);
        }
        wave_lds_fence();
      }
      if (half == 0 && lr < R) {
        slot1[(int64_t)p.rmax * D + lr] = m[nt];
        slot1[(int64_t)p.rmax * D + p.rmax + lr] = lt;
      }
    }
  }
  // the stashed partial to slot 0
  if (stash_rows > 0) {
    wave_lds_fence();
#pragma unroll 4
    for (int x = lane; x < stash_rows * kChunks; x += kWave) {
      const int row = x / kChunks;
      put4(slots + 4 * (int64_t)x, __builtin_bit_cast(u32x4, sm_stash[wave][row * kChunks + ((x % kChunks) ^ (row & (kChunks - 1)))]));
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 32 + col;
      if (half == 0 && r < stash_rows) {
        slots[(int64_t)p.rmax * D + r] = st_m[nt];
        slots[(int64_t)p.rmax * D + p.rmax + r] = st_l[nt];
      }
    }
  }
  // header of the slot-1 partial: the item this wave starts and a later share finishes
  if (lane == 0) {
    *reinterpret_cast<u32x4*>(hdr) =
        u32x4{head ? 1u : 0u, (uint32_t)item.b, (uint32_t)(sh.g0 + at - item.t), (uint32_t)item.nt};
    *reinterpret_cast<u32x4*>(hdr + 4) = u32x4{(uint32_t)sh.P, (uint32_t)q0, (uint32_t)(R / p.group), (uint32_t)sh.dlt};
  }
}

template <int D, int BS, int NT>
static hipError_t launch_attn8_t(const AttnParams& p, hipStream_t s) {
  hipLaunchKernelGGL((verify_attn8_kernel<D, BS, NT>), dim3((unsigned)(p.nwaves / 4)), dim3(256), 0, s, p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_attn_merge(p, s);
}
template <int D, int BS>
static hipError_t launch_attn8_nt(const AttnParams& p, hipStream_t s) {
  return p.rmax <= 32 ? launch_attn8_t<D, BS, 1>(p, s) : launch_attn8_t<D, BS, 2>(p, s);
}

hipError_t launch_attention8(const AttnParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.block_size == 16 ? launch_attn8_nt<128, 16>(p, s) : launch_attn8_nt<128, 32>(p, s);
  return p.block_size == 16 ? launch_attn8_nt<64, 16>(p, s) : launch_attn8_nt<64, 32>(p, s);
}

}  // namespace spexis
