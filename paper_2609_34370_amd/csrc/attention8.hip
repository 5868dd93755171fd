// Verification attention over the cache held in 8 bits: attention.hip's work split (a head's 32-key tiles cut into
// equal shares, one wave a share, partials merged), on tiles of half the bytes.
//
// A tile is 32 keys: two units of 16 slots, which in blocks of 16 are two blocks.  Codes come from HBM straight into
// registers, 16 bytes a lane, and are widened there to the bf16 operands of v_mfma_f32_32x32x16_bf16 by
// v_cvt_scalef32_pk_bf16_fp8, two at a time, which also applies the block's scale (a power of two: no rounding).
//   S^T[key][row] = K Q^T: lane l holds key l%32 and, of 32 dims, the 16 from 16 (l/32) on: its 16 bytes feed two
//     products, each of 8 dims of the lower and 8 of the upper half; Q's registers hold the same dims.
//   O^T[d][row] += V^T P^T: 16 bytes hold 8 slots of dims d and d + 32, the slots in the order in which a lane of the
//     score tile holds keys, so they feed the products of two head-dim tiles.
#include "attention.h"

namespace spexis {

// Eight e4m3 codes times a power of two, as a matrix operand.
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return as_bf16x8(u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                         __builtin_bit_cast(uint32_t, d)});
}

typedef const __attribute__((address_space(4))) f32x2 sf32x2;

template <int D, int BS, int NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1)))
void verify_attn8_kernel(AttnParams p) {
  constexpr int KS = D / 16;   // k-steps of the score product
  constexpr int KL = D / 32;   // 16-byte loads of K: two k-steps each
  constexpr int VP = D / 64;   // pairs of head-dim tiles: a 16-byte load of V holds both
  constexpr int MT = D / 32;   // 32-wide head-dim tiles of the output
  // Tiles in flight: the register file of one wave per SIMD holds DEPTH operand buffers.
  constexpr int DEPTH = NT == 1 ? 5 : 3;
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  // Physical wave qw -> (share s, head h); wid = s * hkv + h names its partial slots and header.
  // Paired shares (skew > 0): workgroups alternate between the XCDs of even and odd index, and
  // wave qw = 8m + 4 par + r takes u = 4m + r: share 2 (u / hkv) + par of head u % hkv.  So the
  // two shares of each pair run on XCDs of opposite parity, and the four waves of a workgroup
  // take neighbouring heads of one share.  The host makes nwaves a multiple of 8 and of 2 hkv,
  // which makes the map a bijection of [0, nwaves).
  const int qw = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6));
  int s_, h_;
  if (p.skew > 0) {
    const int u = ((qw >> 3) << 2) | (qw & 3);
    s_ = 2 * (u / p.hkv) + ((qw >> 2) & 1);
    h_ = u % p.hkv;
  } else {
    s_ = qw / p.hkv;
    h_ = qw % p.hkv;
  }
  const int wid = s_ * p.hkv + h_;
  const int64_t slot_f = attn_slot_floats(p.rmax, D);
  float* slots = p.ws + (int64_t)wid * 2 * slot_f;
  int32_t* hdr = reinterpret_cast<int32_t*>(p.ws + (int64_t)p.nwaves * 2 * slot_f) + (int64_t)wid * kAttnHdrInts;

  auto no_share = [&]() {
    if (lane == 0) *reinterpret_cast<u32x4*>(hdr) = u32x4{0u, 0u, 0u, 0u};
  };
  const int h = h_, share = s_;
  if (share >= p.nshares) return no_share();

  Share sh;   // this wave's share [g0, g0 + cnt) of head h's tile stream
  if (!find_share(p, share, lane, sh)) return no_share();
  const int P = sh.P, dlt = sh.dlt, g0 = sh.g0, cnt = sh.cnt;
  const Cursor start = sh.start;

  const uint8_t* kc = reinterpret_cast<const uint8_t*>(p.k_cache);
  const uint8_t* vc = reinterpret_cast<const uint8_t*>(p.v_cache);
  const int64_t head_stride = (int64_t)BS * D;   // bytes of one (block, head) chunk
  // Physical blocks of a tile: keys 0..15 and 16..31 (one block when BS = 32).  The second id
  // repeats the first past the sequence end; those keys are masked.
  auto tile_blocks = [&](const Cursor& c, int& ka, int& kb) {
    sint32* row = (sint32*)p.block_tables + (int64_t)c.b * p.max_blocks;
    if (BS == 16) {
      ka = clampi(row[2 * c.t], 0, p.num_blocks - 1);
      kb = clampi(row[min(2 * c.t + 1, (c.S - 1) >> 4)], 0, p.num_blocks - 1);
    } else {
      ka = kb = clampi(row[c.t], 0, p.num_blocks - 1);
    }
  };

  // load side: the tile being issued (lc, its block ids) and the next one (nc), one step ahead
  Cursor lc = start, nc = start;
  int lidx = 0, la, lb, na = 0, nb = 0;
  // both tiles' block ids fetched together (with one tile, the next cursor is the same one)
  if (cnt > 1) advance(p, nc);
  tile_blocks(lc, la, lb);
  tile_blocks(nc, na, nb);

  // Operand buffers; DEPTH rotate so that DEPTH-1 tiles are in flight while one is computed.
  // Loads are issued unconditionally -- past the share's end they re-read its last tile (an L2
  // hit) -- so the count of outstanding loads is the same on every path and waits stay partial.
  struct Buf {
    u32x4 k[KL];
    u32x4 v[2][VP];      // [unit]
    f32x2 s[2];          // [unit] the scales of K and V
  };
  Buf buf[DEPTH];

  auto load_tile = [&](Buf& B, int i) {
    if (i < cnt && i > lidx) {
      lc = nc;
      la = na;
      lb = nb;
      lidx = i;
      if (i + 1 < cnt) {
        advance(p, nc);
        tile_blocks(nc, na, nb);
      }
    }
    // lane col's key lies in unit col / 16
    const bool second = col >= 16;
    const int64_t kblk = (int64_t)(BS == 16 && second ? lb : la) * p.hkv + h;
    const uint8_t* kp = kc + kblk * head_stride + (BS == 32 && second ? 16 * D : 0) + (half * 16 + (col & 15)) * 16;
#pragma unroll
    for (int j = 0; j < KL; ++j) B.k[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + j * 512));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t vblk = (int64_t)(BS == 16 && u == 1 ? lb : la) * p.hkv + h;
      const uint8_t* vp = vc + vblk * head_stride + (BS == 32 ? u * 16 * D : 0) + (col * 2 + half) * 16;
#pragma unroll
      for (int i2 = 0; i2 < VP; ++i2) B.v[u][i2] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + i2 * 1024));
      B.s[u] = ((sf32x2*)p.scales)[vblk];
    }
  };

  // process side: the item being computed and its online-softmax state
  Cursor pc = start;
  int q0 = 0, n = 1, L = 0, R = 0;
  bool starts_before = false;
  int head_b = 0, head_f = 0, head_nt = 0, head_q0 = 0, head_n = 0, head_flag = 0;
  int lim[NT];
  // Q, the score product's B operand, in operand order: with two row tiles, row tile 0 in this
  // wave's part of LDS and row tile 1 in registers (both in registers would not fit next to two
  // tiles' accumulators); one row tile in registers.
  constexpr bool kQinLds = NT == 2;
  u32x4 qr[kQinLds ? 1 : NT][KS];
  const int wave = threadIdx.x >> 6;
  // Each wave's KS KB of LDS: Q's row tile 0 while an item runs (two row tiles), and the scratch
  // through which an item's outputs are transposed at its end.
  __shared__ u32x4 sm_q[4][KS][kWave];
  u32x4* const scr = &sm_q[wave][0][0];
  // The partial of the share's first item (its later part, which ends inside the share) waits in
  // this wave's LDS, its maxima and sums in registers, and goes to memory when the wave ends:
  // stores issued in the middle of a share cost far more than their bytes (a timing-only copy
  // without them ran 9% faster at 20 and at 63 rows per item).  With two row tiles of 128-wide
  // heads the four waves' stashes and row tile 0 of Q fill the 160 KB of LDS exactly.
  __shared__ f32x4 sm_stash[4][NT * 32 * D / 4];
  float st_m[NT], st_l[NT];
  bool stashed = false;
  int stash_rows = 0;
  float m[NT], l[NT];
  f32x16 acc[NT][MT];

  auto begin_item = [&](int i) {
    const SeqGeo g = seq_geo(p, (sint32*)p.qsl, (sint32*)p.seq_lens, pc.b);
    q0 = g.q0;
    n = g.n;
    L = pc.S - n;
    R = p.group * n;
    starts_before = i == 0 && pc.t != 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // row r = nt*32 + col is (token j, head g) with r = j*G + g; padding rows repeat a real row
      const int r = nt * 32 + col;
      const int j = r < R ? r / p.group : n - 1;
      const int gq = r < R ? r % p.group : 0;
      lim[nt] = L + j;   // keys 0..L+j are visible
      const uint16_t* qrow = reinterpret_cast<const uint16_t*>(p.q) +
                             ((int64_t)(q0 + j) * p.hq + h * p.group + gq) * D + 16 * half;
      if (kQinLds && nt == 0) {
        u32x4 t[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) t[s] = ld16(qrow + s / 2 * 32 + s % 2 * 8);
#pragma unroll
        for (int s = 0; s < KS; ++s) sm_q[wave][s][lane] = t[s];
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) qr[kQinLds ? 0 : nt][s] = ld16(qrow + s / 2 * 32 + s % 2 * 8);
      }
      m[nt] = kNegBig;
      l[nt] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[nt][mt][e] = 0.f;
    }
    // Wait for Q here, explicitly (this drains the tiles in flight, once per item): the wait
    // counter then knows Q complete on every path, and the tile loop's waits stay partial.
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  };

  auto end_item = [&](int i) {
    const bool ends_after = pc.t < pc.nt - 1;
    const bool whole = !starts_before && !ends_after;
    if (!whole && !starts_before) {   // this wave holds the item's first tiles
      head_flag = 1;
      head_b = pc.b;
      head_f = g0 + i - pc.t;
      head_nt = pc.nt;
      head_q0 = q0;
      head_n = n;
    }
    // Outputs leave through the wave's LDS scratch, transposed, so that each store writes whole
    // 16-byte chunks of consecutive rows: stored straight from the accumulators, an instruction
    // writes 8 bytes into each of 32 rows, and a timing-only copy without the output stores ran
    // 29 us (10%) faster at 63 rows per item.  The scratch holds Q's row tile 0 during the item,
    // no longer needed here; a wave's LDS operations run in order.
    constexpr int kOc = D / 8;   // 16-byte chunks of a bf16 output row
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float lt = halves_sum(l[nt]);
      const int lr = nt * 32 + col;   // row of the item (and of the partial slot)
      if (whole) {
        // bf16 rows, chunk c of row col at chunk c ^ (col mod kOc) of the scratch row
        const float inv = 1.0f / lt;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            u32x2 w;
            w[0] = pack_bf16x2(acc[nt][mt][4 * a] * inv, acc[nt][mt][4 * a + 1] * inv);
            w[1] = pack_bf16x2(acc[nt][mt][4 * a + 2] * inv, acc[nt][mt][4 * a + 3] * inv);
            const int c = 4 * mt + a;
            reinterpret_cast<u32x2*>(scr)[(col * kOc + (c ^ (col & (kOc - 1)))) * 2 + half] = w;
            __builtin_amdgcn_sched_barrier(0);   // one chunk at a time: few registers live
          }
        wave_lds_fence();
#pragma unroll 1
        for (int q = lane; q < 32 * kOc; q += kWave) {
          const int row = q / kOc, c = q % kOc, r = nt * 32 + row;
          const u32x4 v = scr[row * kOc + (c ^ (row & (kOc - 1)))];
          if (r < R) {
            const int j = r / p.group, gq = r % p.group;
            // written once, read by a later kernel: non-temporal (1-4 us faster at workloads 2-5)
            __builtin_nontemporal_store(
                v, reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(p.out) +
                                            ((int64_t)(q0 + j) * p.hq + h * p.group + gq) * D + 8 * c));
          }
        }
        wave_lds_fence();   // the next row tile's writes, or the next item's Q, follow these reads
      } else if (starts_before) {
        if (lr < R) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int a = 0; a < 4; ++a)
              sm_stash[wave][(lr * D + 32 * mt + 8 * a + 4 * half) / 4] =
                  f32x4{acc[nt][mt][4 * a], acc[nt][mt][4 * a + 1], acc[nt][mt][4 * a + 2], acc[nt][mt][4 * a + 3]};
        }
        st_m[nt] = m[nt];
        st_l[nt] = lt;
      }
      // (an item this wave starts and a later share finishes is the share's last: its partial
      // is stored after the tile loop, from the accumulators it leaves behind)
    }
    if (starts_before) {
      stashed = true;
      stash_rows = R;
    }
  };

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

  auto process = [&](Buf& B, int i) {
    if (i >= cnt) return;   // padding past the share's end
    if (i == 0 || pc.t == 0) begin_item(i);
    const int t0 = pc.t * 32;
    const int S = pc.S;
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
    const bool need_mask = t0 + 31 > L;   // causal edge (keys >= S are past every row's limit)
    if (need_mask) part_nans(B);
    const float ks = col >= 16 ? B.s[1][0] : B.s[0][0];
    bf16x8 kop[KS];
#pragma unroll
    for (int j = 0; j < KL; ++j) {
      kop[2 * j] = widen8(B.k[j][0], B.k[j][1], ks);
      kop[2 * j + 1] = widen8(B.k[j][2], B.k[j][3], ks);
    }

#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      f32x16 sc;
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            kop[s],
            as_bf16x8(kQinLds && nt == 0 ? sm_q[wave][s][lane] : qr[kQinLds ? 0 : nt][s]),
            sc, 0, 0, 0);
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = sc[e] * p.scale_log2e;
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
      // Lazy rescaling: the reference maximum moves only when a score exceeds it by more than
      // 2^kLazy, so 2^(x - m) stays <= 2^kLazy and the accumulators are rescaled rarely.
      if (__builtin_amdgcn_ballot_w64(mx > m[nt] + kLazy) != 0) {
        const float mold = m[nt];
        const float mnew = fmaxf(mold, mx);
        const float alpha = fast_exp2(mold - mnew);
        m[nt] = mnew;
        l[nt] *= alpha;
        // a row still at kNegBig has added nothing yet (its accumulators are zero): the first tile
        // of an item moves every row's maximum and scales nothing
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
      for (int s2 = 0; s2 < 2; ++s2) {
        u32x4 pw;
#pragma unroll
        for (int w = 0; w < 4; ++w) pw[w] = pack_bf16x2(x[8 * s2 + 2 * w], x[8 * s2 + 2 * w + 1]);
        const bf16x8 pb = as_bf16x8(pw);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          acc[nt][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              widen8(B.v[s2][mt / 2][2 * (mt % 2)], B.v[s2][mt / 2][2 * (mt % 2) + 1], B.s[s2][1]), pb, acc[nt][mt], 0, 0, 0);
      }
    }
    if (pc.t == pc.nt - 1 || i == cnt - 1) end_item(i);
    if (i + 1 < cnt) advance(p, pc);
  };

  // Wait counts retire in issue order, so the loop is shaped for them: every pass runs a whole
  // group of DEPTH tiles with no exit inside it (an exit edge back to the loop head would make
  // one buffer look younger than the next, and each wait for it would drain the prefetched
  // tiles); the share is padded to a multiple of DEPTH with tiles that are loaded but skipped.
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load_tile(buf[d], d);
  for (int i = 0; i < cnt; i += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      process(buf[d], i + d);
      load_tile(buf[d], i + d + DEPTH);
    }
  }

  // The share's last item, if a later share finishes it: its partial to slot 1, through the LDS
  // scratch in two halves of the head dimension (32 rows x D/2 columns each), so that each store
  // writes 16-byte chunks of consecutive rows.  Here, past the tile loop, the transpose costs no
  // registers the loop needs (inside it, it spilled).
  // Partials are written once and read by the merge launch.  With two row tiles (33 to 64 rows:
  // large partials) they are stored non-temporally, like the outputs, so that the end of this
  // launch does not wait for them to be written back from the caches (the call 11.6 us faster at
  // 63 rows per item, 99 MB of partials); with one row tile plain stores leave the merge's reads
  // to the caches (at 20 rows per item the merge ran 6.0 against 7.6 us, the call 1 us faster).
  auto put4 = [](float* a, u32x4 v) {
    if (NT == 2) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a));
    else *reinterpret_cast<u32x4*>(a) = v;
  };
  auto put1 = [](float* a, float v) {
    if (NT == 2) __builtin_nontemporal_store(v, a);
    else *a = v;
  };
  if (head_flag) {
    constexpr int kHc = D / 8;   // 16-byte chunks of half an fp32 row
    float* slot1 = slots + slot_f;
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
                u32x4{__float_as_uint(acc[nt][mt][4 * a]), __float_as_uint(acc[nt][mt][4 * a + 1]),
                      __float_as_uint(acc[nt][mt][4 * a + 2]), __float_as_uint(acc[nt][mt][4 * a + 3])};
          }
        wave_lds_fence();
        for (int q = lane; q < 32 * kHc; q += kWave) {
          const int row = q / kHc, c = q % kHc, r = nt * 32 + row;
          const u32x4 v = scr[row * kHc + (c ^ (row & (kHc - 1)))];
          if (r < R) put4(slot1 + (int64_t)r * D + hm * (D / 2) + 4 * c, v);
        }
        wave_lds_fence();
      }
      if (half == 0 && lr < R) {
        put1(slot1 + (int64_t)p.rmax * D + lr, m[nt]);
        put1(slot1 + (int64_t)p.rmax * D + p.rmax + lr, lt);
      }
    }
  }

  // the stashed partial to slot 0, 16 bytes per lane and step, stored as above (the wave's own
  // LDS writes are complete before its reads).  (Issued instead right after the share's last tile load, so that
  // the stores drain under the last tiles' compute, it needed the loop split in two, and the
  // kernel ran slower.)
  if (stashed) {
    wave_lds_fence();
    for (int idx = lane; idx < stash_rows * D / 4; idx += kWave)
      put4(slots + 4 * (int64_t)idx, __builtin_bit_cast(u32x4, sm_stash[wave][idx]));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 32 + col;
      if (half == 0 && r < stash_rows) {
        put1(slots + (int64_t)p.rmax * D + r, st_m[nt]);
        put1(slots + (int64_t)p.rmax * D + p.rmax + r, st_l[nt]);
      }
    }
  }

  // header of the slot-1 partial: the item this wave starts and a later share finishes
  if (lane == 0) {
    *reinterpret_cast<u32x4*>(hdr) = u32x4{(uint32_t)head_flag, (uint32_t)head_b, (uint32_t)head_f, (uint32_t)head_nt};
    *reinterpret_cast<u32x4*>(hdr + 4) = u32x4{(uint32_t)P, (uint32_t)head_q0, (uint32_t)head_n, (uint32_t)dlt};
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
