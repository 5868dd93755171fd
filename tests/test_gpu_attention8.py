"""Attention over the 8-bit cache against its 64-bit form.

The tolerance of an output element, with A the weighted mean of |v| (the weights sum to 1):
  * every weight is rounded to bf16 (2^-8 of it) in front of the product with V, the sum of the weights is not: 2^-8 A;
  * a score is an fp32 sum of D exact products and three more roundings; its error e = (D + 4) 2^-24 max_t sum |q k|
    scale moves a weight by e times itself, in the output and in the sum: 2 e A; exp2 and the merge of shares add a few
    units of 2^-24 each, counted as 32 * 2^-24 A; sums of S terms in fp32, one after the other at worst: 2 S 2^-24 A;
  * the output is rounded to bf16: 2^-8 |o|.
"""
import sys

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import spexis as sx
from tests.test_gpu_rotate import batch, dev

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def cache(blocks, bs, hkv, D, r, wild=True):
    """Logical codes, scales and the flat pools.  Codes of all sizes but NaN (wild), or of about N(0, 1)."""
    if wild:
        codes = [(r.integers(0, 2, s) * 128 + r.integers(0, 127, s)).astype(np.uint8) for s in [(blocks, bs, hkv, D)] * 2]
        scales = np.exp2(r.integers(-9, -6, (blocks, hkv, 2))).astype(np.float32)
    else:
        codes = [osv.encode(64 * r.standard_normal((blocks, bs, hkv, D))) for _ in range(2)]
        scales = np.exp2(r.integers(-7, -5, (blocks, hkv, 2))).astype(np.float32)
    return codes, scales


def pools(codes, bs):
    blocks, _, hkv, D = codes[0].shape
    out = []
    for c, p in zip(codes, osv.places8(blocks, hkv, bs, D)):
        flat = np.zeros(c.size, np.uint8)
        flat[p] = c
        out.append(dev(flat).view(torch.float8_e4m3fn))
    return out


def attend(pool, scales, blocks, hkv, bs, D, qsl, S, tables, q, scale, chunk=0, stream=None):
    T, hq = q.shape[:2]
    most = int(np.diff(qsl).max())
    ws = sx.spexis_verify_attention_kv8_workspace_size(len(S), hq, hkv, D, most, int(S.max()), chunk)
    out = torch.full_like(q, 777.0)
    sx.spexis_verify_attention_kv8(*pool, scales, blocks, hkv, bs, D, dev(qsl), dev(S), dev(tables), T, most, int(S.max()), q,
                                   hq, scale, out, torch.empty(max(ws, 16), dtype=torch.uint8, device="cuda"),
                                   kv_chunk_tokens=chunk, stream=stream)
    torch.cuda.synchronize()
    return out


def check(got, codes, scales, qsl, S, tables, q, scale):
    ref, mean, most = osv.attention8(*codes, scales, qsl, S, tables, q.double().cpu().numpy(), scale)
    D, u = q.shape[2], 2.0 ** -24
    row = np.repeat(S, np.diff(qsl))[:, None, None]
    bound = (2.0 ** -8 + 2 * (D + 4) * u * most[:, :, None] + 32 * u + 2 * row * u) * mean + 2.0 ** -8 * np.abs(ref) + 1e-30
    err = np.abs(got.double().cpu().numpy() - ref)
    say(f"  max err/bound {(err / bound).max():.3f}")
    assert (err <= bound).all()


SHAPES = [
    # hq, hkv, D, bs, new tokens, cached tokens, wild
    (8, 2, 64, 16, [1, 1, 1, 1], [0, 31, 15, 200], True),
    (32, 8, 128, 16, [5, 1, 0, 5], [100, 16, 40, 0], False),
    (28, 4, 128, 32, [9, 9, 1, 4], [31, 500, 1, 32], False),
    (7, 1, 128, 16, [3, 2], [1000, 17], True),
    (6, 3, 64, 32, [32, 1, 17], [0, 63, 90], True),
    (64, 1, 64, 16, [1, 1], [45, 300], False),
    (1, 1, 128, 32, [33, 64], [0, 5], False),
    (16, 2, 64, 16, [1] * 70, list(range(70)), False),
    (12, 6, 128, 16, [2, 0, 0, 7], [1, 9, 0, 250], True),
    (4, 2, 128, 32, [1], [4000], False),
]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("chunk", [0, 32, 100])
def test_against_64_bits(shape, chunk):
    hq, hkv, D, bs, n, ctx, wild = SHAPES[shape]
    r = np.random.default_rng(shape)
    qsl, S, tables, blocks = batch(n, ctx, bs, shape)
    codes, scales = cache(blocks, bs, hkv, D, r, wild)
    q = torch.from_numpy(r.standard_normal((int(qsl[-1]), hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    say(f"[attention 8 bit] {SHAPES[shape]} chunk {chunk}")
    scale = float(np.float32(D ** -0.5))
    got = attend(pools(codes, bs), dev(scales), blocks, hkv, bs, D, qsl, S, tables, q, scale, chunk)
    check(got, codes, scales, qsl, S, tables, q, scale)


def test_what_lies_behind_a_sequence_does_not_matter():
    """NaN codes in the slots behind each sequence and in the spare blocks, whatever scale those have: the same bits."""
    hq, hkv, D, bs = 8, 2, 128, 16
    r = np.random.default_rng(3)
    qsl, S, tables, blocks = batch([2, 1, 3], [20, 0, 44], bs, 3)
    codes, scales = cache(blocks, bs, hkv, D, r, False)
    q = torch.from_numpy(r.standard_normal((6, hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    a = attend(pools(codes, bs), dev(scales), blocks, hkv, bs, D, qsl, S, tables, q, 0.1)
    used = np.zeros((blocks, bs), bool)
    for b in range(3):
        t = np.arange(S[b])
        used[tables[b, t // bs], t % bs] = True
    for c in codes:
        c[~used] = 255
    scales[~used.any(axis=1)] = np.nan
    b = attend(pools(codes, bs), dev(scales), blocks, hkv, bs, D, qsl, S, tables, q, 0.1)
    assert torch.equal(a, b) and torch.isfinite(a).all()


def test_a_nan_reaches_those_that_see_it_alone():
    hq, hkv, D, bs = 4, 2, 64, 16
    r = np.random.default_rng(4)
    qsl, S, tables, blocks = batch([4, 2], [30, 5], bs, 4)
    codes, scales = cache(blocks, bs, hkv, D, r, False)
    q = torch.from_numpy(r.standard_normal((6, hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    codes[0][tables[0, 2], 0, 0, 3] = 127      # K of KV head 0 at position 32: query tokens 2 and 3
    codes[1][tables[0, 2], 1, 1, 3] = 255      # V of KV head 1 at position 33, dim 3: query token 3
    out = attend(pools(codes, bs), dev(scales), blocks, hkv, bs, D, qsl, S, tables, q, 0.1).cpu()
    bad = torch.isnan(out)
    want = torch.zeros_like(bad)
    want[2:4, :2] = True
    want[3, 2:, 3] = True
    assert torch.equal(bad, want)


def test_an_offset_past_31_bits():
    """A pool of more than 2^31 bytes: the sequence's blocks lie at its end."""
    hq, hkv, D, bs = 8, 8, 128, 32
    r = np.random.default_rng(6)
    blocks = (1 << 31) // (hkv * bs * D) + 4
    qsl, S, tables, own = batch([3], [90], bs, 6)
    codes, scales = cache(own, bs, hkv, D, r, False)
    small = pools(codes, bs)
    big = [torch.zeros(blocks * hkv * bs * D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for f, s in zip(big, small):
        f[-s.numel():] = s.view(torch.uint8)
    sc = torch.ones((blocks, hkv, 2), device="cuda")
    sc[-own:] = dev(scales)
    q = torch.from_numpy(r.standard_normal((3, hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    a = attend(small, dev(scales), own, hkv, bs, D, qsl, S, tables, q, 0.09)
    b = attend([f.view(torch.float8_e4m3fn) for f in big], sc, blocks, hkv, bs, D, qsl, S, tables + blocks - own, q, 0.09)
    assert torch.equal(a, b)
    # and an append there
    new = [torch.from_numpy(r.standard_normal((3, hkv, D)).astype(np.float32)).to(torch.bfloat16).cuda() for _ in range(2)]
    ssc = dev(scales)
    for f, s_, nb, t in ((small, ssc, own, tables), ([f.view(torch.float8_e4m3fn) for f in big], sc, blocks, tables + blocks - own)):
        sx.spexis_rotate_append_kv8(*f, s_, nb, hkv, bs, D, dev(qsl), dev(S), dev(t), 3, 3, *new)
    torch.cuda.synchronize()
    assert torch.equal(ssc, sc[-own:])
    for f, s in zip(big, small):
        assert torch.equal(f[-s.numel():], s.view(torch.uint8)) and not f[: -s.numel()].any()


@pytest.mark.parametrize("chunk", [0, 32])
def test_a_padded_batch(chunk):
    """More rows than the sequences have, and sequences without rows at the end: the same bits, nothing written behind."""
    hq, hkv, D, bs, n, pad = 8, 2, 64, 16, [2, 1, 5, 0, 0], 3
    r = np.random.default_rng(8)
    qsl, S, tables, blocks = batch(n, [300, 0, 44, 0, 0], bs, 8)
    T = int(qsl[-1])
    codes, scales = cache(blocks, bs, hkv, D, r)
    q = torch.from_numpy(r.standard_normal((T + pad, hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    pool, sc = pools(codes, bs), dev(scales)
    say(f"[attention 8 bit] padded, chunk {chunk}")
    got, want = (attend(pool, sc, blocks, hkv, bs, D, qsl, S, tables, x, 0.125, chunk) for x in (q, q[:T]))
    assert torch.equal(got[:T], want) and (got[T:] == 777.0).all()


@pytest.mark.parametrize("B,hq,hkv,bs,most", [(20, 8, 8, 16, 90), (65, 4, 1, 32, 700), (300, 2, 2, 16, 300), (600, 6, 1, 16, 120)])
def test_many_items_of_any_length(B, hq, hkv, bs, most):
    """Shares that begin behind a sequence's last tile, hold several sequences or a part of one; sequences without rows."""
    r = np.random.default_rng(B)
    n = r.integers(0, 6, B)
    ctx = (most * r.random(B) ** 3).astype(np.int32)
    n[-1] = 0
    qsl, S, tables, blocks = batch(n, ctx, bs, B)
    codes, scales = cache(blocks, bs, hkv, 64, r, False)
    q = torch.from_numpy(r.standard_normal((int(qsl[-1]), hq, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    say(f"[attention 8 bit] {B} sequences of up to {most} keys")
    got = attend(pools(codes, bs), dev(scales), blocks, hkv, bs, 64, qsl, S, tables, q, 0.125)
    check(got, codes, scales, qsl, S, tables, q, 0.125)


@pytest.mark.parametrize("B,most", [(1, 500), (3, 900), (16, 1000), (40, 300)])   # either merge of 63-row items
def test_tall_items_in_many_shares(B, most):
    r = np.random.default_rng(B)
    qsl, S, tables, blocks = batch([9] * B, r.integers(most // 3, most + 1, B), 32, B)
    codes, scales = cache(blocks, 32, 2, 128, r, False)
    q = torch.from_numpy(r.standard_normal((9 * B, 14, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    scale = float(np.float32(128 ** -0.5))
    say(f"[attention 8 bit] {B} sequences of up to {most} keys, 63 rows")
    check(attend(pools(codes, 32), dev(scales), blocks, 2, 32, 128, qsl, S, tables, q, scale), codes, scales, qsl, S, tables, q, scale)
