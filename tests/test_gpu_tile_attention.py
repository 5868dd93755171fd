"""Attention of whole prompts and of batches with shared prefixes against its 64-bit form.

The tolerance of an output element, with A the weighted mean of |v| (the weights sum to 1) and u = 2^-24:
  * every weight is rounded to bf16 (2^-8 of it) in front of the product with V, the sum of the weights is not: 2^-8 A;
  * a score is an fp32 sum of D exact products; the scale, the difference to the maximum and the maximum's own product with
    the scale round too, and again where the maximum moves or parts are joined: e = (D + 16) u max_t sum |q k| scale moves a
    weight by e times itself, in the output and in the sum: 2 e A; exp2 and the joining of parts add a few units of u each,
    counted as 32 u A; sums of S terms in fp32, one after the other at worst: 2 S u A;
  * the output is rounded to bf16: 2^-8 |o|.
Of lse: e + (S + 32) u of the sum, and roundings of its terms, 4 u (max_t sum |q k| scale + ln S + 1).
"""
import sys

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import spexis as sx
from tests import layout_ref
from tests.test_gpu_attention8 import pools as pools8
from tests.test_gpu_rotate import batch, dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def say(*a):
    print(*a, file=sys.stderr, flush=True)


class Cache:
    """A cache of values of about N(0, 1): logical k, v [block][slot][head][dim] in 64 bits, and the library's arguments."""

    def __init__(self, blocks, bs, hkv, D, r, in8):
        self.blocks, self.bs, self.hkv, self.D, self.in8 = blocks, bs, hkv, D, in8
        shape = (blocks, bs, hkv, D)
        if in8:
            self.codes = [osv.encode(64 * r.standard_normal(shape)) for _ in range(2)]
            self.scales = np.exp2(r.integers(-7, -5, (blocks, hkv, 2))).astype(np.float32)
            self.refresh()
        else:
            self.k, self.v = (torch.from_numpy(r.standard_normal(shape).astype(np.float32)).to(torch.bfloat16).double().numpy()
                              for _ in range(2))

    def refresh(self):
        self.k, self.v = (osv.E4M3[c] * self.scales[:, None, :, i, None].astype(np.float64) for i, c in enumerate(self.codes))

    def pools(self):
        if self.in8:
            return (*pools8(self.codes, self.bs), dev(self.scales))
        out = []
        for x, f in ((self.k, layout_ref.k_offsets), (self.v, layout_ref.v_offsets)):
            flat = np.zeros(x.size)
            blk, slot, h, d = np.ogrid[:self.blocks, :self.bs, :self.hkv, :self.D]
            flat[f(blk, h, slot, d, self.hkv, self.bs, self.D)] = x
            out.append(dev(flat).to(torch.bfloat16))
        return tuple(out)


def attend(c, pools, qsl, S, tables, q, scale, groups=None, lse=True, stream=None, longer=600):
    """Outputs and lse; rows that the call does not write hold 777.  longer: how far the call's bound is above the longest
    sequence (where it is at most 512, prefixes are not read apart and tiles not in parts)."""
    T, hq = q.shape[:2]
    n = int(np.diff(qsl).max())
    most = max(n, 1), int(max(S.max(), 1)) + longer
    out, ls = torch.full_like(q, 777.0), torch.full((T, hq), 777.0, device="cuda") if lse else None
    where = (c.blocks, c.hkv, c.bs, c.D, dev(qsl), dev(S), dev(tables), T, *most)
    if groups is None:
        size = sx.spexis_prompt_attention_workspace_size(len(S), hq, c.hkv, c.D, T, *most)
        f, more = (sx.spexis_prompt_attention_kv8 if c.in8 else sx.spexis_prompt_attention), ()
    else:
        size = sx.spexis_shared_attention_workspace_size(len(S), len(groups[1]), hq, c.hkv, c.D, T, *most)
        f = sx.spexis_shared_attention_kv8 if c.in8 else sx.spexis_shared_attention
        more = (dev(np.asarray(groups[0], np.int32)), dev(np.asarray(groups[1], np.int32)))
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
    f(*pools, *where, *more, q, hq, scale, out, ws, lse=ls, stream=stream)
    torch.cuda.synchronize()
    return out, ls


def check(got, lse, c, qsl, S, tables, q, scale):
    T = int(qsl[-1])
    ref, mean, most, ref_lse = osv.attention_rows(c.k, c.v, qsl, S, tables, q[:T].double().cpu().numpy(), scale)
    row = np.repeat(S, np.diff(qsl)).astype(np.float64)
    e = (c.D + 16) * U * most
    bound = (2.0 ** -8 + 2 * e[:, :, None] + 32 * U + 2 * row[:, None, None] * U) * mean + 2.0 ** -8 * np.abs(ref) + 1e-30
    err = np.abs(got[:T].double().cpu().numpy() - ref)
    say(f"  max err/bound {(err / bound).max() if T else 0:.3f}")
    assert (err <= bound).all()
    if lse is not None:
        bound = e + (row[:, None] + 32) * U + 4 * U * (most + np.log(row[:, None]) + 1)
        err = np.abs(lse[:T].double().cpu().numpy() - ref_lse)
        say(f"  lse max err/bound {(err / bound).max() if T else 0:.3f}")
        assert (err <= bound).all()


def queries(T, hq, D, r):
    return torch.from_numpy(r.standard_normal((T, hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()


PROMPTS = [
    # hq, hkv, D, bs, new tokens, cached tokens
    (8, 2, 64, 16, [1, 7, 60, 33], [0, 31, 15, 200]),
    (32, 8, 128, 16, [129, 1, 0, 32], [100, 16, 40, 0]),
    (28, 4, 128, 32, [75, 18, 1], [31, 0, 500]),
    (7, 1, 128, 16, [300], [1000]),
    (6, 3, 64, 32, [64, 65, 63], [0, 63, 64]),
    (64, 1, 64, 16, [5, 2], [45, 300]),
    (1, 1, 128, 32, [257, 128], [0, 5]),
    (2, 2, 64, 16, [1] * 300, list(range(300))),
    (4, 4, 128, 16, [600, 1, 1000], [0, 700, 3]),
    (16, 8, 64, 32, [900] * 9, [0] * 9),     # more tiles than workgroups at a time: no parts
    (4, 2, 128, 32, [1], [4000]),
    (3, 1, 64, 16, [1], [0]),
    (4, 2, 64, 16, [0] * 300 + [1], [0] * 300 + [9]),   # fewer row tiles than sequences
    (8, 2, 128, 32, [0, 3, 0, 0, 200, 1] * 30, [40, 3, 0, 700, 90, 5] * 30),
]


@pytest.mark.parametrize("in8,longer", [(False, 0), (False, 600), (True, 600)])
@pytest.mark.parametrize("shape", range(len(PROMPTS)))
def test_prompts_against_64_bits(shape, in8, longer):
    hq, hkv, D, bs, n, ctx = PROMPTS[shape]
    r = np.random.default_rng(shape)
    qsl, S, tables, blocks = batch(n, ctx, bs, shape)
    c = Cache(blocks, bs, hkv, D, r, in8)
    q = queries(int(qsl[-1]), hq, D, r)
    scale = float(np.float32(D ** -0.5))
    say(f"[prompt] {PROMPTS[shape][:4]} 8 bit {in8}")
    out, lse = attend(c, c.pools(), qsl, S, tables, q, scale, longer=longer)
    check(out, lse, c, qsl, S, tables, q, scale)


def shared_batch(bs, groups, alone, r, seed):
    """Sequences of groups (prefix, [(own cached tokens, new tokens), ...]), `alone` = (in front, behind) ones without a
    group.  Tables of a group begin with the same blocks."""
    seqs, start, prefix = [], [], []
    for own in alone[0]:
        seqs.append((0, None, *own))
    for pre, members in groups:
        start.append(len(seqs))
        prefix.append(pre)
        seqs += [(pre, len(start) - 1, *own) for own in members]
    start.append(len(seqs))
    for own in alone[1]:
        seqs.append((0, None, *own))
    n = np.array([s[3] for s in seqs], np.int32)
    ctx = np.array([s[0] + s[2] for s in seqs], np.int32)
    qsl, S, tables, blocks = batch(n, ctx, bs, seed)
    for i in range(len(groups)):
        for b in range(start[i], start[i + 1]):
            w = prefix[i] // bs
            tables[b, :w] = tables[start[i], :w]
    return qsl, S, tables, blocks, (start, prefix)


SHARED = [
    # hq, hkv, D, bs, groups, alone
    (8, 2, 64, 16, [(64, [(3, 5), (0, 5), (40, 1), (17, 2)])], ([], [])),
    (32, 8, 128, 16, [(200, [(10, 5), (100, 5), (0, 1)]), (16, [(0, 1)]), (0, [(5, 2), (90, 5)])], ([(30, 3)], [(0, 4), (500, 1)])),
    (28, 4, 128, 32, [(1000, [(33, 9)] * 20), (64, [(0, 9)] * 3)], ([], [])),
    (4, 4, 128, 16, [(4000, [(0, 1)])], ([], [])),
    (16, 2, 64, 32, [(96, [(i % 7, i % 4) for i in range(290)])], ([], [])),    # some without query tokens
    (6, 3, 64, 16, [(77, [(20, 3), (31, 1)]), (47, [(0, 2), (1, 1)])], ([], [(9, 1)])),   # prefixes that end inside a block
    (2, 1, 128, 32, [(128, [(0, 200), (300, 1), (5, 40)])], ([], [])),         # prompts behind an instruction
    (8, 8, 64, 16, [(160, [(11, 2)] * 6)] * 40, ([], [])),                     # prefixes in a launch of their own
    (56, 8, 64, 32, [(2000, [(i % 50, 9) for i in range(66)]), (0, [(3, 1)] * 30), (320, [(7, 70)] * 20)], ([(9, 2)], [(0, 1)] * 3)),
]


@pytest.mark.parametrize("in8,longer", [(False, 0), (False, 600), (True, 600)])
@pytest.mark.parametrize("shape", range(len(SHARED)))
def test_shared_prefixes_against_64_bits(shape, in8, longer):
    hq, hkv, D, bs, groups, alone = SHARED[shape]
    r = np.random.default_rng(100 + shape)
    qsl, S, tables, blocks, g = shared_batch(bs, groups, alone, r, shape)
    c = Cache(blocks, bs, hkv, D, r, in8)
    q = queries(int(qsl[-1]), hq, D, r)
    scale = float(np.float32(D ** -0.5))
    say(f"[shared] {SHARED[shape][:4]} 8 bit {in8}")
    out, lse = attend(c, c.pools(), qsl, S, tables, q, scale, groups=g, longer=longer)
    check(out, lse, c, qsl, S, tables, q, scale)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-30, 1.5])
@pytest.mark.parametrize("shared", [False, True])
def test_scales(scale, shared):
    """None, a negative one, and one that makes single keys decide."""
    r = np.random.default_rng(5)
    qsl, S, tables, blocks, g = shared_batch(16, [(48, [(30, 9), (0, 40)])], ([], []), r, 5)
    c = Cache(blocks, 16, 2, 64, r, False)
    q = queries(int(qsl[-1]), 8, 64, r)
    scale = float(np.float32(scale))
    out, lse = attend(c, c.pools(), qsl, S, tables, q, scale, groups=g if shared else None)
    check(out, lse, c, qsl, S, tables, q, scale)


def test_scores_that_grow_along_the_keys():
    """The maximum moves at every step of the keys: by far, and by less than what moves the reference."""
    for step in (0.02, 0.3):
        r = np.random.default_rng(6)
        qsl, S, tables, blocks = batch([40], [500], 16, 6)
        c = Cache(blocks, 16, 1, 64, r, False)
        t = np.arange(540)
        rows = np.zeros((540, 64))
        rows[:, 0] = t * step
        rows[:, 1:] = 0.1 * r.standard_normal((540, 63))
        c.k[tables[0, t // 16], t % 16, 0] = torch.from_numpy(rows).to(torch.bfloat16).double().numpy()
        q = queries(40, 4, 64, r)
        q[:, :, 0] = 4.0
        out, lse = attend(c, c.pools(), qsl, S, tables, q, 0.125)
        check(out, lse, c, qsl, S, tables, q, 0.125)


@pytest.mark.parametrize("in8", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_what_lies_behind_a_sequence_does_not_matter(in8, shared):
    """NaN in the slots behind each sequence and in spare blocks: the same bits."""
    r = np.random.default_rng(3)
    qsl, S, tables, blocks, g = shared_batch(16, [(32, [(20, 70), (0, 1), (44, 3)])], ([], []), r, 3)
    c = Cache(blocks, 16, 2, 128, r, in8)
    q = queries(int(qsl[-1]), 8, 128, r)
    a = attend(c, c.pools(), qsl, S, tables, q, 0.1, groups=g if shared else None)
    used = np.zeros((blocks, 16), bool)
    for b in range(len(S)):
        t = np.arange(S[b])
        used[tables[b, t // 16], t % 16] = True
    if in8:
        for x in c.codes:
            x[~used] = 255
        c.scales[~used.any(axis=1)] = np.nan
    else:
        for x in (c.k, c.v):
            x[~used] = np.nan
    b = attend(c, c.pools(), qsl, S, tables, q, 0.1, groups=g if shared else None)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.isfinite(a[0]).all()


@pytest.mark.parametrize("in8", [False, True])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_finite_reaches_those_that_see_it_alone(in8, shared, D):
    r = np.random.default_rng(4)
    qsl, S, tables, blocks, g = shared_batch(16, [(32, [(10, 100), (0, 5)])], ([], []), r, 4)
    c = Cache(blocks, 16, 2, D, r, in8)
    q = queries(int(qsl[-1]), 4, D, r)

    def put(part, pos, head, dim, value):
        at = tables[0, pos // 16], pos % 16, head, dim
        if in8:
            c.codes[part][at] = 255
        else:
            (c.k, c.v)[part][at] = value
    put(0, 60, 0, 3, np.nan)              # K of KV head 0 at position 60: tokens from 18 on
    put(1, 42 + 33, 1, 37, np.inf)        # V of KV head 1, its own tokens: from 33, 70 and 99 on
    put(1, 42 + 70, 1, D - 1, -np.inf)
    put(1, 42 + 99, 1, 0, np.nan)
    put(1, 42 + 50, 1, 37, np.nan)
    out, lse = attend(c, c.pools(), qsl, S, tables, q, 0.1, groups=g if shared else None)
    bad = ~torch.isfinite(out).cpu()
    want = torch.zeros_like(bad)
    want[18:100, :2] = True
    want[33:100, 2:, 37] = True
    want[70:100, 2:, D - 1] = True
    want[99, 2:, 0] = True
    assert torch.equal(bad, want)
    assert torch.equal(~torch.isfinite(lse).cpu(), want[:, :, 1])


@pytest.mark.parametrize("shared", [False, True])
def test_a_padded_batch(shared):
    """More rows than the sequences have, sequences without rows or keys at the end: the same bits, nothing behind them."""
    r = np.random.default_rng(8)
    n, pad = [70, 1, 5, 0, 0], 40
    qsl, S, tables, blocks = batch(n, [300, 0, 44, 20, 0], 16, 8)
    c = Cache(blocks, 16, 2, 64, r, False)
    T = int(qsl[-1])
    q = queries(T + pad, 8, 64, r)
    g = ([0, 1, 5], [160, 0]) if shared else None
    out, lse = attend(c, c.pools(), qsl, S, tables, q, 0.125, groups=g)
    check(out, lse, c, qsl, S, tables, q, 0.125)
    assert (out[T:] == 777.0).all() and (lse[T:] == 777.0).all()


@pytest.mark.parametrize("hkv", [2, 16])   # together and merged; the prefixes in front
def test_groups_that_overlap_write_nothing_outside(hkv):
    """More prefix units than an ascending list of groups can have: outputs unspecified, what is around them as it was, also
    with a workspace in which a call of more rows has left its headers."""
    r = np.random.default_rng(12)
    n, G, groups = [5, 9, 3, 8], 16, 400
    qsl, S, tables, blocks = batch(n, [700, 650, 800, 640], 16, 12)
    tables[:, :38] = tables[0, :38]
    c = Cache(blocks, 16, hkv, 64, r, False)
    k, v = c.pools()
    T, more = int(qsl[-1]), 40
    q, out = queries(T + more, G * hkv, 64, r), torch.full((T + more, G * hkv, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + more, G * hkv), 5.0, device="cuda")
    starts = np.array([0, 4] * (groups // 2) + [4], np.int32)   # every other group is all of them
    lens = np.full(groups, 38 * 16, np.int32)
    size = sx.spexis_shared_attention_workspace_size(4, groups, G * hkv, hkv, 64, T, 9, 809)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    ws[: size // 16 * 16].view(torch.int32).view(-1, 4)[:] = torch.tensor([1, T + 20, 16, 0], dtype=torch.int32, device="cuda")
    sx.spexis_shared_attention(k, v, blocks, hkv, 16, 64, dev(qsl), dev(S), dev(tables), T, 9, 809, dev(starts), dev(lens), q,
                               G * hkv, 0.125, out, ws, lse=lse)
    torch.cuda.synchronize()
    assert (out[T:] == 3.0).all() and (lse[T:] == 5.0).all()


def test_without_lse_and_without_groups():
    r = np.random.default_rng(9)
    qsl, S, tables, blocks = batch([40, 3], [20, 700], 32, 9)
    c = Cache(blocks, 32, 2, 64, r, False)
    q = queries(43, 6, 64, r)
    p = c.pools()
    a, _ = attend(c, p, qsl, S, tables, q, 0.125)
    b, _ = attend(c, p, qsl, S, tables, q, 0.125, lse=False)
    d, _ = attend(c, p, qsl, S, tables, q, 0.125, lse=False, groups=([0], []))
    assert torch.equal(a, b) and torch.equal(a, d)
    out = torch.zeros_like(q)
    ws = torch.empty(sx.spexis_shared_attention_workspace_size(2, 0, 6, 2, 64, 43, 40, 1303), dtype=torch.uint8, device="cuda")
    sx.spexis_shared_attention(*p, c.blocks, 2, 32, 64, dev(qsl), dev(S), dev(tables), 43, 40, 1303, None, None, q, 6, 0.125, out, ws)
    assert torch.equal(a, out)


def test_an_offset_past_31_bits():
    """A pool of more than 2^31 elements: the sequence's blocks lie at its end."""
    r = np.random.default_rng(6)
    hkv, D, bs = 8, 128, 32
    blocks = (1 << 31) // (hkv * bs * D) + 4
    qsl, S, tables, own = batch([90], [100], bs, 6)
    c = Cache(own, bs, hkv, D, r, False)
    q = queries(90, 8, D, r)
    small = c.pools()
    big = [torch.zeros(blocks * hkv * bs * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for f, s in zip(big, small):
        f[-s.numel():] = s
    a = attend(c, small, qsl, S, tables, q, 0.09)
    c.blocks = blocks
    b = attend(c, big, qsl, S, tables + blocks - own, q, 0.09)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("shared", [False, True])
def test_replays_and_streams(shared):
    """Two captured calls that share a workspace, replayed with eager calls between them; two streams at once."""
    r = np.random.default_rng(11)
    calls = []
    for n, ctx in (([30, 5], [500, 20]), ([7, 60, 1], [90, 0, 333])):
        qsl, S, tables, blocks = batch(n, ctx, 16, len(calls))
        c = Cache(blocks, 16, 2, 64, r, False)
        T, most, keys = int(qsl[-1]), max(n), int(S.max()) + 600
        q, out = queries(T, 8, 64, r), torch.empty((T, 8, 64), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((T, 8), device="cuda")
        where = (c.blocks, 2, 16, 64, dev(qsl), dev(S), dev(tables), T, most, keys)
        if shared:
            where = (*where, dev(np.array([0, 1], np.int32)), dev(np.array([16 if ctx[0] > 90 else 80], np.int32)))
            size = sx.spexis_shared_attention_workspace_size(len(S), 1, 8, 2, 64, T, most, keys)
        else:
            size = sx.spexis_prompt_attention_workspace_size(len(S), 8, 2, 64, T, most, keys)
        f = sx.spexis_shared_attention if shared else sx.spexis_prompt_attention
        p = c.pools()
        calls.append((lambda ws, stream=None, a=(f, p, where, q, out, lse):
                      a[0](*a[1], *a[2], a[3], 8, 0.125, a[4], ws, lse=a[5], stream=stream), out, lse, size))
    ws = torch.empty(max(x[3] for x in calls), dtype=torch.uint8, device="cuda")
    want = []
    for call, out, lse, _ in calls:
        call(ws)
        torch.cuda.synchronize()
        want.append((out.clone(), lse.clone()))
    graphs = []
    for call, *_ in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(ws)
        graphs.append(g)
    for _ in range(3):
        for _, out, lse, _ in calls:
            out.zero_()
            lse.zero_()
        calls[1][0](ws)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, out, lse, _), w in zip(calls, want):
            assert torch.equal(out, w[0]) and torch.equal(lse, w[1])
    spaces = [torch.empty(x[3], dtype=torch.uint8, device="cuda") for x in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for _, out, lse, _ in calls:
        out.zero_()
        lse.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for (call, *_), s, w in zip(calls, streams, spaces):
            call(w, stream=s)
    torch.cuda.synchronize()
    for (_, out, lse, _), w in zip(calls, want):
        assert torch.equal(out, w[0]) and torch.equal(lse, w[1])


def test_refusals_of_the_binding():
    r = np.random.default_rng(12)
    qsl, S, tables, blocks = batch([4], [20], 16, 1)
    c = Cache(blocks, 16, 2, 64, r, False)
    k, v = c.pools()
    q, out = queries(4, 8, 64, r), torch.empty((4, 8, 64), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(sx.spexis_prompt_attention_workspace_size(1, 8, 2, 64, 4, 4, 24), dtype=torch.uint8, device="cuda")
    a = dict(k=k, v=v, q=q, out=out, ws=ws, qsl=dev(qsl), lse=None, tables=dev(tables), stream=None, start=None, prefix=None)

    def call(shared=False, **kw):
        x = {**a, **kw}
        f = sx.spexis_shared_attention if shared else sx.spexis_prompt_attention
        more = (x["start"], x["prefix"]) if shared else ()
        f(x["k"], x["v"], c.blocks, 2, 16, 64, x["qsl"], dev(S), x["tables"], 4, 4, 24, *more, x["q"], 8, 0.125, x["out"], x["ws"],
          lse=x["lse"], stream=x["stream"])
    call()
    for kw in (dict(k=k[:-1]), dict(v=v[:-8]), dict(q=q[:3]), dict(out=out[:3]), dict(q=q.float()), dict(q=q.cpu()),
               dict(lse=torch.empty(31, device="cuda")), dict(lse=torch.empty(32)), dict(tables=dev(tables)[:0]), dict(ws=ws.cpu()),
               dict(shared=True, start=dev(np.array([0], np.int32)), prefix=dev(np.array([16], np.int32)))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(ws=ws[:8]), dict(out=q), dict(q=torch.empty(4 * 8 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:]),
               dict(shared=True, start=None, prefix=dev(np.array([16], np.int32)))):
        with pytest.raises(sx.SpexisError):
            call(**kw)
