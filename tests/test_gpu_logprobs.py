"""Token log probabilities against their 64-bit form.

Tolerances, with u = 2^-24, w = (x - max x) / T in units of ln 2 and p the row's probabilities:
  * w has three roundings (difference, 1/T, product): 3 u |w|; 2^w and its argument's error: relative 2 u + 3 u |w|;
    a lane sums at most V / 64 + 8 terms one after the other, then sums go over 64 lanes, 4 waves and 64 parts: (V / 64 +
    90) u relative.  So ln Z is off by at most ez = (V / 64 + 92) u + 3 u sum p |w|;
  * log p: ez + 4 u |w| + 4 u |log p| (product with ln 2, log2, sum);
  * H = ln Z + (sum p |w|) ln 2: ez + sum p |w| (ez + (V / 64 + 96) u) + 4 u sum p w^2 + 4 u H.
The ids of the alternatives are equal (ties by index).
"""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import spexis as sx

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def call(logits, tokens, rows, temperature, top, stream=None):
    n = len(tokens)
    ids = torch.full((n, top), -7, dtype=torch.int32, device="cuda")
    alt, lp, h = torch.full((n, top), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ws = torch.empty(max(sx.spexis_token_logprobs_workspace_size(n, logits.shape[1], top), 16), dtype=torch.uint8, device="cuda")
    sx.spexis_token_logprobs(logits, torch.as_tensor(tokens, dtype=torch.int32).cuda(), lp, ws,
                             row_ids=None if rows is None else torch.as_tensor(rows, dtype=torch.int32).cuda(),
                             entropy=h, top_ids=ids, top_logprobs=alt, temperature=temperature, stream=stream)
    torch.cuda.synchronize()
    return lp.cpu().numpy(), h.cpu().numpy(), ids.cpu().numpy(), alt.cpu().numpy()


def check(logits, tokens, rows, temperature, top):
    compare(call(logits, tokens, rows, temperature, top), logits, tokens, rows, temperature, top)


def compare(got, logits, tokens, rows, temperature, top):
    x = logits.double().cpu().numpy()
    V, u = x.shape[1], 2.0 ** -24
    lp, h, ids, alt = got
    with np.errstate(invalid="ignore"):
        wlp, wh, wids, walt = osv.token_logprobs(x, rows, tokens, temperature, top)
    assert np.array_equal(ids, wids)
    ln2, worst = math.log(2), 0.0
    for i in range(len(tokens)):
        row = i if rows is None else rows[i]
        if np.isnan(wlp[i]) or not (0 <= tokens[i] < V and 0 <= row < len(x)):
            for got, want in ((lp[i], wlp[i]), (h[i], wh[i]), (alt[i], walt[i])):
                assert np.array_equal(got, want, equal_nan=True)
            continue
        w = (x[row] - x[row].max()) / temperature / ln2
        p = np.exp2(w)
        p, w = p / p.sum(), np.where(p > 0, w, 0.0)
        ez = (V / 64 + 92) * u + 3 * u * (p * -w).sum()
        for got, want in [(lp[i], wlp[i])] + list(zip(alt[i], walt[i])):
            with np.errstate(over="ignore"):
                if np.isinf(np.float32(want)):   # a lowest value over T < 1 lies beyond the type's range
                    assert got == np.float32(want)
                    continue
            bound = ez + 4 * u * (abs(want) + wh[i] + 40) + 4 * u * abs(want)
            worst = max(worst, abs(got - want) / bound)
        bound = ez + (p * -w).sum() * (ez + (V / 64 + 96) * u) + 4 * u * (p * w * w).sum() + 4 * u * wh[i] + 1e-30
        worst = max(worst, abs(h[i] - wh[i]) / bound)
        assert lp[i] <= 0 and h[i] >= 0
    say(f"  max err/bound {worst:.3f}")
    assert worst <= 1


def rows_of_every_kind(V, r, dtype):
    """Normal rows, ties, masks, sorted and constant rows, rows without a distribution."""
    low = torch.finfo(dtype).min
    n = r.standard_normal((14, V)) * 4
    n[1] = np.round(n[1])
    n[2] = np.sort(n[2])
    n[3] = np.sort(n[3])[::-1]
    n[4] = 1.25
    n[5][r.random(V) < 0.99] = -math.inf
    n[5][V // 2] = 0.5
    n[6][r.random(V) < 0.9] = low
    n[7] = -math.inf
    n[8] = low
    n[9][V - 1] = math.nan
    n[10][V // 3] = math.inf
    n[11] = -math.inf
    n[11][V - 1] = -3.0
    n[12] = r.integers(0, 3, V) * 0.0 * np.where(r.random(V) < 0.5, -1.0, 1.0)     # zeros of both signs
    n[13][V // 2] = 200.0
    return torch.from_numpy(n).clamp(min=low).where(torch.from_numpy(n) != -math.inf, torch.tensor(-math.inf).double()).to(dtype)


@pytest.mark.parametrize("V", [1, 2, 31, 63, 1000, 2049, 8193, 20001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 1, 5, 20, 32])
def test_rows_of_every_kind(V, dtype, top):
    r = np.random.default_rng(V + top)
    x = rows_of_every_kind(V, r, dtype)
    tokens = r.integers(0, V, len(x)).tolist()
    tokens[2], tokens[3], tokens[5] = V - 1, 0, V // 2
    say(f"[logprobs] V={V} {dtype} top {top}")
    check(x.cuda(), tokens, None, 0.7 if top == 5 else 1.0, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,shift", [(1000, 0, 1), (1001, 0, 0), (4099, 5, 3), (333, 3, 2), (7, 1, 5)])
def test_rows_that_start_anywhere(dtype, V, pad, shift):
    """Odd row lengths, rows further apart than they are long, a first row that is not 16-byte aligned."""
    r = np.random.default_rng(V)
    flat = torch.full((shift + 9 * (V + pad),), math.nan, dtype=dtype)   # what lies between the rows is not read
    x = flat[shift:].view(9, V + pad)[:, :V]
    x.copy_(torch.from_numpy(r.standard_normal((9, V)) * 3))
    on = flat.cuda()[shift:].view(9, V + pad)[:, :V]
    say(f"[logprobs] V={V} {dtype} pad {pad} shift {shift}")
    check(on, r.integers(0, V, 9).tolist(), None, 1.0, 5)


@pytest.mark.parametrize("items", [1, 3, 70, 700])
def test_items_pick_their_rows(items):
    """Rows several times, in any order; tokens and rows out of range; every number of parts of a row."""
    r = np.random.default_rng(items)
    V, n = 30011, 40
    x = torch.from_numpy((r.standard_normal((n, V)) * 3).astype(np.float32)).cuda()
    rows, tokens = r.integers(-1, n + 1, items), r.integers(-2, V + 2, items)
    tokens[::3] = -1
    if items == 1:
        rows[0], tokens[0] = 7, V - 1
    say(f"[logprobs] {items} items")
    check(x, tokens.tolist(), rows.tolist(), 0.9, 20)


def test_a_large_vocabulary_and_far_rows():
    """2^22 entries; a row that starts past 2^31 entries."""
    r = np.random.default_rng(1)
    V = 1 << 22
    x = torch.empty((513, V), dtype=torch.bfloat16, device="cuda")
    x[512] = torch.from_numpy(r.standard_normal(V).astype(np.float32)).cuda().to(torch.bfloat16)
    x[0] = x[512].flip(0)
    say("[logprobs] V=2^22")
    got = call(x, [V - 1, 0, 5], [512, 0, 512], 1.0, 8)
    y = x[[512, 0]]
    check(y, [V - 1, 0, 5], [0, 1, 0], 1.0, 8)
    want = call(y, [V - 1, 0, 5], [0, 1, 0], 1.0, 8)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


def test_no_items():
    sx.spexis_token_logprobs(torch.empty((0, 50), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                             torch.empty(0, device="cuda"))
    with pytest.raises(ValueError):
        sx.spexis_token_logprobs(torch.empty((2, 50), device="cuda").t(), torch.empty(1, dtype=torch.int32, device="cuda"),
                                 torch.empty(1, device="cuda"))


def test_shapes_and_devices_that_are_refused(monkeypatch):
    """What the number of items is taken from, and the buffers that have to be as long."""
    x, three = torch.zeros((4, 50), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    out = torch.zeros(3, device="cuda")
    top = (torch.zeros((3, 5), dtype=torch.int32, device="cuda"), torch.zeros((3, 5), device="cuda"))
    for kw in (dict(logprobs=out[:2]), dict(row_ids=three[:2]), dict(entropy=out[:1]), dict(top_ids=top[0]),
               dict(top_logprobs=top[1]), dict(top_ids=top[0][:2], top_logprobs=top[1][:2]),
               dict(top_ids=top[0], top_logprobs=top[1][:, :4].contiguous())):
        with pytest.raises(ValueError):
            sx.spexis_token_logprobs(x, three, **dict(dict(logprobs=out), **kw))
    sx.spexis_token_logprobs(x, three, out, top_ids=top[0], top_logprobs=top[1])
    torch.cuda.synchronize()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    with pytest.raises(ValueError):
        sx.spexis_token_logprobs(x, three, out)


@pytest.mark.parametrize("items", [1, 9, 100, 300, 600])
def test_every_number_of_parts(items):
    """Long rows: cut into many parts, a few, none; as many items as rows, and more (some without a token)."""
    r = np.random.default_rng(items)
    V, n = 50021, min(items, 40)
    x = torch.from_numpy((r.standard_normal((n, V)) * 3).astype(np.float32)).cuda()
    x[:, 17:900:5] = x[:, 40000:40001]   # equal logits in several parts
    rows = r.integers(0, n, items)
    tokens = r.integers(0, V, items)
    say(f"[logprobs] {items} items of {n} rows of {V}")
    check(x, tokens.tolist(), rows.tolist(), 1.3, 12)
    if items <= n:
        check(x, tokens.tolist(), None, 1.3, 12)
    else:
        wide = x.repeat(-(-items // n), 1)[:items]
        check(wide, tokens.tolist(), None, 1.3, 12)
        tokens[::2] = -1
        check(x, tokens.tolist(), rows.tolist(), 1.3, 0)
