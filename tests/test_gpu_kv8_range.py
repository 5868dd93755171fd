"""Values next to the type's largest in the 8-bit cache: what is stored times its scale is finite in bf16, so that a
weight of 0 makes nothing of it."""
import sys

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import spexis as sx
from tests.test_gpu_attention8 import attend
from tests.test_gpu_rotate import dev, same_codes, table

pytestmark = pytest.mark.gpu

# bf16 values around 448 * 2^119 (2.98e38), 240 * 2^120 (3.19e38), half way to 256 * 2^120 (3.30e38), and the largest
LARGE = [2.97e38, 2.99e38, 3.18e38, 3.2e38, 3.29e38, 3.31e38, 3.35e38, 3.3895e38]


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def logical(pool, place):
    return pool.view(torch.uint8).cpu().numpy()[place]


@pytest.mark.parametrize("D,bs", [(64, 16), (128, 32)])
@pytest.mark.parametrize("turned", [False, True])
def test_codes_of_large_values(D, bs, turned):
    """Bit for bit the plain form's; every stored value is finite in bf16 and within half a step of what was given, or
    the largest that is.  Rows with an infinity and a NaN among them, and rows that a block held before."""
    hkv, held, n = 2, 3, 2 * bs
    r = np.random.default_rng(D)
    x = r.standard_normal((2, n, hkv, D)) * 1e37
    flat = x.reshape(-1)
    at = r.permutation(flat.size)[:600]
    flat[at] = np.resize(np.array(LARGE) * np.array([1, -1, 1, -1, 1, -1, -1, 1]), 600)
    x[0, 5, 0, 3], x[1, 6, 1, 4] = np.inf, np.nan
    new = [torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16) for a in x]
    assert all(torch.isfinite(a).sum() == a.numel() - 1 for a in new)
    qsl, S, tables = np.array([0, n], np.int32), np.array([held + n], np.int32), np.array([[2, 0, 1]], np.int32)
    codes = [r.integers(0, 127, (3, bs, hkv, D)).astype(np.uint8) for _ in range(2)]
    scales = np.exp2(r.integers(118, 120, (3, hkv, 2))).astype(np.float32)
    places = osv.places8(3, hkv, bs, D)
    pools = []
    for c, p in zip(codes, places):
        flat = np.zeros(c.size, np.uint8)
        flat[p] = c
        pools.append(dev(flat).view(torch.float8_e4m3fn))
    sc, cs = dev(scales), table(64 + n, D)
    say(f"[kv8 range] D={D} bs={bs} turned {turned}")
    rotation = dict(cos_sin=dev(cs)) if turned else {}
    sx.spexis_rotate_append_kv8(*pools, sc, 3, hkv, bs, D, dev(qsl), dev(S), dev(tables), n, n, new[0].cuda(), new[1].cuda(),
                                **rotation)
    torch.cuda.synchronize()
    rows = [a.double().numpy() for a in new]
    if turned:
        with np.errstate(invalid="ignore", over="ignore"):
            rows[0] = osv.rotate(rows[0], cs, osv.token_positions(qsl, S), 0).astype(np.float32)
    for part in range(2):
        one = scales[:, :, part].copy()
        osv.append8(codes[part], one, qsl, S, tables, rows[part])
        assert np.array_equal(sc[:, :, part].cpu().numpy(), one)
        got = logical(pools[part], places[part])
        same_codes(got, codes[part])
        # by position: the stored values against the given ones
        t = np.arange(held, held + n)
        value = osv.E4M3[got[tables[0, t // bs], t % bs]] * one[tables[0, t // bs]][:, :, None].astype(np.float64)
        x = np.asarray(rows[part], np.float64)
        fine = np.isfinite(x)
        assert np.array_equal(fine, np.isfinite(value))
        kept = torch.from_numpy(value).to(torch.bfloat16).double().numpy()
        assert np.array_equal(kept[fine], value[fine])
        most = 240 * 2.0 ** 120
        step = one[tables[0, t // bs]][:, :, None] * 2.0 ** -10 + 2.0 ** -4 * np.abs(x)
        x = np.clip(x, -most, most)
        assert (np.abs(value - x)[fine] <= step[fine]).all()


def test_a_large_value_does_not_reach_those_that_do_not_see_it():
    """The last new token's V is the type's largest.  The tokens before it give the bits that they give without it; the
    token itself, whose weight for it underflows to 0, too."""
    hq, hkv, D, bs, n = 4, 2, 64, 16, 3
    r = np.random.default_rng(2)
    qsl, S, tables = np.array([0, n], np.int32), np.array([17], np.int32), np.array([[1, 0]], np.int32)   # the last in a block of its own
    codes = [osv.encode(64 * r.standard_normal((2, bs, hkv, D))) for _ in range(2)]
    places = osv.places8(2, hkv, bs, D)
    new_k, new_v = (torch.from_numpy(r.standard_normal((n, hkv, D)).astype(np.float32)).to(torch.bfloat16) for _ in range(2))
    q = torch.from_numpy(r.standard_normal((n, hq, D)).astype(np.float32)).to(torch.bfloat16)
    q[2], new_k[2] = 20.0, -20.0    # its own key: a score of -20 * 20 * 64 / 8
    outs = []
    for large in (1.0, 3.3895e38, -3.35e38):
        new_v[2] = large
        pools = []
        for c, p in zip(codes, places):
            flat = np.zeros(c.size, np.uint8)
            flat[p] = c
            pools.append(dev(flat).view(torch.float8_e4m3fn))
        sc = torch.full((2, hkv, 2), 2.0 ** -6, device="cuda")
        sx.spexis_rotate_append_kv8(*pools, sc, 2, hkv, bs, D, dev(qsl), dev(S), dev(tables), n, n, new_k.cuda(), new_v.cuda())
        say(f"[kv8 range] attention next to {large}")
        outs.append(attend(pools, sc, 2, hkv, bs, D, qsl, S, tables, q.cuda(), 0.125))
    for out in outs:
        assert torch.isfinite(out).all() and torch.equal(out, outs[0])
