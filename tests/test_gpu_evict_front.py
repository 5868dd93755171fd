"""Evictions with more keys at the front that stay than a workgroup holds in registers (a long shared document), whose weights
are the largest: they must not count among the keys that are chosen.  Exact."""
import numpy as np
import pytest

from oracle import serving as osv
from tests.test_gpu_evict import evict, logical, say, used_places
from tests.test_gpu_rotate import batch, dev
from tests.test_gpu_tile_attention import Cache

pytestmark = pytest.mark.gpu

SHAPES = [
    # hkv, D, bs, lengths, kept, first, last
    (2, 64, 16, [30000, 20000], [24000, 18000], [20000, 17000], 0),
    (1, 64, 32, [20000, 20000, 20000, 20000], [18000, 18000, 18000, 18000], [16383, 16384, 16385, 16399], 7),
    (1, 128, 16, [20000, 19000], [17500, 17500], [17500, 19000], 5),         # nothing to choose among
    (2, 64, 32, [18000, 40000, 300], [17990, 33001, 200], [17000, 33000, 100], 1000),
    (1, 64, 16, [33000, 20000], [20001, 17001], [20000, 17000], 0),          # one of many
]


@pytest.mark.parametrize("kind", ["heavy", "ties", "odd"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_long_front(shape, kind):
    hkv, D, bs, S, keep, first, last = SHAPES[shape]
    r = np.random.default_rng(40 + shape)
    _, S, tables, blocks = batch([0] * len(S), S, bs, shape)
    c = Cache(blocks, bs, hkv, D, r, False)
    w = r.exponential(size=(blocks, hkv, bs)).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 2).astype(np.float32)
    if kind == "odd":
        for x in (np.nan, np.inf, -np.inf, -1.0):
            w[r.random(w.shape) < 0.1] = x
    for b in range(len(S)):
        t = np.arange(min(first[b], S[b]))
        w[tables[b, t // bs], :, t % bs] += 8.0
    say(f"[evict, long front] {SHAPES[shape]} {kind}")
    for same in (False, True):
        pools, weights = c.pools(), dev(w)
        got, lens = evict(c, pools, weights, S, tables, keep, first, last, out=weights if same else None, lens=same or None)
        k, v, w2, m = osv.evict(c.k, c.v, w, S, tables, keep, first, last)
        assert np.array_equal(lens, m)
        kept = used_places(m, tables, blocks, bs)
        free = used_places(S, tables, blocks, bs) & ~kept
        got = got.cpu().numpy()
        assert np.array_equal(got.transpose(0, 2, 1)[kept], w2.transpose(0, 2, 1)[kept], equal_nan=True)
        if not same:
            assert (got.transpose(0, 2, 1)[~kept] == 777.0).all()
        for pool, want, which in zip(pools, (k, v), "kv"):
            x = logical(pool, c, which)
            assert np.array_equal(x[~free], want[~free]), which
