"""A large scale on small q and k: the scores are ordinary ones.  Against the 64-bit form, with the bounds of the other scales."""
import numpy as np
import pytest

from tests.test_gpu_rotate import batch
from tests.test_gpu_tile_attention import Cache, attend, check, queries, say, shared_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [14, 30, 60])
@pytest.mark.parametrize("shared", [False, True])
def test_large_scales(power, shared):
    """Tiles of 128 tokens in parts of 64 keys and more: a row has no score in a part that begins behind its token."""
    r = np.random.default_rng(70 + power)
    if shared:
        qsl, S, tables, blocks, g = shared_batch(16, [(640, [(0, 700), (900, 9), (3, 40)])], ([], []), r, 7)
    else:
        (qsl, S, tables, blocks), g = batch([1200, 3, 70], [0, 2000, 700], 16, 7), None
    c = Cache(blocks, 16, 2, 64, r, False)
    c.k *= 2.0 ** -(power // 2)
    q = queries(int(qsl[-1]), 2, 64, r) * 2.0 ** -(power // 2)
    scale = float(np.float32(0.125)) * 2.0 ** power
    say(f"[large scale] 2^{power}, shared {shared}")
    for sign in (1, -1):
        out, lse = attend(c, c.pools(), qsl, S, tables, q, sign * scale, groups=g)
        check(out, lse, c, qsl, S, tables, q, sign * scale)
