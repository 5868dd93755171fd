"""Shared prefixes where the sequences' own keys are longer than the prefix, in few segments and with many KV heads: whichever
segment is longest, every part of a prefix counts.  Against the 64-bit form, with the bounds of the other shapes."""
import numpy as np
import pytest

from tests.test_gpu_tile_attention import Cache, attend, check, queries, say, shared_batch

import torch

pytestmark = pytest.mark.gpu

SHAPES = [
    # hq, hkv, D, bs, groups of (prefix, [(own cached tokens, new tokens)])
    (32, 32, 64, 16, [(128, [(500, 5)] * 40)]),
    (32, 16, 128, 16, [(96, [(430, 5)] * 54)]),
    # prefixes shorter than some sequences and longer than others
    (32, 16, 64, 32, [(128, [(500, 3)] * 17), (640, [(60, 7)] * 15), (64, [(450, 2)] * 22)]),
    (24, 24, 64, 16, [(64, [(500, 5)] * 20), (576, [(600, 1)] * 8), (128, [(90, 6)] * 10)]),
    # 64 segments and 65
    (16, 16, 64, 16, [(128, [(450, 9)] * 63)]),
    (16, 16, 64, 16, [(128, [(450, 9)] * 64)]),
    # eight KV heads, more than one row tile a sequence
    (16, 8, 64, 16, [(128, [(450, 68)] * 62)]),
]


@pytest.mark.parametrize("in8", [False, True])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefixes_shorter_than_what_follows(shape, in8):
    hq, hkv, D, bs, groups = SHAPES[shape]
    r = np.random.default_rng(300 + shape)
    qsl, S, tables, blocks, g = shared_batch(bs, groups, ([], []), r, shape)
    c = Cache(blocks, bs, hkv, D, r, in8)
    q = queries(int(qsl[-1]), hq, D, r)
    scale = float(np.float32(D ** -0.5))
    say(f"[shared, short prefixes] {SHAPES[shape][:4]} {len(S)} sequences, 8 bit {in8}")
    pools = c.pools()
    out, lse = attend(c, pools, qsl, S, tables, q, scale, groups=g)
    check(out, lse, c, qsl, S, tables, q, scale)
    again = attend(c, pools, qsl, S, tables, q, scale, groups=g)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
