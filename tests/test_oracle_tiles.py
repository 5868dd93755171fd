"""What pins the plain forms of attention over many rows, of attention weights and of eviction."""
import math

import numpy as np
import torch

from oracle import serving as osv


def cache(blocks, bs, hkv, D, seed):
    r = np.random.default_rng(seed)
    return r.standard_normal((blocks, bs, hkv, D)), r.standard_normal((blocks, bs, hkv, D)), r


def test_attention_is_torchs_and_its_lse_the_logarithm_of_the_sum():
    bs, hkv, G, D = 4, 2, 3, 8
    k, v, r = cache(6, bs, hkv, D, 0)
    tables, qsl, S = np.array([[3, 0, 5], [1, 4, 2]]), [0, 5, 6], [11, 7]
    q = r.standard_normal((6, hkv * G, D))
    out, mean, most, lse = osv.attention_rows(k, v, qsl, S, tables, q, -0.3)
    for b, n in enumerate((5, 1)):
        t = np.arange(S[b])
        kb, vb = (torch.tensor(x[tables[b, t // bs], t % bs]).transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
        qb = torch.tensor(q[qsl[b]:qsl[b + 1]]).transpose(0, 1)
        mask = torch.tensor(t[None, :] <= S[b] - n + np.arange(n)[:, None])
        want = torch.nn.functional.scaled_dot_product_attention(qb, kb, vb, attn_mask=mask, scale=-0.3)
        assert np.allclose(out[qsl[b]:qsl[b + 1]], want.transpose(0, 1).numpy())
        x = (qb @ kb.transpose(1, 2) * -0.3).masked_fill(~mask, -math.inf)
        assert np.allclose(lse[qsl[b]:qsl[b + 1]], torch.logsumexp(x, -1).T.numpy())
        assert np.allclose(mean[qsl[b]:qsl[b + 1]], (torch.softmax(x, -1) @ vb.abs()).transpose(0, 1).numpy())
        y = (qb.abs() @ kb.abs().transpose(1, 2) * 0.3).masked_fill(~mask, 0)
        assert np.allclose(most[qsl[b]:qsl[b + 1]], y.amax(-1).T.numpy())


def test_equal_keys_share_their_weight():
    """Zero scores: a row that sees s keys gives each 1 / s."""
    k, _, r = cache(4, 4, 1, 8, 1)
    q, tables = np.zeros((3, 2, 8)), np.array([[2, 0], [1, 3]])
    before = r.random((4, 1, 4))
    lse = np.log(np.array([[5.0] * 2, [6.0] * 2, [1.0] * 2]))
    got, size = osv.attention_weights(k, [0, 2, 3], [6, 1], tables, q, 1.0, lse, before)
    old = before[2, 0].tolist() + [0.0] * 2   # the cached four, then the step's two
    w = np.array([2 / 5 + 2 / 6] * 5 + [2 / 6]) + (old[:4] + [0, 0])
    assert np.allclose(np.concatenate([got[2, 0], got[0, 0, :2]]), w)
    assert got[1, 0, 0] == 2.0 and np.array_equal(got[3], before[3]) and np.array_equal(got[1, 0, 1:], before[1, 0, 1:])
    assert (size[3] == 0).all() and (size[2] > 0).all()
    # one accepted of two, and the first keys left as they were
    got, _ = osv.attention_weights(k, [0, 2, 3], [5, 1], tables, q, 1.0, lse, before, [0, 0], [4, 9])
    assert np.array_equal(got[2], before[2]) and np.allclose(got[0, 0, 0], 2 / 5) and np.array_equal(got[1], before[1])
    got, _ = osv.attention_weights(k, [0, 2, 3], [6, 1], tables, q, 1.0, lse, None)
    assert np.allclose(got.sum(), 3 * 2)


def test_eviction_keeps_the_front_the_end_and_the_most_weighty():
    k, v, _ = cache(3, 4, 1, 2, 2)
    tables = np.array([[2, 0, 1]])
    t = np.arange(10)
    blk, slot = tables[0, t // 4], t % 4
    w = np.zeros((3, 1, 4), np.float32)
    w[blk, 0, slot] = [9, 1, 5, np.nan, 5, 2, -np.inf, 5, 0, 0]
    for keep, first, last, src in ((5, 1, 2, [0, 2, 4, 8, 9]), (6, 0, 1, [0, 2, 4, 5, 7, 9]), (9, 2, 1, [0, 1, 2, 4, 5, 6, 7, 8, 9]),
                                   (3, 5, 4, [0, 1, 2]), (3, 0, 9, [7, 8, 9]), (0, 1, 1, []), (-4, 0, 0, []), (99, 0, 0, list(range(10)))):
        k2, v2, w2, m = osv.evict(k, v, w, [10], tables, [keep], [first], last)
        assert m.tolist() == [len(src)]
        to = np.arange(len(src))
        for a, b in ((k2, k), (v2, v), (w2.transpose(0, 2, 1), w.transpose(0, 2, 1))):
            assert np.array_equal(a[blk[to], slot[to]], b[blk[src], slot[src]], equal_nan=True)
