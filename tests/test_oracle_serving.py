"""What pins the plain forms of oracle/serving.py, and the documented shape of the 8-bit cache."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as osv


def test_e4m3_codes_agree_with_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(osv.E4M3, want, equal_nan=True)
    assert np.array_equal(osv.encode(osv.E4M3[:127]), codes[:127])
    x = np.random.default_rng(0).uniform(-448, 448, 20000).astype(np.float32) * 2.0 ** -(np.arange(20000) % 19)
    x = np.concatenate([x, (osv._MIDDLE).astype(np.float32), -osv._MIDDLE.astype(np.float32)]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(osv.encode(x), want)
    assert osv.encode([math.inf, -math.inf, math.nan]).tolist() == [127] * 3


def test_least_scale_is_the_least():
    for most in (0.0, 1.0, 448.0, 448.0001, 224.0, 1e-3, 3e38, 2.0 ** -130):
        s = osv.least_scale(most)
        assert most <= 448 * s and (s == 2.0 ** osv.LEAST_EXP or most > 448 * s / 2)


@pytest.mark.parametrize("bs,D,hkv", [(16, 64, 3), (32, 64, 1), (16, 128, 2), (32, 128, 2)])
def test_the_8_bit_layout_is_a_bijection_with_16_byte_operands(bs, D, hkv):
    k, v = osv.places8(3, hkv, bs, D)
    for p in (k, v):
        assert np.array_equal(np.sort(p.reshape(-1)), np.arange(3 * hkv * bs * D))
    # 16 dims of a slot, and 8 slots of dims d and d + 32, are 16 contiguous bytes
    assert (np.diff(k[1, 3, 0, 16:32]) == 1).all() and k[1, 3, 0, 16] % 16 == 0
    eight = [0, 1, 2, 3, 8, 9, 10, 11]
    assert (np.diff(v[1, eight, 0, 5]) == 1).all() and v[1, 0, 0, 5] % 16 == 0
    assert (v[1, eight, 0, 37] == v[1, eight, 0, 5] + 8).all()


def test_rotation_keeps_lengths_and_differences():
    """A rotated pair keeps its length, and <rotate(q, m), rotate(k, n)> depends on m - n alone."""
    r = np.random.default_rng(1)
    inv = 10000.0 ** (-np.arange(8) / 8)
    ang = np.arange(64)[:, None] * inv
    table = np.concatenate([np.cos(ang), np.sin(ang)], axis=1)
    q, k = r.standard_normal((1, 1, 64)), r.standard_normal((1, 1, 64))
    for style in (0, 1):
        dots = [(osv.rotate(q, table, [m], style) * osv.rotate(k, table, [m + 7], style)).sum() for m in (0, 5, 50)]
        assert np.allclose(dots, dots[0], atol=1e-12)
        y = osv.rotate(q, table, [13], style)
        assert np.allclose((y ** 2).sum(), (q ** 2).sum()) and np.array_equal(y[..., 16:], q[..., 16:])
    assert np.array_equal(osv.rotate(q, table, [0], 0), q)


def test_append8_keeps_what_a_block_held():
    """A later row of 2^6 times the size re-codes the block's earlier rows, within half a step of the new scale."""
    r = np.random.default_rng(2)
    codes, scales = np.full((2, 16, 1, 64), 0x55, np.uint8), np.full((2, 1), 7.0, np.float32)
    first, second = r.standard_normal((3, 1, 64)), 64 * r.standard_normal((2, 1, 64))
    tables = np.array([[1, 0]])
    osv.append8(codes, scales, [0, 3], [3], tables, first)
    s0 = float(scales[1, 0])
    assert s0 == osv.least_scale(np.abs(first).max()) and (codes[1, 3:] == 0x55).all() and (codes[0] == 0x55).all()
    before = osv.E4M3[codes[1, :3, 0]] * s0
    assert (np.abs(before - first[:, 0]) <= 2.0 ** -4 * np.abs(first[:, 0]) + 2.0 ** -10 * s0).all()
    osv.append8(codes, scales, [0, 2], [5], tables, second)
    s1 = float(scales[1, 0])
    assert s1 > s0
    after = osv.E4M3[codes[1, :3, 0]] * s1
    assert (np.abs(after - before) <= 2.0 ** -10 * s1).all()
    again = codes.copy()
    osv.append8(codes, scales, [0, 2], [5], tables, second)   # the same rows again: nothing changes
    assert np.array_equal(codes, again) and scales[1, 0] == s1


def test_attention8_is_a_mean_under_equal_scores():
    r = np.random.default_rng(3)
    v = r.integers(0, 120, (2, 16, 1, 64)).astype(np.uint8)
    scales = np.array([[[1.0, 2.0]], [[4.0, 0.5]]], dtype=np.float32)
    out, mean, most = osv.attention8(np.zeros_like(v), v, scales, [0, 2], [20], np.array([[1, 0]]), r.standard_normal((2, 3, 64)), 0.1)
    rows = np.concatenate([osv.E4M3[v[1, :, 0]] * 0.5, osv.E4M3[v[0, :, 0]] * 2.0])
    for j in range(2):
        assert np.allclose(out[j], rows[: 19 + j].mean(axis=0)) and np.array_equal(out, mean) and not most.any()


def test_logprobs_closed_forms():
    x = np.zeros((4, 8))
    x[1, :4] = -math.inf
    x[2, 3] = math.nan
    x[3] = -math.inf
    lp, h, ids, alt = osv.token_logprobs(x, [0, 1, 1, 2, 3, 9], [5, 5, 1, 0, 0, 0], 0.5, 3)
    assert np.allclose(lp[:2], [-math.log(8), -math.log(4)]) and lp[2] == -math.inf
    assert np.allclose(h[:3], [math.log(8), math.log(4), math.log(4)])
    assert ids[0].tolist() == [0, 1, 2] and ids[1].tolist() == [4, 5, 6] and ids[5].tolist() == [-1] * 3
    assert np.isnan(lp[3:5]).all() and np.isnan(h[3:5]).all() and lp[5] == 0 and (alt[5] == -math.inf).all()
    y = np.random.default_rng(4).standard_normal((1, 50))
    lp, h, ids, alt = osv.token_logprobs(y, None, [7], 0.7, 60)
    p = np.exp(y[0] / 0.7) / np.exp(y[0] / 0.7).sum()
    assert np.isclose(lp[0], math.log(p[7])) and np.isclose(h[0], -(p * np.log(p)).sum())
    assert sorted(ids[0, :50]) == list(range(50)) and (ids[0, 50:] == -1).all() and (np.diff(alt[0, :50]) <= 0).all()
