"""Plain 64-bit forms of the operators around the verification step (test infrastructure, like the rest of this
package): the rotary position embedding, appends into the 8-bit cache, attention over it, and token log
probabilities.  numpy on the host, from the definitions in include/spexis.h, in the caches' logical coordinates
[block][slot][KV head][dim]; `places8` is the only statement of the 8-bit layout.
"""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0
LEAST_EXP = -100
MOST = 240 * 2.0 ** 120   # the largest magnitude stored: the next code at that scale, 256, times 2^120 is infinity in bf16


# ------------------------------------------------------------------ e4m3 codes


def _e4m3_values() -> np.ndarray:
    """The value of every code: sign, exponent (bias 7), mantissa; no infinity, 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


E4M3 = _e4m3_values()
_POSITIVE = E4M3[:127]
_MIDDLE = (_POSITIVE[1:] + _POSITIVE[:-1]) / 2


def encode(x) -> np.ndarray:
    """e4m3 codes of x, to nearest, ties to the even code; beyond 448 the largest code, not finite: NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    lo, hi = np.searchsorted(_MIDDLE, a, side="left"), np.searchsorted(_MIDDLE, a, side="right")
    code = np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))   # lo != hi: a is half way between lo and hi
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def least_scale(most: float) -> float:
    """The least power of two, from 2^LEAST_EXP up, by which `most` is at most 448."""
    e = LEAST_EXP
    while most > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


# ------------------------------------------------------------------ the 8-bit cache's layout


def places8(num_blocks, hkv, bs, D):
    """Places in the flat K and V pools of element [block][slot][head][dim]."""
    blk, slot, h, d = np.ogrid[:num_blocks, :bs, :hkv, :D]
    units, unit, u = bs // 16, slot // 16, slot % 16
    base = (blk * hkv + h) * units + unit
    k = ((base * (D // 16) + d // 16) * 16 + u) * 16 + d % 16
    v = ((((base * (D // 64) + d // 64) * 32 + d % 32) * 2 + (u >> 2 & 1)) * 2 + (d >> 5 & 1)) * 8 + (u >> 3) * 4 + (u & 3)
    return k, v


# ------------------------------------------------------------------ rotation and appends


def rotate(x, cos_sin, positions, style) -> np.ndarray:
    """x [T][H][D] turned by its tokens' angles, in 64 bits."""
    y = np.array(x, dtype=np.float64)
    r = cos_sin.shape[1]
    for t, pos in enumerate(positions):
        for i in range(r // 2):
            a, b = (i, i + r // 2) if style == 0 else (2 * i, 2 * i + 1)
            c, s = float(cos_sin[pos, i]), float(cos_sin[pos, r // 2 + i])
            xa, xb = y[t, :, a].copy(), y[t, :, b].copy()
            y[t, :, a], y[t, :, b] = xa * c - xb * s, xb * c + xa * s
    return y


def token_positions(qsl, seq_lens) -> np.ndarray:
    return np.concatenate([np.arange(seq_lens[b] - (qsl[b + 1] - qsl[b]), seq_lens[b]) for b in range(len(seq_lens))])


def append8(codes, scales, qsl, seq_lens, tables, rows):
    """New rows [T][Hkv][D] (values to be stored) into codes [block][slot][Hkv][D] and scales [block][Hkv], in
    place; one of K and V."""
    bs, hkv = codes.shape[1], codes.shape[2]
    rows = np.asarray(rows, dtype=np.float64)
    rows = np.where(np.isfinite(rows), np.clip(rows, -MOST, MOST), rows)
    for b in range(len(seq_lens)):
        L = int(seq_lens[b]) - int(qsl[b + 1] - qsl[b])
        for t in range(L // bs, (int(seq_lens[b]) - 1) // bs + 1):
            lo, hi = max(L, t * bs), min(int(seq_lens[b]), (t + 1) * bs)
            if lo >= hi:
                continue
            blk, held = int(tables[b, t]), lo - t * bs
            new = rows[int(qsl[b]) + lo - L: int(qsl[b]) + hi - L]
            for h in range(hkv):
                x = new[:, h]
                fine = np.abs(x[np.isfinite(x)])
                s = least_scale(float(fine.max()) if fine.size else 0.0)
                if held:
                    old = float(scales[blk, h])
                    s = max(s, old)
                    if s != old:
                        codes[blk, :held, h] = encode(E4M3[codes[blk, :held, h]] * (old / s))
                scales[blk, h] = s
                codes[blk, held: held + hi - lo, h] = encode(x / s)


# ------------------------------------------------------------------ attention


def attention8(k_codes, v_codes, scales, qsl, seq_lens, tables, q, scale) -> np.ndarray:
    """Causal attention of every query token over its sequence; q [T][Hq][D]; scales [block][Hkv][2].  Also the
    weighted mean of |v| and the largest sum of |q_d k_d| * scale of a key, which errors are measured in."""
    hkv, D, bs = k_codes.shape[2], k_codes.shape[3], k_codes.shape[1]
    q = np.asarray(q, dtype=np.float64)
    out, mean, most = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    G = q.shape[1] // hkv
    for b in range(len(seq_lens)):
        S = int(seq_lens[b])
        n = int(qsl[b + 1] - qsl[b])
        if n == 0:
            continue
        ids = tables[b, : -(-S // bs)].astype(np.int64)
        s = scales[ids].astype(np.float64)
        k = (E4M3[k_codes[ids]] * s[:, None, :, 0, None]).reshape(-1, hkv, D)[:S]
        v = (E4M3[v_codes[ids]] * s[:, None, :, 1, None]).reshape(-1, hkv, D)[:S]
        for j in range(n):
            seen = S - n + j + 1
            for h in range(q.shape[1]):
                x = k[:seen, h // G] @ q[int(qsl[b]) + j, h] * scale
                p = np.exp(x - x.max())
                at = int(qsl[b]) + j, h
                out[at] = p @ v[:seen, h // G] / p.sum()
                mean[at] = p @ np.abs(v[:seen, h // G]) / p.sum()
                most[at] = (np.abs(k[:seen, h // G]) @ np.abs(q[at])).max() * abs(scale)
    return out, mean, most


# ------------------------------------------------------------------ log probabilities


def token_logprobs(logits, rows, tokens, temperature, top):
    """For every item: log softmax(logits[row] / T) at its token, the row's entropy, and the `top` largest by
    (logit, then the lower index).  No token (an id or row out of range): 0, 0, -1 and -inf.  A row without a
    distribution (NaN, +inf, or nothing above -inf): NaN, NaN, -1 and NaN."""
    logits = np.asarray(logits, dtype=np.float64)
    V = logits.shape[1]
    n = len(tokens)
    lp, entropy = np.zeros(n), np.zeros(n)
    ids, alt = np.full((n, top), -1, np.int32), np.full((n, top), -np.inf)
    for i in range(n):
        row = i if rows is None else int(rows[i])
        if not (0 <= tokens[i] < V and 0 <= row < logits.shape[0]):
            continue
        x = logits[row]
        m = x.max()
        if np.isnan(x).any() or not np.isfinite(m):
            lp[i], entropy[i], alt[i] = np.nan, np.nan, np.nan
            continue
        z = (x - m) / temperature
        e = np.exp(z)
        ln = np.log(e.sum())
        lp[i] = z[tokens[i]] - ln
        entropy[i] = ln - np.where(e > 0, e * np.where(e > 0, z, 0.0), 0.0).sum() / e.sum()
        order = np.argsort(-x, kind="stable")[:top]
        ids[i, : len(order)], alt[i, : len(order)] = order, z[order] - ln
    return lp, entropy, ids, alt
