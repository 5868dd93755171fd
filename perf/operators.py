"""What the serving operators around the verification step are measured on.

A case is a dict of plain values; its "kind" says which operator it calls:

  rotate    the position rotation of q and of the new keys, the new K/V rows into the bf16 cache
  rotate8   the same into a cache held in 8 bits, with a scale for each block of tokens and KV head
  attend8   verification attention over the 8-bit cache
  logprobs  log probabilities of given tokens, with the entropy and the top alternatives of their rows

With `own` false, `run` computes the operator in elementary torch operations; with `own` true it calls
this library.  Sizes are those of this repository's workloads and of the range between them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
HALVES, PAIRS = 0, 1      # which elements rotate together: (i, i + r/2), or (2i, 2i + 1)
LEAST_EXP = -100          # the least scale of the 8-bit cache is 2^-100
E4M3_MAX = 448.0

# a drawn case stays below the largest listed one of its kind
_MAX_ROWS_BYTES = 0.9e8
_MAX_CACHE_BYTES = 6.5e8
_MAX_LOGIT_BYTES = 2.5e9


def listed():
    return [
        # the step of an 8B model's ordinary batch (this repository's headline workload)
        dict(name="rotate_decode", kind="rotate", batch=64, hq=32, hkv=8, dim=128, block=16, ctx_lo=1024, ctx_hi=4096,
             n_lo=5, n_hi=5, rot=128, style=HALVES),
        # prompts: a few thousand new tokens a sequence, some of them behind a cached prefix of odd length
        dict(name="rotate_prompt", kind="rotate", batch=4, hq=28, hkv=4, dim=128, block=32, ctx_lo=0, ctx_hi=777,
             n_lo=2001, n_hi=4096, rot=128, style=HALVES),
        # a test or development server: launches and latency; half of a head rotated, in pairs
        dict(name="rotate8_tiny", kind="rotate8", batch=4, hq=8, hkv=2, dim=64, block=16, ctx_lo=32, ctx_hi=256,
             n_lo=5, n_hi=5, rot=32, style=PAIRS),
        # a large batch with many drafts (the acceptance-stress workload), blocks of 32
        dict(name="rotate8_decode", kind="rotate8", batch=512, hq=28, hkv=4, dim=128, block=32, ctx_lo=512,
             ctx_hi=2048, n_lo=9, n_hi=9, rot=128, style=HALVES),
        # prompts into the 8-bit cache, of very different lengths
        dict(name="rotate8_prompt", kind="rotate8", batch=8, hq=32, hkv=8, dim=128, block=16, ctx_lo=0, ctx_hi=300,
             n_lo=100, n_hi=3500, rot=128, style=HALVES),
        # one token a sequence, short caches: latency
        dict(name="attend8_token", kind="attend8", batch=4, hq=8, hkv=2, dim=64, block=16, ctx_lo=32, ctx_hi=256,
             n_lo=1, n_hi=1),
        # one user with a long document: a single sequence split over the whole chip
        dict(name="attend8_one_long", kind="attend8", batch=1, hq=32, hkv=8, dim=128, block=16, ctx_lo=16000,
             ctx_hi=16384, n_lo=5, n_hi=5),
        # the ordinary batch
        dict(name="attend8_batch", kind="attend8", batch=64, hq=32, hkv=8, dim=128, block=16, ctx_lo=1024,
             ctx_hi=4096, n_lo=5, n_hi=5),
        # the large batch: 63 query rows per KV head, blocks of 32, seven heads a group
        dict(name="attend8_stress", kind="attend8", batch=512, hq=28, hkv=4, dim=128, block=32, ctx_lo=512,
             ctx_hi=2048, n_lo=9, n_hi=9),
        # a development server's emitted tokens
        dict(name="logprobs_tiny", kind="logprobs", batch=4, n_lo=5, n_hi=5, vocab=1024, std=2.0, temp=1.0, top=5,
             type="f32", emitted=True),
        # the ordinary batch's emitted tokens with twenty alternatives: the rows behind a rejection are not asked for
        dict(name="logprobs_emitted", kind="logprobs", batch=64, n_lo=1, n_hi=9, vocab=128256, std=3.0, temp=1.0,
             top=20, type="f32", emitted=True),
        # scoring prompts: every row has its token
        dict(name="logprobs_score", kind="logprobs", batch=512, n_lo=9, n_hi=9, vocab=152064, std=4.0, temp=0.7,
             top=5, type="f32", emitted=False),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate8", "attend8", "attend8", "logprobs", "logprobs"])
    if kind == "logprobs":
        vocab = rng.choice([32000, 128256, 152064, _log(rng, 1000, 152064), _log(rng, 1000, 152064)])
        n_hi = rng.randint(1, 9)
        most = int(min(512, _MAX_LOGIT_BYTES / (n_hi * vocab * 4)))
        return dict(kind=kind, batch=_log(rng, 1, max(1, most)), n_lo=rng.choice([1, n_hi]), n_hi=n_hi, vocab=vocab,
                    std=rng.choice([2.0, 3.0, 4.0]), temp=rng.choice([1.0, 1.0, 0.7]), top=rng.choice([0, 1, 5, 20, 32]),
                    type=rng.choice(["f32", "f32", "bf16"]), emitted=rng.random() < 0.5)
    hkv, group, dim = rng.choice([2, 4, 8]), rng.choice([1, 4, 7, 8]), rng.choice([64, 128])
    c = dict(kind=kind, hq=hkv * group, hkv=hkv, dim=dim, block=rng.choice([16, 32]))
    if kind == "attend8":
        n_hi = rng.randint(1, min(9, 64 // group))
        batch = _log(rng, 1, 512)
        hi = _log(rng, 128, int(min(16384, _MAX_CACHE_BYTES / (batch * hkv * dim * 2))))
        return dict(c, batch=batch, ctx_lo=max(0, hi // 4), ctx_hi=hi, n_lo=rng.choice([1, n_hi]), n_hi=n_hi)
    c.update(rot=rng.choice([dim, dim, dim // 2, 16]), style=rng.choice([HALVES, HALVES, PAIRS]))
    if rng.random() < 0.5:   # a step
        batch, n_hi = _log(rng, 1, 512), rng.randint(1, 9)
        hi = _log(rng, 16, int(min(8192, _MAX_CACHE_BYTES / (batch * hkv * dim * 2))))
        return dict(c, batch=batch, ctx_lo=hi // 4, ctx_hi=hi, n_lo=rng.choice([1, n_hi]), n_hi=n_hi)
    batch = _log(rng, 1, 16)     # prompts
    n_hi = _log(rng, 30, int(min(8192, _MAX_ROWS_BYTES / (batch * (hkv * group + 2 * hkv) * dim * 2))))
    return dict(c, batch=batch, ctx_lo=0, ctx_hi=rng.choice([0, 300]), n_lo=max(1, n_hi // 4), n_hi=n_hi)


# ------------------------------------------------------------------------------------- inputs


def _sizes(case):
    """New tokens and cached tokens of each sequence: the same for every seed, in another order (_batch)."""
    fixed = np.random.default_rng(case["batch"])
    n = fixed.integers(case["n_lo"], case["n_hi"] + 1, size=case["batch"])
    ctx = fixed.integers(case.get("ctx_lo", 0), case.get("ctx_hi", 0) + 1, size=case["batch"])
    asked = fixed.integers(1, n + 1) if case.get("emitted") else n
    return n, ctx, asked


def _batch(case, seed):
    n, ctx, asked = _sizes(case)
    r = np.random.default_rng([int(seed), 7])
    order = r.permutation(case["batch"])
    n, ctx, asked = n[order], ctx[order], asked[order]
    qsl = np.zeros(case["batch"] + 1, dtype=np.int32)
    qsl[1:] = np.cumsum(n)
    return n, ctx, asked, qsl, r


def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 16 + stream)
    return g


def _randn_bf16(shape, g):
    return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)


def _to(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), device=DEV).to(dtype)


def _codes(count, g):
    """e4m3 codes of N(0, 64^2): with a scale of 2^-6, N(0, 1)."""
    out = torch.empty(count, dtype=torch.float8_e4m3fn, device=DEV)
    for s in range(0, count, 1 << 27):
        e = min(count, s + (1 << 27))
        out[s:e] = (torch.randn(e - s, generator=g, device=DEV) * 64.0).clamp_(-E4M3_MAX, E4M3_MAX).to(out.dtype)
    return out


def prepare(case, seed):
    n, ctx, asked, qsl, r = _batch(case, seed)
    st = dict(case=case)
    if case["kind"] == "logprobs":
        return _logits(st, case, seed, n, asked, qsl)
    S = ctx + n
    nblk = -(-S // case["block"])
    ends = np.cumsum(nblk)
    perm = r.permutation(int(nblk.sum())).astype(np.int32)
    tables = np.zeros((case["batch"], int(nblk.max())), dtype=np.int32)
    for b in range(case["batch"]):
        tables[b, : nblk[b]] = perm[ends[b] - nblk[b]: ends[b]]
    hq, hkv, dim, T, blocks = case["hq"], case["hkv"], case["dim"], int(qsl[-1]), int(nblk.sum())
    g = _gen(seed, 0)
    st.update(qsl=_to(qsl), seq_lens=_to(S), tables=_to(tables), T=T, max_n=int(n.max()), max_s=int(S.max()),
              blocks=blocks, q=_randn_bf16((T, hq, dim), g))
    cells = blocks * hkv * case["block"] * dim
    if case["kind"] == "rotate":
        st.update(k_pool=_randn_bf16((cells,), g), v_pool=_randn_bf16((cells,), g))
    else:
        # blocks and heads of different magnitude
        e = torch.randint(-7, -4, (blocks, hkv, 2), generator=g, device=DEV)
        st.update(k_pool=_codes(cells, g), v_pool=_codes(cells, g), scales=((e + 127).to(torch.int32) << 23).view(torch.float32))
    if case["kind"] == "attend8":
        st.update(out=torch.empty_like(st["q"]))
        return st
    st.update(new_k=_randn_bf16((T, hkv, dim), g), new_v=_randn_bf16((T, hkv, dim), g), q_out=torch.empty_like(st["q"]))
    # the angles' table as a model keeps it: cosines, then sines, of every position
    half = case["rot"] // 2
    inv = 500000.0 ** (-np.arange(half) / half)
    ang = np.arange(int(S.max()) + 1)[:, None] * inv[None, :]
    st["cos_sin"] = _to(np.concatenate([np.cos(ang), np.sin(ang)], axis=1), torch.float32)
    return st


def _logits(st, case, seed, n, asked, qsl):
    T, V, B, g = int(qsl[-1]), case["vocab"], case["batch"], _gen(seed, 1)
    dtype = torch.float32 if case["type"] == "f32" else torch.bfloat16
    x = torch.empty((T, V), dtype=dtype, device=DEV)
    ids = torch.empty(T, dtype=torch.int32, device=DEV)
    for s in range(0, T, 1024):
        e = min(T, s + 1024)
        x[s:e] = torch.randn((e - s, V), generator=g, device=DEV) * case["std"]
        # the tokens as a sampler draws them
        gumbel = torch.empty((e - s, V), device=DEV).exponential_(generator=g).log_().neg_()
        ids[s:e] = torch.argmax(x[s:e].float() / case["temp"] + gumbel, dim=1).to(torch.int32)
    st["logits"] = x
    if not case["emitted"]:
        st.update(tokens=ids, rows=None)
        return st
    # as acceptance leaves them: [B][most] tokens, -1 behind the last one emitted
    most = int(n.max())
    rows, j = qsl[:-1, None] + np.minimum(np.arange(most), n[:, None] - 1), np.arange(most)
    rows = _to(rows.reshape(-1))
    keep = _to((j[None, :] < asked[:, None]).reshape(-1), torch.bool)
    st.update(rows=rows, tokens=torch.where(keep, ids[rows.long()], -1).to(torch.int32))
    return st


# ------------------------------------------------------------------------------------- plain forms


def _new_positions(st):
    """Sequence, position, block and slot of every new token."""
    tok = torch.arange(st["T"], device=DEV)
    b = torch.searchsorted(st["qsl"][1:].long(), tok, right=True)
    pos = st["seq_lens"].long()[b] - st["qsl"].long()[b + 1] + tok
    bs = st["case"]["block"]
    return b, pos, st["tables"].long()[b, pos // bs], pos % bs


def _rotated(x, st, pos):
    """In 64 bits (what is rounded next is often next to a border of 8 bits), rounded to 32."""
    r, half = st["case"]["rot"], st["case"]["rot"] // 2
    y = x.double()
    cs = st["cos_sin"][pos].double()[:, None, :]
    c, s = cs[..., :half], cs[..., half:]
    if st["case"]["style"] == HALVES:
        a, b = y[..., :half], y[..., half:r]
        head = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        head = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([head, y[..., r:]], dim=-1).float()


def _cells(case, blk, slot):
    """Places of rows (blk, slot) in the pools: K, V as [rows, hkv, dim]."""
    hkv, D, bs = case["hkv"], case["dim"], case["block"]
    h, d = torch.arange(hkv, device=DEV)[None, :, None], torch.arange(D, device=DEV)[None, None, :]
    at, s = blk[:, None, None] * hkv + h, slot[:, None, None]
    if case["kind"] == "rotate":
        swapped = (s & ~12) | ((s >> 2 & 1) << 3) | ((s >> 3 & 1) << 2)
        return ((at * (D // 8) + d // 8) * bs + s) * 8 + d % 8, (at * D + d) * bs + swapped
    unit, u = at * (bs // 16) + s // 16, s % 16
    k = ((unit * (D // 16) + d // 16) * 16 + u) * 16 + d % 16
    v = ((((unit * (D // 64) + d // 64) * 32 + d % 32) * 2 + (u >> 2 & 1)) * 2 + (d >> 5 & 1)) * 8 + (u >> 3) * 4 + (u & 3)
    return k, v


def _least_scale(most):
    """The least power of two (from 2^LEAST_EXP) by which `most` is at most E4M3_MAX."""
    m, e = torch.frexp(most)
    e = torch.where(m <= 0.875, e - 9, e - 8)          # E4M3_MAX = 0.875 * 2^9
    e = torch.where(most > 0, e, LEAST_EXP).clamp(min=LEAST_EXP)
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _plain_rotate(st):
    _, pos, blk, slot = _new_positions(st)
    at_k, at_v = _cells(st["case"], blk, slot)
    st["k_pool"][at_k] = _rotated(st["new_k"], st, pos).to(torch.bfloat16)
    st["v_pool"][at_v] = st["new_v"]
    return _rotated(st["q"], st, pos).to(torch.bfloat16), st["k_pool"], st["v_pool"]


def _plain_append8(st, x, pool, scale, at, b, pos, blk, slot, places):
    """One of K and V: new scales [blocks][hkv] of the blocks that get new rows, then the codes."""
    case, raw = st["case"], pool.view(torch.uint8)
    hkv, bs = case["hkv"], case["block"]
    mag = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dim=-1)
    key = (blk[:, None] * hkv + torch.arange(hkv, device=DEV)).reshape(-1)
    most = torch.zeros(scale.numel(), device=DEV).scatter_reduce_(0, key, mag.reshape(-1), "amax").view_as(scale)
    first = torch.full((scale.shape[0],), bs, device=DEV).scatter_reduce_(0, blk, slot, "amin")[:, None]
    need = _least_scale(most)
    new = torch.where(first == bs, scale, torch.where(first > 0, torch.maximum(scale, need), need))
    # the rows that a sequence's first touched block held before
    n = (st["qsl"][1:] - st["qsl"][:-1]).long()
    L = st["seq_lens"].long() - n
    fb = st["tables"].long()[torch.arange(len(n), device=DEV), L // bs]
    old_at = places(fb[:, None].expand(-1, bs).reshape(-1), torch.arange(bs, device=DEV).repeat(len(n)))[at]
    old = raw[old_at]                                                   # [B * bs, hkv, dim]
    ratio = (scale / new)[fb].repeat_interleave(bs, dim=0)[:, :, None]
    held = (torch.arange(bs, device=DEV)[None, :] < (L % bs)[:, None]).reshape(-1, 1, 1)
    again = (old.view(torch.float8_e4m3fn).float() * ratio).to(torch.float8_e4m3fn).view(torch.uint8)
    raw[old_at] = torch.where(held & (ratio != 1), again, old)
    raw[places(blk, slot)[at]] = (x / new[blk][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    scale.copy_(new)


def _plain_rotate8(st):
    b, pos, blk, slot = _new_positions(st)
    places = lambda blk, slot: _cells(st["case"], blk, slot)  # noqa: E731
    for at, x in enumerate((_rotated(st["new_k"], st, pos), st["new_v"].float())):
        _plain_append8(st, x, st["v_pool" if at else "k_pool"], st["scales"][:, :, at], at, b, pos, blk, slot, places)
    return _rotated(st["q"], st, pos).to(torch.bfloat16), st["k_pool"], st["v_pool"], st["scales"]


def _rows_of_blocks(st):
    """K and V of every block as [blocks, slots, hkv, dim], in 32 bits."""
    case = st["case"]
    hkv, D, u = case["hkv"], case["dim"], case["block"] // 16
    k = st["k_pool"].float().view(-1, hkv, u, D // 16, 16, 16).permute(0, 2, 4, 1, 3, 5).reshape(-1, u * 16, hkv, D)
    v = st["v_pool"].float().view(-1, hkv, u, D // 64, 32, 2, 2, 2, 4)   # dim / 64, dim % 32, slot bit 2, dim bit 5, slot bit 3, slot % 4
    v = v.permute(0, 2, 7, 5, 8, 1, 3, 6, 4).reshape(-1, u * 16, hkv, D)
    s = st["scales"][:, None, :, :, None]
    return k * s[..., 0, :], v * s[..., 1, :]


def _plain_attend8(st):
    case = st["case"]
    B, hkv, G, D, T = case["batch"], case["hkv"], case["hq"] // case["hkv"], case["dim"], st["T"]
    k, v = _rows_of_blocks(st)
    k, v = k[st["tables"].long()].flatten(1, 2), v[st["tables"].long()].flatten(1, 2)    # [B, keys, hkv, dim]
    j, n = torch.arange(st["max_n"], device=DEV), (st["qsl"][1:] - st["qsl"][:-1]).long()
    row = (st["qsl"][:-1].long()[:, None] + j).clamp(max=T - 1)                          # [B, most]
    q = st["q"].float()[row].view(B, -1, hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, D)
    x = torch.matmul(q.contiguous(), k.permute(0, 2, 3, 1).contiguous()) * D ** -0.5     # [B, hkv, most * G, keys]
    last = (st["seq_lens"].long() - n)[:, None] + j                                      # the last key a token sees
    seen = torch.arange(x.shape[-1], device=DEV) <= last.repeat_interleave(G, dim=1)[:, None, :, None]
    x = torch.where(seen, x, -math.inf)
    p = torch.exp(x - x.amax(dim=-1, keepdim=True))
    v = torch.where((torch.arange(v.shape[1], device=DEV) < st["seq_lens"][:, None])[..., None, None], v, 0.0)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()) / p.sum(dim=-1, keepdim=True)
    o = o.view(B, hkv, -1, G, D).permute(0, 2, 1, 3, 4).reshape(B, -1, hkv * G, D)
    tok = torch.arange(T, device=DEV)
    b = torch.searchsorted(st["qsl"][1:].long(), tok, right=True)
    return o[b, tok - st["qsl"].long()[b]].to(torch.bfloat16)


def _order(x):
    """Whole numbers in the order of x, equal values by the lowest index first."""
    bits = (x.float() + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return (bits << 32) - torch.arange(x.shape[-1], device=x.device)


def _plain_logprobs(st):
    case, x, rows, tok = st["case"], st["logits"], st["rows"], st["tokens"].long()
    top = min(case["top"], case["vocab"])
    z = x.float()
    m = z.amax(dim=1, keepdim=True)
    z = (z - m) / case["temp"]
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    entropy = torch.log(total) - (e * z).sum(dim=1, keepdim=True) / total
    key = torch.topk(_order(x), top, dim=1).values
    ids = -key & 0xFFFFFFFF
    z = z - torch.log(total)
    if rows is not None:
        z, entropy, ids = z[rows.long()], entropy[rows.long()], ids[rows.long()]
    none = tok[:, None] < 0
    lp = torch.where(none, 0.0, z.gather(1, tok.clamp(min=0)[:, None]))[:, 0]
    alt = torch.where(none, -math.inf, z.gather(1, ids))
    return lp, torch.where(none, 0.0, entropy)[:, 0], torch.where(none, -1, ids).to(torch.int32), alt


# ------------------------------------------------------------------------------------- the library's calls


def _space(st, size):
    """A workspace, as a program keeps one beside its buffers."""
    if "space" not in st:
        st["space"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
    return st["space"]


def _own(st):
    from paper_2609_34370_amd import spexis as sx
    case = st["case"]
    kind = case["kind"]
    if kind == "logprobs":
        items, top = st["tokens"].shape[0], case["top"]
        if "lp" not in st:
            st.update(lp=torch.empty(items, device=DEV), entropy=torch.empty(items, device=DEV),
                      ids=torch.empty((items, top), dtype=torch.int32, device=DEV), alt=torch.empty((items, top), device=DEV))
        space = _space(st, sx.spexis_token_logprobs_workspace_size(items, case["vocab"], top))
        sx.spexis_token_logprobs(st["logits"], st["tokens"], st["lp"], space, row_ids=st["rows"], entropy=st["entropy"],
                                 top_ids=st["ids"], top_logprobs=st["alt"], temperature=case["temp"])
        return st["lp"], st["entropy"], st["ids"], st["alt"]
    where = (st["blocks"], case["hkv"], case["block"], case["dim"], st["qsl"], st["seq_lens"], st["tables"], st["T"], st["max_n"])
    if kind == "attend8":
        space = _space(st, sx.spexis_verify_attention_kv8_workspace_size(
            case["batch"], case["hq"], case["hkv"], case["dim"], st["max_n"], st["max_s"]))
        sx.spexis_verify_attention_kv8(st["k_pool"], st["v_pool"], st["scales"], *where, st["max_s"], st["q"], case["hq"],
                                       case["dim"] ** -0.5, st["out"], space)
        return st["out"]
    rotation = dict(cos_sin=st["cos_sin"], style=case["style"], q=st["q"], q_out=st["q_out"])
    if kind == "rotate":
        sx.spexis_rotate_append_kv(st["k_pool"], st["v_pool"], *where, st["new_k"], st["new_v"], **rotation)
        return st["q_out"], st["k_pool"], st["v_pool"]
    sx.spexis_rotate_append_kv8(st["k_pool"], st["v_pool"], st["scales"], *where, st["new_k"], st["new_v"], **rotation)
    return st["q_out"], st["k_pool"], st["v_pool"], st["scales"]


def run(st):
    if own:
        return _own(st)
    return {"rotate": _plain_rotate, "rotate8": _plain_rotate8, "attend8": _plain_attend8,
            "logprobs": _plain_logprobs}[st["case"]["kind"]](st)


def work(case):
    n, ctx, asked = _sizes(case)
    T, S = int(n.sum()), int((n + ctx).sum())
    if case["kind"] == "logprobs":
        size = 4 if case["type"] == "f32" else 2
        items = case["batch"] * int(n.max()) if case["emitted"] else T
        rows, V = int(asked.sum()), case["vocab"]
        return {"bytes": rows * V * size + items * (4 + 8 + 8 * case["top"]) + (items * 4 if case["emitted"] else 0),
                "flops": 6 * rows * V}
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    blocks = -(-(n + ctx) // case["block"])
    meta = 8 * case["batch"] + 4
    if case["kind"] == "attend8":
        pairs = float((n * ctx + n * (n + 1) // 2).sum())     # (query token, key it sees)
        return {"bytes": S * hkv * dim * 2 + int(blocks.sum()) * (8 * hkv + 4) + T * hq * dim * 4 + meta,
                "flops": 4 * pairs * hq * dim}
    touched = int((blocks - ctx // case["block"]).sum())
    size = 2 if case["kind"] == "rotate" else 1
    scales = 0 if size == 2 else touched * hkv * 8
    # a position's row of the table is used by every sequence that has a new token there
    at = np.concatenate([np.arange(c, c + k) for c, k in zip(ctx, n)])
    table = len(np.unique(at)) * case["rot"] * 4
    return {"bytes": T * (hq * 4 + hkv * 2 * (2 + size)) * dim + table + scales + touched * 4 + meta,
            "flops": 3 * T * (hq + hkv) * case["rot"]}


# ------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "logprobs":
        return _exact_logprobs(case, st)
    qsl, S, tables = (st[n].cpu().numpy() for n in ("qsl", "seq_lens", "tables"))
    if case["kind"] == "attend8":
        return _exact_attend8(case, st, qsl, S, tables)
    return _exact_append(case, st, qsl, S, tables)


def _turned(x, cos_sin, pos, rot, style):
    """The rotation as a product with complex numbers."""
    cs = cos_sin.double()[pos][:, None, :]
    w = torch.complex(cs[..., : rot // 2], cs[..., rot // 2:])
    x = x.double()
    if style == HALVES:
        y = torch.view_as_real(torch.complex(x[..., : rot // 2], x[..., rot // 2: rot]) * w).transpose(-1, -2)
    else:
        y = torch.view_as_real(torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * w)
    return torch.cat([y.flatten(-2), x[..., rot:]], dim=-1)


def _exact_append(case, st, qsl, S, tables):
    """Sequence by sequence and block by block of the pools, in the pools' layouts."""
    hkv, D, bs, rot, style = case["hkv"], case["dim"], case["block"], case["rot"], case["style"]
    in8 = case["kind"] == "rotate8"
    pos = np.concatenate([np.arange(S[b] - (qsl[b + 1] - qsl[b]), S[b]) for b in range(len(S))])
    at = torch.as_tensor(pos, device=DEV)
    q = _turned(st["q"], st["cos_sin"], at, rot, style)
    new = [_turned(st["new_k"], st["cos_sin"], at, rot, style), st["new_v"].double()]
    # views of the pools with the axes (block, head, slot in three parts, dim in parts)
    if in8:
        shapes = [(-1, hkv, bs // 16, D // 16, 16, 16), (-1, hkv, bs // 16, D // 64, 32, 2, 2, 2, 4)]
        axes = [(0, 1, 2, 4, 3, 5), (0, 1, 2, 7, 5, 8, 3, 6, 4)]
    else:
        shapes = [(-1, hkv, D // 8, bs, 8), (-1, hkv, D, bs // 16, 2, 2, 4)]
        axes = [(0, 1, 3, 2, 4), (0, 1, 3, 5, 4, 6, 2)]
    out, scales = [q], st["scales"].double().clone() if in8 else None
    for part, name in enumerate(("k_pool", "v_pool")):
        pool = st[name].double()
        back = np.argsort(axes[part]).tolist()
        rows = pool.view(shapes[part]).permute(axes[part])
        moved = rows.shape
        rows = rows.reshape(-1, hkv, bs, D).clone()
        for b in range(len(S)):
            n = int(qsl[b + 1] - qsl[b])
            L = int(S[b]) - n
            lo, hi = L // bs, -(-int(S[b]) // bs)
            ids = torch.as_tensor(tables[b, lo:hi].astype(np.int64), device=DEV)
            x = rows[ids].transpose(1, 2).reshape(-1, hkv, D)                     # [slots, hkv, dim]
            fresh = new[part][int(qsl[b]): int(qsl[b + 1])]
            held = L - lo * bs
            if not in8:
                x[held: held + n] = fresh
            else:
                size = torch.zeros_like(x)
                size[held: held + n] = fresh.abs()
                size = size.view(hi - lo, bs, hkv, D).amax(dim=(1, 3))
                s = torch.exp2(torch.ceil(torch.log2(size / E4M3_MAX)).clamp(min=LEAST_EXP))
                before = scales[ids, :, part]
                if held:
                    s[0] = torch.maximum(s[0], before[0])
                    x[:held] *= (before[0] / s[0])[:, None]
                scales[ids, :, part] = s
                x[held: held + n] = fresh / s.repeat_interleave(bs, dim=0)[held: held + n, :, None]
            rows[ids] = x.view(hi - lo, bs, hkv, D).transpose(1, 2)
        out.append(rows.view(moved).permute(back).reshape(-1))
    return tuple(out) + ((scales,) if in8 else ())


def _exact_attend8(case, st, qsl, S, tables):
    hkv, G, D, bs = case["hkv"], case["hq"] // case["hkv"], case["dim"], case["block"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    k_pool = st["k_pool"].view(-1, hkv, bs // 16, D // 16, 16, 16)
    v_pool = st["v_pool"].view(-1, hkv, bs // 16, D // 64, 32, 2, 2, 2, 4)
    for b in range(len(S)):
        n = int(qsl[b + 1] - qsl[b])
        ids = torch.as_tensor(tables[b, : -(-int(S[b]) // bs)].astype(np.int64), device=DEV)
        s = st["scales"][ids].double()
        k = k_pool.view(torch.uint8)[ids].view(torch.float8_e4m3fn).double().permute(1, 0, 2, 4, 3, 5).reshape(hkv, len(ids), bs, D)
        v = v_pool.view(torch.uint8)[ids].view(torch.float8_e4m3fn).double().permute(1, 0, 2, 7, 5, 8, 3, 6, 4).reshape(hkv, len(ids), bs, D)
        k = (k * s[:, :, 0].t()[:, :, None, None]).reshape(hkv, -1, D)[:, : int(S[b])]
        v = (v * s[:, :, 1].t()[:, :, None, None]).reshape(hkv, -1, D)[:, : int(S[b])]
        q = st["q"][int(qsl[b]): int(qsl[b + 1])].double().view(n, hkv, G, D).permute(1, 0, 2, 3).reshape(hkv, n * G, D)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        key = torch.arange(int(S[b]), device=DEV)
        lim = int(S[b]) - n + torch.arange(n, device=DEV).repeat_interleave(G)
        x = x.masked_fill(key[None, None, :] > lim[None, :, None], -math.inf)
        o = torch.matmul(torch.softmax(x, dim=-1), v)
        out[int(qsl[b]): int(qsl[b + 1])] = o.view(hkv, n, G, D).permute(1, 0, 2, 3).reshape(n, hkv * G, D)
    return out


def _exact_logprobs(case, st):
    items, top, tok = st["tokens"].shape[0], case["top"], st["tokens"].long()
    f64 = dict(dtype=torch.float64, device=DEV)
    lp, entropy, alt = torch.zeros(items, **f64), torch.zeros(items, **f64), torch.full((items, top), -math.inf, **f64)
    where = torch.nonzero(tok >= 0)[:, 0]
    for part in torch.split(where, 512):
        rows = st["rows"].long()[part] if st["rows"] is not None else part
        y = torch.log_softmax(st["logits"][rows].double() / case["temp"], dim=1)
        lp[part] = y[torch.arange(len(part), device=DEV), tok[part]]
        entropy[part] = -(torch.exp(y) * y).sum(dim=1)
        alt[part] = torch.topk(y, top, dim=1).values
    return lp, entropy, None, alt
