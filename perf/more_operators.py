"""What the operators that fill, share and thin out the paged cache are measured on.

A case is a dict of plain values; its "kind" says which operator it calls:

  prompt   causal attention of whole prompts (any number of new tokens a sequence) over the paged cache
  shared   verification attention of a batch whose sequences begin with a prefix that they share, group by group
  weights  the softmax weight that every cached key gets from the query rows, added up for each KV head
  evict    the keys of least accumulated weight leave the cache, the others move together

"in8" holds the cache in 8 bits.  With `own` false, `run` computes the operator in elementary torch operations; with
`own` true it calls this library.  Sizes are those of this repository's workloads and of the range between them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0
_CHUNK = 1 << 28           # scores that the plain forms hold at a time

# a drawn case stays below the largest listed one of its kind
_MAX_FLOPS = dict(prompt=2.0e12, shared=1.0e12, weights=1.0e11, evict=1.0)
_MAX_CACHE_BYTES = dict(prompt=6.0e8, shared=6.0e8, weights=6.0e8, evict=6.0e8)


def listed():
    return [
        # a test or development server's prompts: launches and latency
        dict(name="prompt_tiny", kind="prompt", in8=False, batch=4, hq=8, hkv=2, dim=64, block=16, ctx_lo=0, ctx_hi=100,
             n_lo=5, n_hi=60, lse=False),
        # new requests of very different lengths packed into one pass, some behind a cached turn of the conversation
        dict(name="prompt_packed", kind="prompt", in8=False, batch=8, hq=32, hkv=8, dim=128, block=16, ctx_lo=0,
             ctx_hi=300, n_lo=100, n_hi=3500, lse=True),
        # one long document
        dict(name="prompt_long", kind="prompt", in8=False, batch=1, hq=32, hkv=8, dim=128, block=16, ctx_lo=0, ctx_hi=0,
             n_lo=16001, n_hi=16001, lse=False),
        # a chunk of a long prompt whose earlier chunks are cached: few rows, many keys
        dict(name="prompt_chunk", kind="prompt", in8=False, batch=1, hq=28, hkv=4, dim=128, block=32, ctx_lo=15001,
             ctx_hi=15001, n_lo=257, n_hi=257, lse=False),
        # prompts over the cache held in 8 bits
        dict(name="prompt8_packed", kind="prompt", in8=True, batch=4, hq=64, hkv=8, dim=128, block=16, ctx_lo=0,
             ctx_hi=777, n_lo=700, n_hi=2500, lse=False),
        # the development server's batch behind one short instruction
        dict(name="shared_tiny", kind="shared", in8=False, batch=4, hq=8, hkv=2, dim=64, block=16, groups=1, pre_lo=160,
             pre_hi=160, ctx_lo=3, ctx_hi=100, n_lo=5, n_hi=5, lse=False),
        # the ordinary batch's verification step behind one long instruction
        dict(name="shared_batch", kind="shared", in8=False, batch=64, hq=32, hkv=8, dim=128, block=16, groups=1,
             pre_lo=4096, pre_hi=4096, ctx_lo=64, ctx_hi=1024, n_lo=5, n_hi=5, lse=True),
        # many answers to each of sixteen problems (rollouts), the cache in 8 bits, blocks of 32
        dict(name="shared8_groups", kind="shared", in8=True, batch=512, hq=28, hkv=4, dim=128, block=32, groups=16,
             pre_lo=512, pre_hi=2048, ctx_lo=30, ctx_hi=600, n_lo=9, n_hi=9, lse=False),
        # a verification step's accepted tokens
        dict(name="weights_step", kind="weights", batch=64, hq=32, hkv=8, dim=128, block=16, ctx_lo=1024, ctx_hi=4096,
             n_lo=5, n_hi=5, accepted=True, add=True),
        # the last tokens of fresh prompts, whose attention says what of a prompt is kept
        dict(name="weights_window", kind="weights", batch=6, hq=28, hkv=4, dim=128, block=32, ctx_lo=2001, ctx_hi=8000,
             n_lo=64, n_hi=64, accepted=False, add=False),
        # one long conversation cut to a quarter
        dict(name="evict_one", kind="evict", batch=1, hkv=8, dim=128, block=16, ctx_lo=16001, ctx_hi=16001, keep_lo=0.25,
             keep_hi=0.25, first=4, last=256),
        # the ordinary batch cut to about a half
        dict(name="evict_batch", kind="evict", batch=64, hkv=8, dim=128, block=16, ctx_lo=1024, ctx_hi=4096, keep_lo=0.4,
             keep_hi=0.6, first=16, last=128),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    hi = max(lo, int(hi))
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "shared", "shared", "weights", "evict"])
    hkv, group, dim, block = rng.choice([2, 4, 8]), rng.choice([1, 4, 7, 8]), rng.choice([64, 128]), rng.choice([16, 32])
    c = dict(kind=kind, hq=hkv * group, hkv=hkv, dim=dim, block=block)
    keys = _MAX_CACHE_BYTES[kind] / (hkv * dim * 4)       # of all sequences together
    pairs = _MAX_FLOPS[kind] / (4 * hkv * group * dim)    # (query token, key) of all sequences together
    if kind == "prompt":
        batch = _log(rng, 1, 16)
        n_hi = _log(rng, 8, min(16384, math.sqrt(pairs / batch)))
        ctx = rng.choice([0, 300, _log(rng, 64, 16384)])
        ctx = int(min(ctx, keys / batch - n_hi, pairs / (batch * n_hi) - n_hi / 2))
        return dict(c, in8=rng.random() < 0.3, batch=batch, ctx_lo=max(0, ctx) // 2, ctx_hi=max(0, ctx), n_lo=max(1, n_hi // 4),
                    n_hi=n_hi, lse=rng.random() < 0.5)
    if kind == "shared":
        batch, n_hi = _log(rng, 2, 512), rng.randint(1, min(9, 64 // group))
        groups = _log(rng, 1, min(batch, 32))
        pre = _log(rng, 64, min(16384, keys / (2 * groups), pairs / (batch * n_hi) / 2))
        ctx = _log(rng, 8, min(4096, keys / (2 * batch), pairs / (batch * n_hi) / 2))
        return dict(c, in8=rng.random() < 0.4, batch=batch, groups=groups, pre_lo=pre // 2, pre_hi=pre, ctx_lo=ctx // 8,
                    ctx_hi=ctx, n_lo=rng.choice([1, n_hi]), n_hi=n_hi, lse=rng.random() < 0.5)
    if kind == "weights":
        batch = _log(rng, 1, 256)
        n_hi = rng.choice([rng.randint(1, 9), _log(rng, 10, 128)])
        hi = _log(rng, 128, min(16384, keys / batch, pairs / (batch * n_hi)))
        return dict(c, batch=batch, ctx_lo=hi // 4, ctx_hi=hi, n_lo=rng.choice([1, n_hi]), n_hi=n_hi,
                    accepted=rng.random() < 0.5, add=rng.random() < 0.5)
    batch = _log(rng, 1, 256)
    hi = _log(rng, 128, min(16384, keys / batch))
    keep = rng.uniform(0.1, 0.9)
    del c["hq"]
    return dict(c, batch=batch, ctx_lo=hi // 4, ctx_hi=hi, keep_lo=0.9 * keep, keep_hi=keep, first=rng.choice([0, 4, 16, 100]),
                last=rng.choice([0, 1, 32, 128]))


# ------------------------------------------------------------------------------------- inputs


def _sizes(case):
    """Of each sequence: query tokens, tokens before them, the ones that count; of each group of sequences: its first
    sequence and its prefix.  The same for every seed, in another order (_batch)."""
    B = case["batch"]
    fixed = np.random.default_rng(B)
    n = fixed.integers(case.get("n_lo", 0), case.get("n_hi", 0) + 1, size=B)
    ctx = fixed.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=B)
    used = fixed.integers(1, n + 1) if case.get("accepted") else n
    start = np.zeros(0, dtype=np.int64)
    pre = np.zeros(0, dtype=np.int64)
    if case["kind"] == "shared":
        start = np.arange(case["groups"]) * B // case["groups"]
        pre = fixed.integers(case["pre_lo"], case["pre_hi"] + 1, size=case["groups"]) // case["block"] * case["block"]
        ctx = ctx + np.repeat(pre, np.diff(np.append(start, B)))
    keep = np.maximum(1, (ctx * fixed.uniform(case.get("keep_lo", 0), case.get("keep_hi", 0), size=B)).astype(np.int64))
    return n, ctx, used, keep, start, pre


def _batch(case, seed):
    n, ctx, used, keep, start, pre = _sizes(case)
    r = np.random.default_rng([int(seed), 7])
    ends = np.append(start[1:], case["batch"]) if len(start) else [case["batch"]]
    order = np.concatenate([a + r.permutation(e - a) for a, e in zip(start if len(start) else [0], ends)])
    n, ctx, used, keep = n[order], ctx[order], used[order], keep[order]
    qsl = np.zeros(case["batch"] + 1, dtype=np.int32)
    qsl[1:] = np.cumsum(n)
    return n, ctx, used, keep, start, pre, qsl, r


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
    n, ctx, used, keep, start, pre, qsl, r = _batch(case, seed)
    B, bs, hkv, dim = case["batch"], case["block"], case["hkv"], case["dim"]
    S = ctx + used
    nblk = -(-S // bs)
    # a group's sequences begin with the blocks of its prefix
    head = np.zeros(B, dtype=np.int64)
    if len(start):
        head = np.repeat(pre // bs, np.diff(np.append(start, B)))
    blocks = int((nblk - head).sum() + (pre // bs).sum())
    perm = r.permutation(blocks).astype(np.int32)
    tables = np.zeros((B, int(nblk.max())), dtype=np.int32)
    at = 0
    for g in range(len(start)):
        p = int(pre[g]) // bs
        tables[start[g]: (start[g + 1] if g + 1 < len(start) else B), :p] = perm[at: at + p]
        at += p
    for b in range(B):
        own_blocks = int(nblk[b] - head[b])
        tables[b, head[b]: nblk[b]] = perm[at: at + own_blocks]
        at += own_blocks
    g = _gen(seed, 0)
    st = dict(case=case, qsl=_to(qsl), seq_lens=_to(S), tables=_to(tables), T=int(qsl[-1]), max_n=int(n.max()),
              max_s=int(S.max()), blocks=blocks, n=used, S=S, starts=qsl[:-1].astype(np.int64))
    cells = blocks * hkv * bs * dim
    if case.get("in8"):
        # blocks and heads of different magnitude
        e = torch.randint(-7, -4, (blocks, hkv, 2), generator=g, device=DEV)
        st.update(k_pool=_codes(cells, g), v_pool=_codes(cells, g), scales=((e + 127).to(torch.int32) << 23).view(torch.float32))
    else:
        st.update(k_pool=_randn_bf16((cells,), g), v_pool=_randn_bf16((cells,), g))
    if case["kind"] == "evict":
        # weights as they add up: many small ones, equal ones among them, few large
        w = torch.empty((blocks, hkv, bs), device=DEV).exponential_(generator=g)
        st.update(weights=torch.round(w * w * 256.0) / 256.0, weights_out=torch.zeros((blocks, hkv, bs), device=DEV),
                  keep=_to(keep), first=_to(np.full(B, case["first"])), new_lens=torch.zeros(B, dtype=torch.int32, device=DEV))
        return st
    st.update(q=_randn_bf16((st["T"], case["hq"], dim), g))
    if case["kind"] == "weights":
        st.update(weights_in=torch.empty((blocks, hkv, bs), device=DEV).exponential_(generator=g) if case["add"] else None,
                  weights_out=torch.zeros((blocks, hkv, bs), device=DEV), lse=_plain_attend(st, values=False)[1],
                  accepted=_to(used - 1) if case["accepted"] else None)
        return st
    st.update(out=torch.empty_like(st["q"]))
    st["lse"] = torch.empty((st["T"], case["hq"]), device=DEV) if case["lse"] else None
    if case["kind"] == "shared":
        st.update(group_start=_to(np.append(start, B)), prefix=_to(pre))
    return st


# ------------------------------------------------------------------------------------- plain forms


def _swap23(s):
    return (s & ~12) | ((s >> 2 & 1) << 3) | ((s >> 3 & 1) << 2)


def _rows_of_blocks(st, name, dtype):
    """K or V of every block as [blocks, slots, hkv, dim]."""
    case = st["case"]
    hkv, D, bs = case["hkv"], case["dim"], case["block"]
    x = st[name].to(dtype)
    if case.get("in8"):
        u = bs // 16
        if name == "k_pool":
            x = x.view(-1, hkv, u, D // 16, 16, 16).permute(0, 2, 4, 1, 3, 5)
        else:
            x = x.view(-1, hkv, u, D // 64, 32, 2, 2, 2, 4).permute(0, 2, 7, 5, 8, 1, 3, 6, 4)
        x = x.reshape(-1, bs, hkv, D)
        return x * st["scales"].to(dtype)[:, None, :, 0 if name == "k_pool" else 1, None]
    if name == "k_pool":
        return x.view(-1, hkv, D // 8, bs, 8).permute(0, 3, 1, 2, 4).reshape(-1, bs, hkv, D)
    return x.view(-1, hkv, D, bs)[..., _swap23(torch.arange(bs, device=DEV))].permute(0, 3, 1, 2)


def _parts(st, rows):
    """Runs of sequences, and of their query tokens, whose padded scores fit: (sequences, first token, tokens, keys)."""
    case = st["case"]
    b, B = 0, case["batch"]
    while b < B:
        e = b + 1
        while e < B and (e + 1 - b) * rows[b: e + 1].max() * st["S"][b: e + 1].max() * case["hq"] <= _CHUNK:
            e += 1
        n, keys = int(rows[b:e].max()), int(st["S"][b:e].max())
        step = n if e - b > 1 else max(1, _CHUNK // (keys * case["hq"]))
        for j in range(0, n, step):
            yield b, e, j, min(step, n - j), keys
        b = e


def _part_scores(st, k, b, e, j, n, keys):
    """Scores [sequences, hkv, tokens * group, keys] of the part, -inf where a token does not see a key; the q rows
    [sequences, tokens]; whether the token exists."""
    case = st["case"]
    hkv, G, D, bs = case["hkv"], case["hq"] // case["hkv"], case["dim"], case["block"]
    S, most = _to(st["S"][b:e], torch.int64), _to(st["n"][b:e], torch.int64)
    tok = j + torch.arange(n, device=DEV)
    row = (_to(st["starts"][b:e], torch.int64)[:, None] + tok).clamp(max=st["T"] - 1)
    q = st["q"].float()[row].view(e - b, n, hkv, G, D).permute(0, 2, 1, 3, 4).reshape(e - b, hkv, n * G, D)
    k = k[st["tables"][b:e, : -(-keys // bs)].long()].flatten(1, 2)[:, :keys]
    x = torch.matmul(q.contiguous(), k.permute(0, 2, 3, 1).contiguous()) * D ** -0.5
    last = (S - most)[:, None] + tok
    seen = torch.arange(keys, device=DEV) <= last.repeat_interleave(G, dim=1)[:, None, :, None]
    return torch.where(seen, x, -math.inf), row, tok < most[:, None]


def _plain_attend(st, values=True):
    """Outputs and the logarithms of the sums of exponentials of every query token's row, in 32 bits."""
    case = st["case"]
    hkv, hq, D, bs = case["hkv"], case["hq"], case["dim"], case["block"]
    k = _rows_of_blocks(st, "k_pool", torch.float32)
    v = _rows_of_blocks(st, "v_pool", torch.float32) if values else None
    out = torch.zeros((st["T"], hq, D), device=DEV) if values else None
    lse = torch.zeros((st["T"], hq), device=DEV)
    for b, e, j, n, keys in _parts(st, st["n"]):
        x, row, real = _part_scores(st, k, b, e, j, n, keys)
        m = x.amax(dim=-1, keepdim=True)
        p = torch.exp(x - m)
        del x
        total = p.sum(dim=-1, keepdim=True)
        by_token = lambda y: y.view(e - b, hkv, n, hq // hkv, -1).permute(0, 2, 1, 3, 4).reshape(e - b, n, hq, -1)  # noqa: E731
        lse[row[real]] = by_token(m + torch.log(total))[real][..., 0]
        if values:
            w = v[st["tables"][b:e, : -(-keys // bs)].long()].flatten(1, 2)[:, :keys]
            w = torch.where((torch.arange(keys, device=DEV) < _to(st["S"][b:e])[:, None])[..., None, None], w, 0.0)
            o = torch.matmul(p, w.permute(0, 2, 1, 3).contiguous()) / total
            out[row[real]] = by_token(o)[real]
    return out, lse


def _plain_weights(st):
    case = st["case"]
    hkv, G, bs = case["hkv"], case["hq"] // case["hkv"], case["block"]
    k = _rows_of_blocks(st, "k_pool", torch.float32)
    out = st["weights_out"].zero_()
    for b, e, j, n, keys in _parts(st, st["n"]):
        x, row, real = _part_scores(st, k, b, e, j, n, keys)
        lse = st["lse"][row].view(e - b, n, hkv, G).permute(0, 2, 1, 3).reshape(e - b, hkv, n * G, 1)
        p = torch.where(real.repeat_interleave(G, dim=1)[:, None, :, None], torch.exp(x - lse), 0.0)
        key = torch.arange(keys, device=DEV)
        seq = torch.arange(e - b, device=DEV)[:, None].expand(-1, keys)
        mine = key < _to(st["S"][b:e])[:, None]                       # [sequences, keys]
        blk = st["tables"][b:e].long()[seq, key // bs][mine]
        slot = (key % bs).expand(e - b, -1)[mine]
        out[blk, :, slot] += p.sum(dim=2).permute(0, 2, 1)[mine]
        if case["add"] and j == 0:
            old = key < _to(st["S"][b:e] - st["n"][b:e])[:, None]
            out[blk, :, slot] += torch.where(old[mine][:, None], st["weights_in"][blk, :, slot], 0.0)
    return out


def _ranks(w):
    """Whole numbers in the order of w, equal values by the lowest index first."""
    bits = (w + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return (bits << 32) - torch.arange(w.shape[-1], device=w.device)


def _plain_evict(st):
    """Sequences of all lengths together: the places that they keep, then one gather and one scatter a pool."""
    case = st["case"]
    B, hkv, D, bs, keys = case["batch"], case["hkv"], case["dim"], case["block"], st["max_s"]
    S = st["seq_lens"].long()[:, None]
    m = torch.minimum(st["keep"].long()[:, None], S)
    f = torch.minimum(st["first"].long()[:, None], m)
    l = torch.minimum(torch.full_like(m, case["last"]), m - f)
    key = torch.arange(keys, device=DEV)[None, :]
    blk = st["tables"].long()[:, (key[0] // bs)]                             # [B, keys]
    w = st["weights"][blk, :, key % bs].permute(0, 2, 1)                     # [B, hkv, keys]
    always = (key < f) | ((key >= S - l) & (key < S))
    rank = torch.where((always | (key >= S))[:, None, :], torch.iinfo(torch.int64).min, _ranks(w))
    place = torch.argsort(torch.argsort(rank, dim=-1, descending=True), dim=-1)
    kept = always[:, None, :] | ((place < (m - f - l)[:, None, :]) & (key < S)[:, None, :])
    b, h, src = torch.nonzero(kept, as_tuple=True)
    dst = (torch.cumsum(kept, dim=-1) - 1)[b, h, src]
    for name, shape in (("k_pool", (-1, hkv, D // 8, bs, 8)), ("v_pool", (-1, hkv, D, bs))):
        pool = st[name].view(shape)
        if name == "k_pool":
            rows = pool[blk[b, src], h, :, src % bs]
            pool[blk[b, dst], h, :, dst % bs] = rows
        else:
            rows = pool[blk[b, src], h, :, _swap23(src % bs)]
            pool[blk[b, dst], h, :, _swap23(dst % bs)] = rows
    st["weights_out"][blk[b, dst], h, dst % bs] = st["weights"][blk[b, src], h, src % bs]
    st["new_lens"].copy_(m[:, 0])
    return st["k_pool"], st["v_pool"], st["weights_out"], st["new_lens"]


# ------------------------------------------------------------------------------------- the library's calls


def _space(st, size):
    """A workspace, as a program keeps one beside its buffers."""
    if "space" not in st:
        st["space"] = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
    return st["space"]


def _own(st):
    from paper_2609_34370_amd import spexis as sx
    case = st["case"]
    kind, B, hkv, D, bs = case["kind"], case["batch"], case["hkv"], case["dim"], case["block"]
    if kind == "evict":
        space = _space(st, sx.spexis_evict_kv_workspace_size(B, hkv, st["max_s"]))
        sx.spexis_evict_kv(st["k_pool"], st["v_pool"], st["weights"], st["blocks"], hkv, bs, D, st["seq_lens"], st["tables"],
                           st["max_s"], st["keep"], case["last"], st["weights_out"], st["new_lens"], space,
                           first_keys=st["first"])
        return st["k_pool"], st["v_pool"], st["weights_out"], st["new_lens"]
    where = (st["blocks"], hkv, bs, D, st["qsl"], st["seq_lens"], st["tables"], st["T"], st["max_n"], st["max_s"])
    if kind == "weights":
        sx.spexis_attention_weights(st["k_pool"], *where, st["q"], case["hq"], D ** -0.5, st["lse"], st["weights_out"],
                                    weights_in=st["weights_in"], accepted_len=st["accepted"])
        return st["weights_out"]
    pools = (st["k_pool"], st["v_pool"], st["scales"]) if case["in8"] else (st["k_pool"], st["v_pool"])
    rows = (st["q"], case["hq"], D ** -0.5, st["out"])
    if kind == "prompt":
        space = _space(st, sx.spexis_prompt_attention_workspace_size(B, case["hq"], hkv, D, st["T"], st["max_n"], st["max_s"]))
        f = sx.spexis_prompt_attention_kv8 if case["in8"] else sx.spexis_prompt_attention
        f(*pools, *where, *rows, space, lse=st["lse"])
    else:
        space = _space(st, sx.spexis_shared_attention_workspace_size(B, case["groups"], case["hq"], hkv, D, st["T"], st["max_n"],
                                                                     st["max_s"]))
        f = sx.spexis_shared_attention_kv8 if case["in8"] else sx.spexis_shared_attention
        f(*pools, *where, st["group_start"], st["prefix"], *rows, space, lse=st["lse"])
    return st["out"] if st["lse"] is None else (st["out"], st["lse"])


def run(st):
    if own:
        return _own(st)
    kind = st["case"]["kind"]
    if kind == "evict":
        return _plain_evict(st)
    if kind == "weights":
        return _plain_weights(st)
    out, lse = _plain_attend(st)
    return (out.to(torch.bfloat16), lse) if st["case"]["lse"] else out.to(torch.bfloat16)


def work(case):
    n, ctx, used, keep, start, pre = _sizes(case)
    hkv, dim, B = case["hkv"], case["dim"], case["batch"]
    S = ctx + used
    blocks = int((-(-S // case["block"])).sum())
    meta = 8 * B + 4 + 4 * blocks
    if case["kind"] == "evict":
        moved = float((keep - np.minimum(case["first"], keep)).sum())     # in front of these rows none leaves
        return {"bytes": moved * hkv * dim * 8 + (float(S.sum()) + float(keep.sum())) * hkv * 4 + 12 * B + meta, "flops": 0}
    hq = case["hq"]
    pairs = float((used * (S - used) + used * (used + 1) // 2).sum())     # (query token, key it sees)
    T = float(used.sum())
    if case["kind"] == "weights":
        return {"bytes": float(S.sum()) * hkv * (dim * 2 + 4) + (float(ctx.sum()) * hkv * 4 if case["add"] else 0) +
                T * hq * (dim * 2 + 4) + meta, "flops": 2 * pairs * hq * dim}
    cached = S.sum()
    if len(start):
        cached = cached - (np.repeat(pre, np.diff(np.append(start, B)))).sum() + pre.sum()
    size = 2 if case["in8"] else 4
    return {"bytes": float(cached) * hkv * (dim * size + (8 / case["block"] if case["in8"] else 0)) +
            T * hq * (dim * 4 + (4 if case["lse"] else 0)) + meta, "flops": 4 * pairs * hq * dim}


# ------------------------------------------------------------------------------------- 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    return {"evict": _exact_evict, "weights": _exact_weights}.get(case["kind"], _exact_attend)(case, st)


def _exact_rows(case, st, b):
    """Of sequence b: its blocks' keys and values [hkv, keys, dim]."""
    hkv, D, bs, S = case["hkv"], case["dim"], case["block"], int(st["S"][b])
    ids = st["tables"][b, : -(-S // bs)].long()
    if case.get("in8"):
        k = st["k_pool"].view(torch.uint8).view(-1, hkv, bs // 16, D // 16, 16, 16)[ids].view(torch.float8_e4m3fn).double()
        v = st["v_pool"].view(torch.uint8).view(-1, hkv, bs // 16, D // 64, 32, 2, 2, 2, 4)[ids].view(torch.float8_e4m3fn).double()
        k = k.permute(1, 0, 2, 4, 3, 5).reshape(hkv, len(ids), bs, D) * st["scales"][ids].double()[:, :, 0].t()[:, :, None, None]
        v = v.permute(1, 0, 2, 7, 5, 8, 3, 6, 4).reshape(hkv, len(ids), bs, D) * st["scales"][ids].double()[:, :, 1].t()[:, :, None, None]
    else:
        k = st["k_pool"].view(-1, hkv, D // 8, bs, 8)[ids].double().permute(1, 0, 3, 2, 4)
        # slots in four parts, of which the two middle ones are stored in the other order
        v = st["v_pool"].view(-1, hkv, D, bs // 16, 2, 2, 4)[ids].double().permute(1, 0, 3, 5, 4, 6, 2)
    return k.reshape(hkv, -1, D)[:, :S], v.reshape(hkv, -1, D)[:, :S]


def _exact_scores(case, st, b, k, j, n):
    """Scores of the query tokens j .. j + n of sequence b, as [hkv, n * group, keys up to the last that they see]."""
    hkv, G, D = case["hkv"], case["hq"] // case["hkv"], case["dim"]
    first = int(st["S"][b]) - int(st["n"][b])
    at = int(st["starts"][b]) + j
    q = st["q"][at: at + n].double().view(n, hkv, G, D).permute(1, 0, 2, 3).reshape(hkv, n * G, D)
    k = k[:, : first + j + n]
    x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
    limit = (first + j + torch.arange(n, device=DEV)).repeat_interleave(G)
    return x.masked_fill_(torch.arange(k.shape[1], device=DEV)[None, None, :] > limit[None, :, None], -math.inf), at


def _exact_attend(case, st):
    hkv, hq, D = case["hkv"], case["hq"], case["dim"]
    out = torch.zeros((st["T"], hq, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((st["T"], hq), dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        k, v = _exact_rows(case, st, b)
        step = max(1, (_CHUNK // 2) // (hq * int(st["S"][b])))
        for j in range(0, int(st["n"][b]), step):
            n = min(step, int(st["n"][b]) - j)
            x, at = _exact_scores(case, st, b, k, j, n)
            o = torch.matmul(torch.softmax(x, dim=-1), v[:, : x.shape[-1]])
            out[at: at + n] = o.view(hkv, n, hq // hkv, D).permute(1, 0, 2, 3).reshape(n, hq, D)
            lse[at: at + n] = torch.logsumexp(x, dim=-1).view(hkv, n, hq // hkv).permute(1, 0, 2).reshape(n, hq)
    return (out, lse) if case["lse"] else out


def _exact_weights(case, st):
    hkv, G, bs = case["hkv"], case["hq"] // case["hkv"], case["block"]
    out = torch.zeros(st["weights_out"].shape, dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        S, n = int(st["S"][b]), int(st["n"][b])
        total = torch.zeros((hkv, S), dtype=torch.float64, device=DEV)
        k, _ = _exact_rows(case, st, b)
        step = max(1, (_CHUNK // 2) // (case["hq"] * S))
        for j in range(0, n, step):
            rows = min(step, n - j)
            x, at = _exact_scores(case, st, b, k, j, rows)
            lse = st["lse"][at: at + rows].double().view(rows, hkv, G).permute(1, 0, 2).reshape(hkv, rows * G, 1)
            total[:, : x.shape[-1]] += torch.exp(x - lse).sum(dim=1)
        for i in range(0, S, bs):
            blk, e = int(st["tables"][b, i // bs]), min(S, i + bs)
            out[blk, :, : e - i] = total[:, i:e]
            old = min(e, S - n) - i
            if case["add"] and old > 0:
                out[blk, :, :old] += st["weights_in"][blk, :, :old].double()
    return out


def _exact_evict(case, st):
    """Sequence by sequence and head by head on the host's copy of the weights; rows move as whole numbers."""
    hkv, D, bs = case["hkv"], case["dim"], case["block"]
    k = st["k_pool"].view(-1, hkv, D // 8, bs, 8).permute(0, 3, 1, 2, 4).reshape(-1, hkv, D).clone()     # [places, hkv, dim]
    v = st["v_pool"].view(-1, hkv, D, bs // 16, 2, 2, 4).permute(0, 3, 5, 4, 6, 1, 2).reshape(-1, hkv, D).clone()
    w = st["weights"].permute(0, 2, 1).reshape(-1, hkv).double().cpu().numpy()
    w_out = np.zeros_like(w)
    tables, lens = st["tables"].cpu().numpy().astype(np.int64), []
    keeps = st["keep"].cpu().numpy()
    for b in range(case["batch"]):
        S = int(st["S"][b])
        m = min(int(keeps[b]), S)
        f = min(case["first"], m)
        last = min(case["last"], m - f)
        t = np.arange(S)
        place = tables[b, t // bs] * bs + t % bs
        lens.append(m)
        for h in range(hkv):
            middle = np.arange(f, S - last)
            best = middle[np.argsort(-w[place[middle], h], kind="stable")[: m - f - last]]
            src = place[np.sort(np.concatenate([np.arange(f), best, np.arange(S - last, S)]))]
            w_out[place[:m], h] = w[src, h]
            to, src = _to(place[:m], torch.int64), _to(src, torch.int64)
            k[to, h] = k[src, h]
            v[to, h] = v[src, h]
    k = k.view(-1, bs, hkv, D // 8, 8).permute(0, 2, 3, 1, 4).reshape(-1).double()
    v = v.view(-1, bs // 16, 2, 2, 4, hkv, D).permute(0, 5, 6, 1, 3, 2, 4).reshape(-1).double()
    w_out = torch.as_tensor(w_out, device=DEV).view(-1, bs, hkv).permute(0, 2, 1).contiguous()
    return k, v, w_out, torch.as_tensor(lens, dtype=torch.int32, device=DEV)
