"""Refusals of the attention of prompts and behind shared prefixes, of the attention weights and of evictions, and their
workspaces: scalar arguments are checked on the host before any device call (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest
import torch

from paper_2609_34370_amd import spexis as sx
from tests.test_abi_serving import FAKE, INVALID, ODD, SMALL, UNSUPPORTED
from tests.test_abi_serving_edges import B, BF, BS, D, F32, HKV, HQ, I32, LIKE, MB, NB, POOLS, POOLS8, T, WHERE, marked, placed, recorded  # noqa: F401

OUT = ctypes.c_void_p(512)
ATTENTIONS = ["spexis_prompt_attention", "spexis_prompt_attention_kv8", "spexis_shared_attention", "spexis_shared_attention_kv8"]


def attend(name, **kw):
    a = dict(k=FAKE, v=FAKE, sc=FAKE, nb=10, hkv=2, bs=16, d=64, B=2, qsl=FAKE, sl=FAKE, bt=FAKE, mb=40, T=4, mq=2, ms=640, ng=1,
             gs=FAKE, pl=FAKE, q=FAKE, hq=8, scale=0.125, out=OUT, lse=None, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    scales = [a["sc"]] if name.endswith("kv8") else []
    groups = [a["ng"], a["gs"], a["pl"]] if "shared" in name else []
    return getattr(sx.lib(), name)(a["k"], a["v"], *scales, a["nb"], a["hkv"], a["bs"], a["d"], a["B"], a["qsl"], a["sl"],
                                   a["bt"], a["mb"], a["T"], a["mq"], a["ms"], *groups, a["q"], a["hq"], a["scale"], a["out"],
                                   a["lse"], a["ws"], a["wsb"], None)


@marked
@pytest.mark.parametrize("name", ATTENTIONS)
def test_attention(name):
    bad = [dict(nb=0), dict(hkv=0), dict(hq=0), dict(hq=7), dict(B=-1), dict(mb=0), dict(T=-1), dict(mq=0), dict(ms=0),
           dict(scale=float("nan")), dict(scale=float("inf")), dict(mb=1, mq=17), dict(k=None), dict(v=None), dict(qsl=None),
           dict(sl=None), dict(bt=None), dict(q=None), dict(out=None), dict(out=FAKE), dict(k=ODD), dict(v=ODD), dict(q=ODD),
           dict(out=ODD), dict(ws=ODD)]
    if name.endswith("kv8"):
        bad += [dict(sc=None), dict(sc=ODD)]
    if "shared" in name:
        bad += [dict(ng=-1), dict(gs=None), dict(pl=None)]
    for kw in bad:
        assert attend(name, **kw) == INVALID, kw
        assert sx.lib().spexis_last_error().startswith(name.encode() + b":")
    for kw in (dict(bs=8), dict(bs=64), dict(d=96), dict(d=256), dict(T=2**28), dict(mb=2**26), dict(B=2**30),
               dict(hkv=2**14, hq=2**14, T=2**15, B=2**15, mq=1)):
        assert attend(name, **kw) == UNSUPPORTED, kw
    if "shared" in name:
        need = sx.spexis_shared_attention_workspace_size(2, 1, 8, 2, 64, 4, 2, 640)
    else:
        need = sx.spexis_prompt_attention_workspace_size(2, 8, 2, 64, 4, 2, 640)
    assert need > 0 and attend(name, wsb=need - 1) == SMALL and attend(name, ws=None) == SMALL
    assert attend(name, B=0, k=None, ws=None, gs=None) == 0 and attend(name, T=0, q=None, out=None, ws=None, wsb=0) == 0


def weigh(**kw):
    a = dict(k=FAKE, nb=10, hkv=2, bs=16, d=64, B=2, qsl=FAKE, sl=FAKE, bt=FAKE, mb=40, T=4, mq=2, ms=640, q=FAKE, hq=8, scale=0.125,
             lse=ctypes.c_void_p(260), acc=None, first=None, win=None, w=FAKE)
    a.update(kw)
    return sx.lib().spexis_attention_weights(a["k"], a["nb"], a["hkv"], a["bs"], a["d"], a["B"], a["qsl"], a["sl"], a["bt"], a["mb"],
                                             a["T"], a["mq"], a["ms"], a["q"], a["hq"], a["scale"], a["lse"], a["acc"], a["first"],
                                             a["win"], a["w"], None)


@marked
def test_weights():
    for kw in (dict(nb=0), dict(hkv=0), dict(hq=0), dict(hq=7), dict(B=-1), dict(mb=0), dict(T=-1), dict(mq=0), dict(ms=0),
               dict(scale=float("nan")), dict(mb=1, mq=17), dict(k=None), dict(qsl=None), dict(sl=None), dict(bt=None), dict(q=None),
               dict(lse=None), dict(w=None), dict(k=ODD), dict(q=ODD), dict(w=ODD), dict(win=ODD)):
        assert weigh(**kw) == INVALID, kw
        assert sx.lib().spexis_last_error().startswith(b"spexis_attention_weights:")
    for kw in (dict(bs=8), dict(d=96), dict(T=2**28), dict(mb=2**26), dict(B=2**12, ms=2**19)):
        assert weigh(**kw) == UNSUPPORTED, kw
    assert weigh(B=0, k=None, w=None) == 0 and weigh(T=0, q=None, lse=None) == 0


def evict(**kw):
    a = dict(k=FAKE, v=FAKE, w=FAKE, nb=10, hkv=2, bs=16, d=64, B=2, sl=FAKE, bt=FAKE, mb=40, ms=640, keep=FAKE, first=None, last=4,
             wo=FAKE, new=FAKE, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    return sx.lib().spexis_evict_kv(a["k"], a["v"], a["w"], a["nb"], a["hkv"], a["bs"], a["d"], a["B"], a["sl"], a["bt"], a["mb"],
                                    a["ms"], a["keep"], a["first"], a["last"], a["wo"], a["new"], a["ws"], a["wsb"], None)


@marked
def test_eviction():
    for kw in (dict(nb=0), dict(hkv=0), dict(B=-1), dict(mb=0), dict(ms=0), dict(last=-1), dict(k=None), dict(v=None), dict(w=None),
               dict(sl=None), dict(bt=None), dict(keep=None), dict(wo=None), dict(new=None), dict(k=ODD), dict(v=ODD), dict(w=ODD),
               dict(wo=ODD), dict(ws=ODD)):
        assert evict(**kw) == INVALID, kw
        assert sx.lib().spexis_last_error().startswith(b"spexis_evict_kv:")
    for kw in (dict(bs=8), dict(d=96), dict(mb=2**26), dict(B=2**17), dict(ms=2**30)):
        assert evict(**kw) == UNSUPPORTED, kw
    need = sx.spexis_evict_kv_workspace_size(2, 2, 640)
    assert need > 0 and evict(wsb=need - 1) == SMALL and evict(ws=None) == SMALL
    assert evict(B=0, k=None, w=None, ws=None, wsb=0) == 0


@marked
def test_workspaces():
    prompt, shared = sx.spexis_prompt_attention_workspace_size, sx.spexis_shared_attention_workspace_size
    for bad in ((0, 8, 2, 64, 4, 2, 640), (2, 7, 2, 64, 4, 2, 640), (2, 8, 0, 64, 4, 2, 640), (2, 8, 2, 0, 4, 2, 640),
                (2, 8, 2, 64, 0, 2, 640), (2, 8, 2, 64, 4, 0, 640), (2, 8, 2, 64, 4, 2, 0), (2, 8, 2, 64, 2**30, 2, 640)):
        assert prompt(*bad) == 0 and shared(bad[0], 1, *bad[1:]) == 0
    assert shared(2, -1, 8, 2, 64, 4, 2, 640) == 0 and sx.spexis_evict_kv_workspace_size(1, 0, 1) == 0
    # without groups, and for short sequences, a shared call is a prompt's
    r = np.random.default_rng(0)
    for _ in range(200):
        seqs, hkv, group, n = (int(x) for x in r.integers(1, [300, 17, 17, 3000]))
        a = (seqs, hkv * group, hkv, 128, seqs * n, n, n + int(r.integers(0, 5000)))
        assert shared(a[0], 0, *a[1:]) == prompt(*a)
        few = (*a[:-1], 512)
        assert shared(a[0], seqs, *few[1:]) == prompt(*few) == 16
        # Prompts: nothing where the chip is full, else at most a half of 768 row tiles (at least one a head) and 768 parts; with
        # a prefix of P and O own row tiles, P + O at most 1536 (at least two a head), P + 768 slots for the one and
        # P + O + 768 for all, or P + 768 alone.
        slot, tiles = 128 * 130 * 4, seqs * -(-group * n // 128) * hkv
        assert prompt(*a) == 16 if tiles > 384 else prompt(*a) < (tiles + 768 + 1) * slot * 1.01
        pre = min(tiles, -(-seqs * n * group // 128) * hkv + hkv)
        assert shared(a[0], 1, *a[1:]) < max(2 * pre + tiles + 2 * 768 if pre + tiles <= 1536 + hkv else 0, pre + 768) * slot * 1.01


# ---- the binding

WEIGHTS = ((NB, HKV, BS), F32)
ATTEND = dict(WHERE, q=((T, HQ, D), BF), out=((T, HQ, D), BF), lse=((T, HQ), F32), workspace=((1 << 20,), torch.uint8))
GROUPS = dict(group_start_loc=((2,), I32), prefix_lens=((1,), I32))
ROWS = dict(LIKE, max_seq_len=40, num_q_heads=HQ, scale=0.125)
CALLS = {
    "spexis_prompt_attention": (dict(POOLS, **ATTEND), ROWS),
    "spexis_prompt_attention_kv8": (dict(POOLS8, **ATTEND), ROWS),
    "spexis_shared_attention": (dict(POOLS, **ATTEND, **GROUPS), ROWS),
    "spexis_shared_attention_kv8": (dict(POOLS8, **ATTEND, **GROUPS), ROWS),
    "spexis_attention_weights": (dict(k_cache=POOLS["k_cache"], **WHERE, q=((T, HQ, D), BF), lse=((T, HQ), F32), weights=WEIGHTS,
                                      weights_in=WEIGHTS, accepted_len=((B,), I32), first_keys=((B,), I32)), ROWS),
    "spexis_evict_kv": (dict(POOLS, weights=WEIGHTS, seq_lens=WHERE["seq_lens"], block_tables=WHERE["block_tables"],
                             keep_lens=((B,), I32), weights_out=WEIGHTS, new_seq_lens=((B,), I32), first_keys=((B,), I32),
                             workspace=((1 << 16,), torch.uint8)),
                        dict(num_blocks=NB, num_kv_heads=HKV, block_size=BS, head_dim=D, max_seq_len=40, keep_last=2)),
}


@pytest.mark.parametrize("call", CALLS)
def test_every_tensor_is_checked(call, recorded):  # noqa: F811
    """Its device, its type, its size."""
    shapes, scalars = CALLS[call]
    f = getattr(sx, call)
    f(**{k: placed(*v) for k, v in shapes.items()}, **scalars)
    assert [name for name, _ in recorded.calls] == [call] and recorded.calls[0][1][-1] == 77
    for other, (shape, dtype) in shapes.items():
        with pytest.raises(ValueError, match="current device"):
            f(**{k: placed(*v, on=int(k == other)) for k, v in shapes.items()}, **scalars)
        if other != "workspace":
            tensors = {k: placed(*v) for k, v in shapes.items()}
            tensors[other] = placed(shape, torch.int64)
            with pytest.raises(ValueError):
                f(**tensors, **scalars)
        if other not in ("workspace", "query_start_loc", "prefix_lens"):   # (these say how many there are)
            if other == "seq_lens" and call == "spexis_evict_kv":
                continue
            tensors[other] = placed((shape[0] - 1, *shape[1:]), dtype)
            with pytest.raises(ValueError):
                f(**tensors, **scalars)
    assert len(recorded.calls) == 1


def test_what_may_be_left_out(recorded):  # noqa: F811
    for call, names in (("spexis_prompt_attention", ["lse"]), ("spexis_shared_attention_kv8", ["lse"]),
                        ("spexis_attention_weights", ["weights_in", "accepted_len", "first_keys"]), ("spexis_evict_kv", ["first_keys"])):
        shapes, scalars = CALLS[call]
        getattr(sx, call)(**{k: placed(*v) for k, v in shapes.items() if k not in names}, **scalars)
    assert len(recorded.calls) == 4


@pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built")
def test_a_step_chooses_its_attention():
    """Up to 64 query rows a KV head the verification's, beyond it and for shared prefixes or weights the tiles'."""
    from paper_2609_34370_amd import workloads as wl
    from paper_2609_34370_amd.step import VerifyStep
    spec = wl.spec_with(1, batch=2)
    for k, kw, tiles in (([4, 2], {}, False), ([300, 2], {}, True), ([4, 2], dict(shared=([0, 2], [16])), True),
                         ([4, 2], dict(weights=torch.zeros(1)), True)):
        batch = wl.make_batch(spec, ctx_lens=[40, 70], k=k)
        batch.block_tables[1, 0] = batch.block_tables[0, 0]
        s = VerifyStep(batch, wl.make_attention_inputs(spec, batch), None, device="cpu", **kw)
        assert s.tiles == tiles
    batch = wl.make_batch(spec, ctx_lens=[40, 70], k=[4, 2])
    batch.block_tables[1, :2] = batch.block_tables[0, :2]
    s = VerifyStep(batch, wl.make_attention_inputs(spec, batch), None, device="cpu", shared=([0, 2], [31]), weights=torch.zeros(1))
    assert s.first_keys.tolist() == [31 // spec.block_size * spec.block_size] * 2


@pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built")
def test_what_a_step_refuses():
    from paper_2609_34370_amd import workloads as wl
    from paper_2609_34370_amd.step import VerifyStep
    spec = wl.spec_with(1, batch=2)
    batch = wl.make_batch(spec, ctx_lens=[40, 70], k=[4, 2])
    batch.block_tables[1, :2] = batch.block_tables[0, :2]
    attn, bs = wl.make_attention_inputs(spec, batch), spec.block_size
    rotary = wl.make_rotary_inputs(80, spec.head_dim)
    VerifyStep(batch, attn, None, device="cpu", shared=([0, 2], [2 * bs]))
    for kw in (dict(shared=([0, 2], [3 * bs])), dict(shared=([0, 2], [41])), dict(positions=[1] * batch.T),
               dict(rotary=rotary, positions=[80] * batch.T), dict(rotary=rotary, positions=[-1] * batch.T)):
        with pytest.raises(ValueError):
            VerifyStep(batch, attn, None, device="cpu", **kw)
    VerifyStep(batch, attn, None, device="cpu", rotary=rotary, positions=[79] * batch.T)
    with pytest.raises(ValueError):
        VerifyStep(batch, wl.make_attention_inputs8(spec, batch), None, device="cpu", weights=torch.zeros(1))
