"""Refusals of the rotating appends, the attention over the 8-bit cache and the log probabilities: scalar arguments
are checked on the host before any device call (no GPU needed)."""
import ctypes
import os

import pytest
import torch

from paper_2609_34370_amd import spexis as sx

pytestmark = [pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built"),
              pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation runs only without a GPU")]

FAKE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)
INVALID, UNSUPPORTED, SMALL = sx.SPEXIS_ERR_INVALID_ARGUMENT, sx.SPEXIS_ERR_UNSUPPORTED, sx.SPEXIS_ERR_WORKSPACE_TOO_SMALL


def rotate(in8, **kw):
    a = dict(k=FAKE, v=FAKE, sc=FAKE, nb=10, hkv=2, bs=16, d=64, B=2, qsl=FAKE, sl=FAKE, bt=FAKE, mb=4, T=4, mq=2,
             nk=FAKE, nv=FAKE, cs=FAKE, mp=100, rot=64, style=0, pos=None, q=FAKE, hq=8, qo=FAKE)
    a.update(kw)
    f = sx.lib().spexis_rotate_append_kv8 if in8 else sx.lib().spexis_rotate_append_kv
    return f(a["k"], a["v"], *([a["sc"]] if in8 else []), a["nb"], a["hkv"], a["bs"], a["d"], a["B"], a["qsl"], a["sl"],
             a["bt"], a["mb"], a["T"], a["mq"], a["nk"], a["nv"], a["cs"], a["mp"], a["rot"], a["style"], a["pos"], a["q"],
             a["hq"], a["qo"], None)


@pytest.mark.parametrize("in8", [False, True])
def test_rotating_appends(in8):
    for kw in (dict(nb=0), dict(hkv=0), dict(B=-1), dict(mb=0), dict(T=-1), dict(mq=0), dict(mp=0), dict(mp=-1), dict(style=2),
               dict(hq=0), dict(k=None), dict(v=None), dict(qsl=None), dict(sl=None), dict(bt=None), dict(nk=None),
               dict(nv=None), dict(cs=None), dict(q=None), dict(qo=None), dict(k=ODD), dict(nv=ODD), dict(cs=ODD),
               dict(q=ODD), dict(qo=ODD)):
        assert rotate(in8, **kw) == INVALID, kw
        assert (b"kv8" in sx.lib().spexis_last_error()) == in8
    for kw in (dict(bs=8), dict(bs=64), dict(d=96), dict(rot=8), dict(rot=24), dict(rot=80), dict(rot=0),
               dict(T=2**30, hkv=64, mq=2**29), dict(mb=2**28)):
        assert rotate(in8, **kw) == UNSUPPORTED, kw
    assert rotate(in8, B=0, k=None, nk=None, q=None, qo=None, qsl=None) == 0
    assert rotate(in8, T=0, k=None, nk=None, q=None, qo=None, sl=None, sc=None) == 0


def test_8_bit_append_without_rotation():
    assert rotate(True, sc=None) == INVALID
    none = dict(cs=None, mp=0, rot=0, style=9, q=None, qo=None, hq=0)
    assert rotate(True, T=0, **none) == 0
    for kw in (dict(q=FAKE, qo=FAKE, hq=8), dict(pos=FAKE), dict(cs=FAKE)):
        assert rotate(True, **dict(none, **kw)) == INVALID, kw


def attend(**kw):
    a = dict(k=FAKE, v=FAKE, sc=FAKE, nb=10, hkv=2, bs=16, d=64, B=2, qsl=FAKE, sl=FAKE, bt=FAKE, mb=4, T=4, mq=2, ms=40,
             q=FAKE, hq=8, scale=0.125, out=ctypes.c_void_p(512), chunk=0, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return sx.lib().spexis_verify_attention_kv8(a["k"], a["v"], a["sc"], a["nb"], a["hkv"], a["bs"], a["d"], a["B"],
                                                a["qsl"], a["sl"], a["bt"], a["mb"], a["T"], a["mq"], a["ms"], a["q"], a["hq"],
                                                a["scale"], a["out"], a["chunk"], a["ws"], a["wsb"], None)


def test_attention_over_the_8_bit_cache():
    for kw in (dict(nb=0), dict(hkv=0), dict(hq=0), dict(hq=7), dict(B=-1), dict(mb=0), dict(T=-1), dict(mq=0), dict(ms=0),
               dict(chunk=-1), dict(scale=float("nan")), dict(mb=1, mq=17, hq=2), dict(k=None), dict(v=None), dict(sc=None),
               dict(qsl=None), dict(sl=None), dict(bt=None), dict(q=None), dict(out=None), dict(out=FAKE), dict(k=ODD),
               dict(sc=ODD), dict(ws=ODD)):
        assert attend(**kw) == INVALID, kw
        assert b"spexis_verify_attention_kv8" in sx.lib().spexis_last_error()
    for kw in (dict(bs=8), dict(d=96), dict(hq=66, mq=2), dict(mb=2**27, B=2**11), dict(chunk=32, B=2**20, mb=2**6, ms=2**16)):
        assert attend(**kw) == UNSUPPORTED, kw
    need = sx.spexis_verify_attention_kv8_workspace_size(2, 8, 2, 64, 2, 40)
    assert need > 0 and attend(wsb=need - 1) == SMALL and attend(ws=None) == SMALL
    assert attend(B=0, k=None, ws=None) == 0 and attend(T=0, q=None, ws=None) == 0
    assert sx.spexis_verify_attention_kv8_workspace_size(0, 8, 2, 64, 2, 40) == 0


def logprobs(**kw):
    a = dict(type=0, x=FAKE, stride=1000, rows=8, V=1000, t=1.0, items=8, ids=None, tok=FAKE, top=5, lp=FAKE, h=None,
             ti=FAKE, tl=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return sx.lib().spexis_token_logprobs(a["type"], a["x"], a["stride"], a["rows"], a["V"], a["t"], a["items"], a["ids"],
                                          a["tok"], a["top"], a["lp"], a["h"], a["ti"], a["tl"], a["ws"], a["wsb"], None)


def test_token_logprobs():
    for kw in (dict(type=2), dict(type=-1), dict(rows=-1), dict(V=0), dict(items=-1), dict(top=-1), dict(stride=999),
               dict(t=0.0), dict(t=-1.0), dict(t=float("inf")), dict(t=float("nan")), dict(items=9), dict(x=None),
               dict(tok=None), dict(lp=None), dict(ti=None), dict(tl=None), dict(x=ctypes.c_void_p(258)),
               dict(x=ctypes.c_void_p(257), type=1), dict(ws=ODD, ids=FAKE, V=200000, stride=200000)):
        assert logprobs(**kw) == INVALID, kw
    for kw in (dict(top=33), dict(V=(1 << 22) + 1, stride=1 << 23)):
        assert logprobs(**kw) == UNSUPPORTED, kw
    need = sx.spexis_token_logprobs_workspace_size(8, 200000, 5)
    assert need > 0 and sx.spexis_token_logprobs_workspace_size(8, 200000, 33) == 0
    big = dict(V=200000, stride=200000)
    assert logprobs(wsb=need - 1, **big) == SMALL and logprobs(ws=None, **big) == SMALL
    assert logprobs(items=0, x=None, tok=None, lp=None) == 0


def test_a_temperature_whose_reciprocal_overflows():
    assert logprobs(t=1e-39) == INVALID
