"""Attention weights of a call without query tokens, on the host: sums of another array have to come over, so its pointers are
checked; nothing is done where there is nothing to write (no GPU needed)."""
import ctypes

from tests.test_abi_serving import FAKE, INVALID, ODD
from tests.test_abi_serving_edges import marked
from tests.test_abi_tiles import weigh

OTHER = ctypes.c_void_p(1024)


@marked
def test_no_query_tokens():
    assert weigh(T=0, q=None, lse=None, win=FAKE) == 0 and weigh(T=0, B=0, win=OTHER) == 0
    for kw in (dict(k=None), dict(qsl=None), dict(sl=None), dict(bt=None), dict(w=None), dict(win=ODD)):
        assert weigh(**{**dict(T=0, q=None, lse=None, win=OTHER), **kw}) == INVALID, kw
