"""Attention weights of a call without query tokens: sums go into another array as they are."""
import numpy as np
import pytest
import torch

from paper_2609_34370_amd import spexis as sx
from tests.test_gpu_evict import used_places
from tests.test_gpu_rotate import batch, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bs", [16, 32])
@pytest.mark.parametrize("first", [None, [3, 40, 0]])
def test_no_query_tokens(bs, first):
    qsl, S, tables, blocks = batch([0, 0, 0], [100, 33, 0], bs, 1)
    hkv, D = 2, 64
    k = torch.zeros(blocks * hkv * bs * D, dtype=torch.bfloat16, device="cuda")
    q, lse = torch.zeros((0, 8, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((0, 8), device="cuda")
    before = torch.rand((blocks, hkv, bs), device="cuda")
    out = torch.full_like(before, 777.0)

    def call(w, w_in):
        sx.spexis_attention_weights(k, blocks, hkv, bs, D, dev(qsl), dev(S), dev(tables), 0, 1, 100, q, 8, 0.125, lse, w, weights_in=w_in,
                                    first_keys=None if first is None else dev(np.asarray(first, np.int32)))
        torch.cuda.synchronize()
    call(out, before)
    lo = np.zeros(3, np.int32) if first is None else np.minimum(first, S)
    mask = used_places(S, tables, blocks, bs) & ~used_places(lo, tables, blocks, bs)
    mask = torch.as_tensor(np.broadcast_to(mask[:, None, :], tuple(out.shape)).copy(), device="cuda")
    assert torch.equal(out[mask], before[mask]) and (out[~mask] == 777.0).all()
    own = before.clone()
    call(own, own)
    assert torch.equal(own, before)
