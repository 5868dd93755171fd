"""Prompts, steps behind a shared prefix, attention weights and evictions together, as a serving loop runs them, against the
64-bit forms on the GPU's own inputs of each stage; as a replayed graph and on another stream, bit for bit."""
import dataclasses
import sys

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import workloads as wl
from paper_2609_34370_amd.step import VerifyStep
from tests import layout_ref
from tests.test_gpu_evict import U, used_places
from tests.test_gpu_tile_attention import check

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


class View:
    """A step's cache in logical coordinates, as it is now."""

    def __init__(self, s):
        b, spec, a = s.batch, s.spec, s.attn
        self.blocks, self.bs, self.hkv, self.D, self.in8 = b.num_blocks, spec.block_size, spec.num_kv_heads, spec.head_dim, s.in8
        if s.in8:
            places = osv.places8(self.blocks, self.hkv, self.bs, self.D)
            scales = a.scales.double().cpu().numpy()
            self.k, self.v = (osv.E4M3[pool.view(torch.uint8).cpu().numpy()[p]] * scales[:, None, :, i, None]
                              for i, (pool, p) in enumerate(zip((a.k_pool, a.v_pool), places)))
        else:
            blk, slot, h, d = np.ogrid[:self.blocks, :self.bs, :self.hkv, :self.D]
            self.k, self.v = (pool.double().cpu().numpy().reshape(-1)[f(blk, h, slot, d, self.hkv, self.bs, self.D)]
                              for pool, f in ((a.k_pool, layout_ref.k_offsets), (a.v_pool, layout_ref.v_offsets)))


def check_attention(s):
    b = s.batch
    check(s.out, s.lse, View(s), b.qsl, b.seq_lens, b.block_tables, s.q, float(np.float32(s.scale)))


@pytest.mark.parametrize("in8", [False, True])
def test_prompts(in8):
    """More rows than the verification attention takes: append with rotation, then attention."""
    spec = wl.spec_with(4, batch=4, num_q_heads=16, num_kv_heads=4)
    batch = wl.make_batch(spec, ctx_lens=[0, 33, 0, 200], k=[300, 70, 0, 129])
    attn = (wl.make_attention_inputs8 if in8 else wl.make_attention_inputs)(spec, batch, device="cuda")
    rotary = wl.make_rotary_inputs(batch.max_seq_len, spec.head_dim, device="cuda")
    s = VerifyStep(batch, attn, None, rotary=rotary)
    s.run()
    torch.cuda.synchronize()
    check_attention(s)


def share(batch, bs, blocks):
    """The batch with every sequence's first `blocks` blocks those of the first one."""
    batch.block_tables[:, :blocks] = batch.block_tables[0, :blocks]
    return (np.array([0, batch.B], np.int32), np.array([blocks * bs], np.int32))


def life(in8=False, seed=None):
    """A step of six sequences behind 608 shared tokens, with acceptance."""
    spec = wl.spec_with(4, batch=6, num_q_heads=16, num_kv_heads=4, vocab=1003)
    batch = wl.make_batch(spec, ctx_lens=[700, 640, 608, 900, 615, 1000], k=[4, 8, 0, 3, 5, 8], seed=seed)
    shared = share(batch, spec.block_size, 608 // spec.block_size)
    attn = (wl.make_attention_inputs8 if in8 else wl.make_attention_inputs)(spec, batch, device="cuda", seed=seed)
    acc = wl.make_accept_inputs(spec, batch, device="cuda", seed=seed)
    weights = None if in8 else torch.rand((batch.num_blocks, spec.num_kv_heads, spec.block_size), device="cuda",
                                          generator=torch.Generator("cuda").manual_seed(5))
    rotary = wl.make_rotary_inputs(batch.max_seq_len, 64, device="cuda", style=1)
    return VerifyStep(batch, attn, acc, rotary=rotary, shared=shared, weights=weights)


def test_step_weights_and_eviction():
    s = life()
    b, spec = s.batch, s.spec
    before = s.weights.double().cpu().numpy()
    s.run()
    torch.cuda.synchronize()
    check_attention(s)
    c = View(s)
    accepted = s.accepted_len.cpu().numpy()
    lens = b.seq_lens - (np.diff(b.qsl) - 1 - accepted)
    assert np.array_equal(s.lens_after.cpu().numpy(), lens)
    # (those of shared blocks stay as they were)
    first = np.full(b.B, 608)
    want, size = osv.attention_weights(c.k, b.qsl, lens, b.block_tables, s.q.double().cpu().numpy(), float(np.float32(s.scale)),
                                       s.lse.double().cpu().numpy(), before, accepted, first)
    got = s.weights.double().cpu().numpy()
    own = used_places(lens, b.block_tables, b.num_blocks, spec.block_size)
    own[b.block_tables[0, : 608 // spec.block_size]] = False
    own = np.broadcast_to(own[:, None, :], got.shape)
    assert (np.abs(got - want) <= U * size + 1e-30)[own].all() and np.array_equal(got[~own], before[~own])
    # eviction to 640 keys, the shared ones and the last 8 among them
    w = s.weights.cpu().numpy().copy()
    keep = np.minimum(640, lens).astype(np.int32)
    new = s.evict(torch.as_tensor(keep).cuda(), 8)
    torch.cuda.synchronize()
    k, v, w2, m = osv.evict(c.k, c.v, w, lens, b.block_tables, keep, first, 8)
    assert np.array_equal(new.cpu().numpy(), m)
    kept = used_places(m, b.block_tables, b.num_blocks, spec.block_size)
    now = View(s)
    assert np.array_equal(now.k[kept], k[kept]) and np.array_equal(now.v[kept], v[kept])
    assert np.array_equal(s.weights.cpu().numpy().transpose(0, 2, 1)[kept], w2.transpose(0, 2, 1)[kept])
    # the next step's tokens follow behind what is left, at the positions that they have in the text
    n = np.array([3, 1, 5, 2, 2, 4], np.int32)   # (no further than the blocks that the sequences have)
    qsl = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    b2 = wl.Batch(spec, m, n - 1, qsl, (m + n).astype(np.int32), b.block_tables, b.num_blocks)
    attn = dataclasses.replace(wl.make_attention_inputs(spec, b2, device="cuda", seed=7), k_pool=s.attn.k_pool, v_pool=s.attn.v_pool)
    positions = np.concatenate([lens[i] + np.arange(n[i]) for i in range(b.B)])
    s2 = VerifyStep(b2, attn, None, rotary=s.rotary, positions=positions, shared=share(b2, spec.block_size, 608 // spec.block_size), weights=s.weights)
    before = s.weights.double().cpu().numpy()
    s2.run()
    torch.cuda.synchronize()
    turned = osv.rotate(attn.q.double().cpu().numpy(), s.rotary.cos_sin.cpu().numpy(), positions, s.rotary.style)
    assert np.allclose(s2.q.double().cpu().numpy(), turned, rtol=2 ** -8, atol=1e-5)   # its rounding; the products' in fp32
    check_attention(s2)
    want, size = osv.attention_weights(View(s2).k, qsl, b2.seq_lens, b.block_tables, s2.q.double().cpu().numpy(),
                                       float(np.float32(s2.scale)), s2.lse.double().cpu().numpy(), before, None, np.full(b.B, 608))
    got = s.weights.double().cpu().numpy()
    own = used_places(b2.seq_lens, b.block_tables, b.num_blocks, spec.block_size)
    own[b.block_tables[0, : 608 // spec.block_size]] = False
    own = np.broadcast_to(own[:, None, :], got.shape)
    assert (np.abs(got - want) <= U * size + 1e-30)[own].all() and np.array_equal(got[~own], before[~own])


def test_step_over_the_8_bit_cache():
    s = life(in8=True)
    s.run()
    torch.cuda.synchronize()
    check_attention(s)


def test_equal_to_a_step_without_sharing():
    """The same batch and blocks through the verification attention: the same but for the order of the sums."""
    s = life()
    plain = VerifyStep(s.batch, s.attn, s.acc, rotary=s.rotary)
    s.run()
    plain.run()
    torch.cuda.synchronize()
    assert torch.equal(s.q, plain.q) and not plain.tiles
    assert torch.allclose(s.out.float(), plain.out.float(), atol=2e-2, rtol=2e-2)   # either is within 1e-2 + 1e-2 |o|
    assert torch.equal(s.accepted_len, plain.accepted_len) and torch.equal(s.out_tokens, plain.out_tokens)


def test_replays_and_streams():
    s = life()
    w0 = s.weights.clone()
    s.run()
    torch.cuda.synchronize()
    outputs = (s.q, s.out, s.lse, s.accepted_len, s.out_tokens, s.lens_after, s.attn.k_pool, s.attn.v_pool, s.weights)
    want = [x.clone() for x in outputs]
    s.capture()
    side = torch.cuda.Stream()
    for turn in range(4):
        s.attn.q.neg_()   # other outputs between
        s.run()
        s.attn.q.neg_()
        s.weights.copy_(w0)
        s.out.zero_()
        torch.cuda.synchronize()
        if turn == 2:
            s.run(stream=side)
        else:
            s.replay()
        torch.cuda.synchronize()
        for x, y in zip(outputs, want):
            assert torch.equal(x, y), turn


def test_refusals():
    spec = wl.spec_with(1, batch=2)
    batch = wl.make_batch(spec, ctx_lens=[40, 50], k=[4, 4])
    attn = wl.make_attention_inputs8(spec, batch, device="cuda")
    with pytest.raises(ValueError):
        VerifyStep(batch, attn, None, weights=torch.zeros(1, device="cuda"))
    s = VerifyStep(batch, wl.make_attention_inputs(spec, batch, device="cuda"), None)
    with pytest.raises(ValueError):
        s.evict(torch.ones(2, dtype=torch.int32, device="cuda"), 1)
