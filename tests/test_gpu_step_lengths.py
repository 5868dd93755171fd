"""What a step with attention weights leaves behind however it is run: as a whole, call by call, behind an eviction,
captured, evicted from more than once.  The same kernels on the same inputs: bit for bit."""
import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import workloads as wl
from paper_2609_34370_amd.step import VerifyStep
from tests.test_gpu_cache_life import View, life
from tests.test_gpu_evict import used_places

pytestmark = pytest.mark.gpu


def prompts():
    """Without acceptance and without sharing."""
    spec = wl.spec_with(4, batch=3, num_q_heads=8, num_kv_heads=4)
    batch = wl.make_batch(spec, ctx_lens=[0, 33, 500], k=[80, 70, 0])
    weights = torch.rand((batch.num_blocks, spec.num_kv_heads, spec.block_size), device="cuda",
                         generator=torch.Generator("cuda").manual_seed(6))
    return VerifyStep(batch, wl.make_attention_inputs(spec, batch, device="cuda"), None, weights=weights)


@pytest.mark.parametrize("make", [life, prompts])
def test_call_by_call(make):
    s = make()
    w0 = s.weights.clone()
    s.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in (s.out, s.lse, s.weights, s.lens_after)]
    t = make()   # (a step of its own: nothing that run() has left)
    t.weights.copy_(w0)
    for turn in range(2):   # the second time behind an eviction, which changes lens_after
        t.append()
        t.attention()
        if t.acc is not None:
            t.accept()
        t.add_weights()
        torch.cuda.synchronize()
        for x, y in zip((t.out, t.lse, t.weights, t.lens_after), want):
            assert torch.equal(x, y), turn
        pools = [x.clone() for x in (t.attn.k_pool, t.attn.v_pool)]
        t.evict(torch.full_like(t.seq_lens, 300), 4)
        for x, y in zip((t.attn.k_pool, t.attn.v_pool), pools):
            x.copy_(y)
        t.weights.copy_(w0)


@pytest.mark.parametrize("capture", [False, True])
def test_a_step_behind_an_eviction_starts_from_its_own_lengths(capture):
    """The next run of the same step is the step's again, also as a graph."""
    s = life()
    w0, pools = s.weights.clone(), [x.clone() for x in (s.attn.k_pool, s.attn.v_pool)]
    s.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in (s.out, s.lse, s.weights, s.lens_after, s.attn.k_pool, s.attn.v_pool)]
    if capture:
        s.weights.copy_(w0)
        s.capture()
    for _ in range(3):
        s.evict(torch.full_like(s.seq_lens, 620), 8)
        s.weights.copy_(w0)
        for x, y in zip((s.attn.k_pool, s.attn.v_pool), pools):
            x.copy_(y)
        s.replay() if capture else s.run()
        torch.cuda.synchronize()
        for x, y in zip((s.out, s.lse, s.weights, s.lens_after, s.attn.k_pool, s.attn.v_pool), want):
            assert torch.equal(x, y)


def test_evictions_one_after_the_other():
    """The second goes on from what the first has left."""
    s = life()
    b, spec = s.batch, s.spec
    s.run()
    torch.cuda.synchronize()
    lens, w = s.lens_after.cpu().numpy(), s.weights.cpu().numpy().copy()
    c, first = View(s), np.full(b.B, 608)
    k, v = c.k, c.v
    for most in (640, 620, 620):
        keep = np.minimum(most, lens).astype(np.int32)
        new = s.evict(torch.as_tensor(keep).cuda(), 8)
        torch.cuda.synchronize()
        k, v, w, lens = osv.evict(k, v, w, lens, b.block_tables, keep, first, 8)
        assert np.array_equal(new.cpu().numpy(), lens)
        kept = used_places(lens, b.block_tables, b.num_blocks, spec.block_size)
        now = View(s)
        assert np.array_equal(now.k[kept], k[kept]) and np.array_equal(now.v[kept], v[kept])
        assert np.array_equal(s.weights.cpu().numpy().transpose(0, 2, 1)[kept], w.transpose(0, 2, 1)[kept])


def test_capture_adds_no_weights():
    """Two replays add the weights of two steps: recording runs the step for warm-up, which must not count."""
    s = life()
    w0 = s.weights.clone()
    s.run()
    s.run()
    torch.cuda.synchronize()
    want = s.weights.clone()
    s.weights.copy_(w0)
    s.capture(warmup=2)
    torch.cuda.synchronize()
    assert torch.equal(s.weights, w0)
    s.replay()
    s.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.weights, want)
