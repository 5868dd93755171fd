"""A verification step with the rotating append, the 8-bit cache and the emitted tokens' log probabilities together:
every stage against its 64-bit form on the GPU's own inputs of the stage, then the step as a replayed graph and on
streams of its own against the eager one, bit for bit."""
import sys

import numpy as np
import pytest
import torch

from oracle import serving as osv
from paper_2609_34370_amd import spexis as sx
from paper_2609_34370_amd import workloads as wl
from paper_2609_34370_amd.step import VerifyStep
from tests import layout_ref
from tests.test_gpu_attention8 import check as check_attention8
from tests.test_gpu_logprobs import compare as compare_logprobs
from tests.test_gpu_rotate import _magnitude, same_codes

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


# workload, batch, contexts, drafts, rotary_dim, style
CASES = [
    (1, 4, [40, 47, 200, 32], [4, 4, 4, 4], 64, 0),
    (4, 5, [300, 31, 17, 256, 64], [0, 8, 3, 1, 5], 128, 0),
    (5, 3, [70, 600, 31], [8, 8, 8], 64, 1),
]


def step_of(case, in8, seed=None, top=7):
    wid, B, ctx, k, rot, style = CASES[case]
    spec = wl.spec_with(wid, batch=B, vocab=min(wl.WORKLOADS[wid].vocab, 5003))
    batch = wl.make_batch(spec, ctx_lens=ctx, k=k, seed=seed)
    attn = (wl.make_attention_inputs8 if in8 else wl.make_attention_inputs)(spec, batch, device="cuda", seed=seed)
    acc = wl.make_accept_inputs(spec, batch, device="cuda", seed=seed)
    rotary = wl.make_rotary_inputs(batch.max_seq_len, rot, device="cuda", style=style)
    return VerifyStep(batch, attn, acc, rotary=rotary, top_logprobs=top)


def outputs(s):
    out = [s.q, s.out, s.accepted_len, s.out_tokens, s.logprob, s.entropy, s.top_ids, s.top_logprob, s.attn.k_pool, s.attn.v_pool]
    return [t.clone().view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.clone() for t in out + ([s.attn.scales] if s.in8 else [])]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("in8", [True, False])
def test_every_stage(case, in8):
    s = step_of(case, in8)
    b, spec, a, r = s.batch, s.spec, s.attn, s.rotary
    say(f"[step] workload {spec.wid} B={b.B} 8 bit {in8}")
    D, hkv, bs = spec.head_dim, spec.num_kv_heads, spec.block_size
    cs, pos = r.cos_sin.cpu().numpy(), osv.token_positions(b.qsl, b.seq_lens)
    new_k, new_v = a.new_k.double().cpu().numpy(), a.new_v.double().cpu().numpy()
    k = osv.rotate(new_k, cs, pos, r.style)
    if in8:
        places = osv.places8(b.num_blocks, hkv, bs, D)
        codes = [pool.view(torch.uint8).cpu().numpy()[p] for pool, p in zip((a.k_pool, a.v_pool), places)]
        scales = a.scales.cpu().numpy().copy()
        for part, rows in enumerate((k.astype(np.float32), new_v)):
            one = scales[:, :, part].copy()
            osv.append8(codes[part], one, b.qsl, b.seq_lens, b.block_tables, rows)
            scales[:, :, part] = one
    s.run()
    torch.cuda.synchronize()
    q = osv.rotate(a.q.double().cpu().numpy(), cs, pos, r.style)
    bound = 2.0 ** -8 * np.abs(q) + 3 * 2.0 ** -24 * _magnitude(a.q.double().cpu().numpy(), cs, pos, r.style)
    assert (np.abs(s.q.double().cpu().numpy() - q) <= bound).all()
    if in8:
        assert np.array_equal(a.scales.cpu().numpy(), scales)
        for pool, c, p in zip((a.k_pool, a.v_pool), codes, places):
            same_codes(pool.view(torch.uint8).cpu().numpy()[p], c)
        check_attention8(s.out, codes, scales, b.qsl, b.seq_lens, b.block_tables, s.q, float(np.float32(s.scale)))
    else:
        kp, vp = a.k_pool.double().cpu().numpy(), a.v_pool.double().cpu().numpy()
        for i in range(b.B):
            lo, hi, L, S = int(b.qsl[i]), int(b.qsl[i + 1]), int(b.ctx_lens[i]), int(b.seq_lens[i])
            rows = layout_ref.gather_seq(kp, "k", b.block_tables[i], S, hkv, bs, D)
            ref = k[lo:hi]
            bound = 2.0 ** -8 * np.abs(ref) + 3 * 2.0 ** -24 * _magnitude(new_k[lo:hi], cs, pos[lo:hi], r.style)
            assert (np.abs(rows[L:] - ref) <= bound).all()
            vrows = layout_ref.gather_seq(vp, "v", b.block_tables[i], S, hkv, bs, D)
            assert np.array_equal(vrows[L:], new_v[lo:hi])
            # the attention's own tolerance is 1e-2 + 1e-2 |o|
            G = spec.num_q_heads // hkv
            for j in range(hi - lo):
                x = np.einsum("thd,hgd->hgt", rows[: L + j + 1], s.q[lo + j].double().cpu().numpy().reshape(hkv, G, D)) * s.scale
                w = np.exp(x - x.max(axis=-1, keepdims=True))
                o = np.einsum("hgt,thd->hgd", w / w.sum(axis=-1, keepdims=True), vrows[: L + j + 1]).reshape(-1, D)
                assert (np.abs(s.out[lo + j].double().cpu().numpy() - o) <= 1e-2 + 1e-2 * np.abs(o)).all()
    accepted, tokens, _ = s.accept_outputs()
    rows = s.rows.cpu().numpy().reshape(-1)
    assert ((tokens >= 0).sum(axis=1) == accepted + 1).all()
    n = tokens.size
    got = [t.cpu().numpy().reshape(n, -1) if t.dim() == 3 else t.cpu().numpy().reshape(n)
           for t in (s.logprob, s.entropy, s.top_ids, s.top_logprob)]
    compare_logprobs(got, s.acc.target_logits, tokens.reshape(-1).tolist(), rows.tolist(), s.acc.temperature, 7)


@pytest.mark.parametrize("in8", [True, False])
def test_replays_equal_the_eager_step(in8):
    """Replays of two captured steps that share nothing, with the eager steps and other inputs between them."""
    steps = [step_of(case, in8) for case in (0, 1)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(outputs(s))
    graphs = [s.capture() for s in steps]
    for turn in range(3):
        for s in steps:   # other queries: the outputs change ...
            s.attn.q.neg_()
            s.run()
            s.attn.q.neg_()
            s.out.zero_()
            s.logprob.zero_()
            s.top_ids.zero_()
        for g in graphs:  # ... and come back
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            for x, y in zip(outputs(s), w):
                assert torch.equal(x, y), turn


def test_steps_on_their_own_streams():
    steps = [step_of(case, True) for case in (0, 1, 2)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(outputs(s))
    streams = [torch.cuda.Stream() for _ in steps]
    for s in steps:
        s.out.zero_()
        s.q.zero_()
        s.top_logprob.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for s, stream in zip(steps, streams):
            s.run(stream=stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for x, y in zip(outputs(s), w):
            assert torch.equal(x, y)


def test_a_rejected_row_is_overwritten():
    """Two steps of one sequence: the second begins where the first's accepted tokens end, inside a block whose scale the
    rejected rows had raised.  The scale stays, what the first step accepted stays, and the attention sees it."""
    hq, hkv, D, bs = 4, 2, 64, 16
    r = np.random.default_rng(8)
    tables = np.array([[2, 0, 1]], np.int32)
    codes = [np.zeros((3, bs, hkv, D), np.uint8) for _ in range(2)]
    scales = np.ones((3, hkv, 2), np.float32)
    places = osv.places8(3, hkv, bs, D)
    pools = [torch.zeros(c.size, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for c in codes]
    sc = torch.ones((3, hkv, 2), device="cuda")
    held = 0
    for n, keep, size in ((20, 20, 1.0), (5, 2, 50.0), (4, 4, 1.0), (9, 1, 3.0), (1, 1, 1.0)):
        S = held + n
        qsl, sl = np.array([0, n], np.int32), np.array([S], np.int32)
        new = [torch.from_numpy((size * r.standard_normal((n, hkv, D))).astype(np.float32)).to(torch.bfloat16) for _ in range(2)]
        dev = [torch.as_tensor(x).cuda() for x in (qsl, sl, tables)]
        sx.spexis_rotate_append_kv8(*pools, sc, 3, hkv, bs, D, *dev, n, n, new[0].cuda(), new[1].cuda())
        torch.cuda.synchronize()
        for part in range(2):
            one = scales[:, :, part].copy()
            osv.append8(codes[part], one, qsl, sl, tables, new[part].double().numpy())
            scales[:, :, part] = one
            same_codes(pools[part].view(torch.uint8).cpu().numpy()[places[part]], codes[part])
        assert np.array_equal(sc.cpu().numpy(), scales)
        q = torch.from_numpy(r.standard_normal((n, hq, D)).astype(np.float32)).to(torch.bfloat16).cuda()
        out = torch.empty_like(q)
        ws = torch.empty(sx.spexis_verify_attention_kv8_workspace_size(1, hq, hkv, D, n, S), dtype=torch.uint8, device="cuda")
        sx.spexis_verify_attention_kv8(*pools, sc, 3, hkv, bs, D, *dev, n, n, S, q, hq, 0.125, out, ws)
        torch.cuda.synchronize()
        check_attention8(out, codes, scales, qsl, sl, tables, q, 0.125)
        held += keep
