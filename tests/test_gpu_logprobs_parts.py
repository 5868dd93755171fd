"""Token log probabilities of rows that are cut into parts (a second launch combines them), and of long rows in one
part: rows of every kind, whole parts masked, as many alternatives as there may be, searched thresholds of later rounds.
Tolerances as tests/test_gpu_logprobs.py."""
import sys

import numpy as np
import pytest
import torch

from paper_2609_34370_amd import spexis as sx
from tests.test_gpu_logprobs import call, check, compare, rows_of_every_kind

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def test_no_row_to_ask_for():
    """Logits without a row: every item's row is out of range."""
    n, top = 3, 4
    lp, h = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ids, alt = torch.full((n, top), -7, dtype=torch.int32, device="cuda"), torch.full((n, top), 7.0, device="cuda")
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    for V in (50, 100000):
        say(f"[logprobs] no rows, V={V}")
        for t in (lp, h, alt):
            t.fill_(7.0)
        ids.fill_(-7)
        ws = torch.empty(max(sx.spexis_token_logprobs_workspace_size(n, V, top), 16), dtype=torch.uint8, device="cuda")
        sx.spexis_token_logprobs(torch.empty((0, V), device="cuda"), zero, lp, ws, row_ids=zero, entropy=h, top_ids=ids,
                                 top_logprobs=alt)
        torch.cuda.synchronize()
        assert not lp.any() and not h.any() and (ids == -1).all() and (alt == -float("inf")).all()


def rows_of_parts(V, r, dtype):
    """What the parts of a row can differ in: masked but in one, equal in all, the largest entries one in each, a value
    that leaves no distribution in one alone."""
    low = torch.finfo(dtype).min
    n = r.standard_normal((10, V)) * 3
    n[0][5:] = -np.inf                       # the first part alone holds logits, fewer than alternatives
    n[1][: V - 40] = -np.inf                 # the last one alone
    n[2][V // 3:] = low
    n[3] = -2.5                              # every part's n-th key has the same logit
    n[4][:: V // 23] = 50.0                  # ties over all parts
    n[5] = np.sort(n[5])
    n[6][V - 2] = np.nan
    n[7][1] = np.inf
    n[8][: V // 2] = -np.inf
    n[8][V // 2:] = low
    n[9][r.random(V) < 0.999] = -np.inf
    n[9][::8192] = np.arange(len(n[9][::8192])) / 7
    t = torch.from_numpy(n)
    return torch.where(t == -np.inf, t, t.clamp(min=low)).to(dtype)


@pytest.mark.parametrize("V", [50021, 131075])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 1, 20, 32])
def test_rows_in_parts(V, dtype, top):
    r = np.random.default_rng(V + top)
    say(f"[logprobs] in parts, V={V} {dtype} top {top}")
    assert sx.spexis_token_logprobs_workspace_size(10, V, top) > 0
    for make in (rows_of_every_kind, rows_of_parts):
        x = make(V, r, dtype)
        tokens = r.integers(0, V, len(x))
        tokens[:2] = 3, V - 1
        check(x.cuda(), tokens.tolist(), None, 0.7 if top == 20 else 1.0, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", [(1, 1), (3, 2)])
def test_parts_of_rows_that_start_anywhere(dtype, pad, shift):
    r = np.random.default_rng(pad)
    V = 50023
    flat = torch.full((shift + 5 * (V + pad),), float("nan"), dtype=dtype)   # what lies between the rows is not read
    x = flat[shift:].view(5, V + pad)[:, :V]
    x.copy_(torch.from_numpy(r.standard_normal((5, V)) * 3))
    say(f"[logprobs] in parts, {dtype} pad {pad} shift {shift}")
    check(flat.cuda()[shift:].view(5, V + pad)[:, :V], r.integers(0, V, 5).tolist(), None, 1.0, 20)


@pytest.mark.parametrize("items", [1, 3, 70, 700])
def test_items_pick_rows_in_parts(items):
    """Rows several times, in any order; tokens and rows out of range."""
    r = np.random.default_rng(items)
    V, n = 60011, 40
    x = torch.from_numpy((r.standard_normal((n, V)) * 3).astype(np.float32)).cuda()
    rows, tokens = r.integers(-1, n + 1, items), r.integers(-2, V + 2, items)
    tokens[::3] = -1
    if items == 1:
        rows[0], tokens[0] = 7, V - 1
    say(f"[logprobs] in parts, {items} items")
    check(x, tokens.tolist(), rows.tolist(), 0.9, 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scored_rows_in_one_part(dtype):
    """As many rows as are scored whole, of a vocabulary that takes a second common threshold: rows of every kind between
    ordinary ones."""
    V, n, top = 152064, 520, 5
    assert sx.spexis_token_logprobs_workspace_size(2100, V, top) == 0   # (a workspace is asked for items that pick rows)
    r = np.random.default_rng(7)
    x = torch.empty((n, V), dtype=dtype, device="cuda")
    x.copy_(torch.from_numpy(r.standard_normal(V).astype(np.float32)).cuda() * 4)
    x += torch.arange(n, device="cuda")[:, None].to(dtype)
    tokens = r.integers(0, V, n)
    special = torch.cat([rows_of_every_kind(V, r, dtype), rows_of_parts(V, r, dtype)])
    at = np.sort(r.permutation(n)[: len(special)])
    x[torch.as_tensor(at).cuda()] = special.cuda()
    say(f"[logprobs] scored whole, {dtype}")
    got = call(x, tokens.tolist(), None, 0.7, top)
    some = np.sort(np.concatenate([at, [0, 1, n - 1]]))
    some = np.unique(some)
    compare([g[some] for g in got], x[torch.as_tensor(some).cuda()], tokens[some].tolist(), None, 0.7, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_rows_in_one_part(dtype):
    """More than 32 rounds of loads a workgroup: a threshold that all four waves share is found a third time."""
    V, items, top = 300007, 2048, 20
    r = np.random.default_rng(8)
    x = torch.cat([rows_of_parts(V, r, dtype), rows_of_every_kind(V, r, dtype)[:4]])
    rows, tokens = r.integers(0, len(x), items), r.integers(0, V, items)
    assert sx.spexis_token_logprobs_workspace_size(items, V, top) == 0
    say(f"[logprobs] long rows, {dtype}")
    got = call(x.cuda(), tokens.tolist(), rows.tolist(), 1.0, top)
    first = np.unique(rows, return_index=True)[1]
    compare([g[first] for g in got], x.cuda(), tokens[first].tolist(), rows[first].tolist(), 1.0, top)
    for i in range(items):   # the same row, the same answer
        j = first[np.searchsorted(rows[first], rows[i])]
        assert np.array_equal(got[1][i], got[1][j], equal_nan=True) and np.array_equal(got[2][i], got[2][j])
