"""Token log probabilities of rows that are cut into parts (a second launch combines them), and of long rows in one
part: rows of every kind, whole parts masked, as many alternatives as there may be, searched thresholds of later rounds.
Tolerances as tests/test_gpu_logprobs.py."""
import sys

import numpy as np
import pytest
import torch

from paper_2609_34370_amd import spexis as sx
from tests.test_gpu_logprobs import call, check, rows_of_every_kind

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
