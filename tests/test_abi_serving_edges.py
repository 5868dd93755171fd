"""More refusals of the serving operators, and the sizes that their binding checks (no GPU needed)."""
import os

import pytest
import torch

from paper_2609_34370_amd import spexis as sx
from tests.test_abi_serving import INVALID, ODD, rotate

no_gpu = [pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built"),
          pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation runs only without a GPU")]


def marked(f):
    for m in no_gpu:
        f = m(f)
    return f


@marked
def test_scales_that_the_attention_refuses_are_refused_by_the_append():
    assert rotate(True, sc=ODD) == INVALID and b"16-byte aligned" in sx.lib().spexis_last_error()
