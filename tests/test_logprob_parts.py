"""How many workgroups share a row of the token log probabilities, on the host, and the workspace that it asks for."""
import os
import subprocess

import pytest

from paper_2609_34370_amd import spexis as sx
from tests.test_attention_shares import ROOT

PROGRAM = r"""
#include <cstdio>
#include "kernels.h"
int main() {
  long long items, vocab, sparse;
  while (std::scanf("%lld %lld %lld", &items, &vocab, &sparse) == 3)
    std::printf("%d\n", spexis::logprob_parts(items, vocab, sparse != 0));
}
"""


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    d = tmp_path_factory.mktemp("parts")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "paper_2609_34370_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def run(*cases):
        text = "\n".join(" ".join(map(str, map(int, c))) for c in cases)
        out = subprocess.run([str(d / "p")], input=text, capture_output=True, text=True, check=True).stdout
        return [int(x) for x in out.split()]

    return run


@pytest.mark.parametrize("items", [129, 170, 200, 256, 500, 5000])
def test_rows_that_two_or_three_parts_would_share_stay_whole(parts, items):
    # 200 rows of 128256 logits took 28.1 us in 2 parts and take 25.6, 256 33.0 and 28.1; of 60000 20.5 and 17.7
    assert parts((items, 60000, False), (items, 128256, False)) == [1, 1]


def test_few_rows_are_cut_where_that_is_quicker(parts):
    # one row of 41000 logits, 5 and 20 alternatives: 11.9 and 15.5 us whole, 11.3 and 12.4 in 6 parts; of 32000 10.6 whole, 11.3
    assert parts((1, 32000, False), (1, 36864, False), (1, 41000, False), (64, 49152, False), (65, 49152, False)) == [1, 1, 6, 6, 1]
    assert parts((128, 49153, False), (128, 128256, False), (1, 128256, False), (1, 1 << 22, False)) == [4, 4, 16, 64]


def test_items_that_pick_rows(parts):
    assert parts((576, 128256, True), (3000, 128256, True), (300, 49152, True), (256, 49152, True)) == [4, 1, 1, 6]


@pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built")
def test_the_workspace_is_enough_for_either_kind(parts):
    cases = [(i, v) for i in (1, 7, 63, 64, 65, 100, 128, 129, 170, 255, 256, 257, 600, 2047, 2048, 4096)
             for v in (1, 8192, 36864, 36865, 49152, 49153, 128256, 1 << 22)]
    most = [max(a, b) for a, b in zip(parts(*[(i, v, 0) for i, v in cases]), parts(*[(i, v, 1) for i, v in cases]))]
    for (i, v), n in zip(cases, most):
        for top in (0, 5, 32):
            assert sx.spexis_token_logprobs_workspace_size(i, v, top) == (i * n * (16 + 8 * top) if n > 1 else 0), (i, v, top)
