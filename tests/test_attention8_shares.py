"""The shares of the attention over the 8-bit cache, on the host: an item counts as more positions than it has tiles, and
the rule for the fewest tiles of a share, which is about tiles, must not see those."""
import os
import subprocess

import pytest

from tests.test_attention_shares import ROOT, restated

PROGRAM = r"""
#include <cstdio>
#include "kernels.h"
int main() {
  int tiles, seqs, hkv, dim, rows, cost, shares;
  while (std::scanf("%d %d %d %d %d %d %d", &tiles, &seqs, &hkv, &dim, &rows, &cost, &shares) == 7)
    std::printf("%d\n", spexis::attn_share_positions(spexis::attn_least(seqs, hkv, dim, rows), tiles, seqs, cost, shares));
}
"""


@pytest.fixture(scope="module")
def positions(tmp_path_factory):
    d = tmp_path_factory.mktemp("shares8")
    (d / "p.cpp").write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "paper_2609_34370_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.run([str(d / "p")], input=text, capture_output=True, text=True, check=True).stdout
        return [int(x) for x in out.split()]

    return run


CASES = [(seqs * nt, seqs, hkv, dim, rows, cost, 1024 // hkv) for seqs in (1, 4, 16, 64, 128, 512) for nt in (1, 2, 3, 4, 5, 8, 20, 300)
         for hkv in (1, 2, 8) for dim in (64, 128) for rows in (4, 8, 20, 63) for cost in (0, 4)]


def test_the_fewest_tiles_of_a_share_follow_from_tiles(positions):
    want = [max(restated(tiles, seqs, hkv, dim, rows), -(-(tiles + cost * seqs) // shares))
            for tiles, seqs, hkv, dim, rows, cost, shares in CASES]
    assert positions(CASES) == want


@pytest.mark.parametrize("seqs,hkv", [(64, 8), (128, 4), (512, 1)])
def test_sequences_of_four_tiles_go_whole_to_one_share(positions, seqs, hkv):
    # counted as eight tiles each they got shares of 6, and took 1.11 to 1.34 times as long (8 and 20 rows)
    for rows in (8, 20):
        assert positions([(4 * seqs, seqs, hkv, 128, rows, 4, 1024 // hkv)]) == [4]
