"""Which keys an eviction chooses among, on the host: those that a workgroup holds in registers and those that it reads again
are together the keys between the ones that stay anyhow, each once."""
import os
import random
import subprocess

import pytest

from tests.test_attention_shares import ROOT

PROGRAM = r"""
#include <cstdio>
#include "tiles.h"
int main() {
  int S, keep, first, last, held;
  while (std::scanf("%d %d %d %d %d", &S, &keep, &first, &last, &held) == 5) {
    const spexis::EvictRange r = spexis::evict_range(S, keep, first, last);
    std::printf("%d %d %d %d\n", r.m, r.lo, r.hi, spexis::evict_rest(held, r.lo));
  }
}
"""


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    d = tmp_path_factory.mktemp("evict")
    (d / "p.cpp").write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "paper_2609_34370_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(cases):
        out = subprocess.run([str(d / "p")], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True,
                             check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return run


def test_keys_that_are_chosen_among(ranges):
    r = random.Random(3)
    cases = [(30000, 24000, 20000, 0, 16384), (20000, 18000, 17000, 7, 16384), (20000, 18000, 16384, 7, 16384),
             (20000, 18000, 16383, 7, 16384), (20000, 18000, 16385, 7, 16384), (40000, 35000, 35000, 9, 16384), (40000, 3, 1, 1, 16384)]
    for _ in range(3000):
        S = r.choice([r.randint(0, 300), r.randint(0, 300), r.randint(16000, 17000), r.randint(0, 60000)])
        near = [0, 1, S, S - 1, 16383, 16384, 16385, r.randint(-5, S + 5), r.randint(-5, S + 5)]
        cases.append((S, r.choice(near), r.choice(near), max(r.choice(near), 0), r.choice([4096, 16384])))
    for (S, keep, first, last, held), (m, lo, hi, rest) in zip(cases, ranges(cases)):
        assert m == min(max(keep, 0), S) and lo == min(max(first, 0), m) and hi == S - min(last, m - lo)
        assert 0 <= lo <= hi <= S and m - lo - (S - hi) >= 0
        # in registers [lo, hi) below `held`, read again [rest, hi): together [lo, hi), each once
        assert rest >= held and rest >= lo
        assert max(min(held, hi) - lo, 0) + max(hi - rest, 0) == hi - lo
