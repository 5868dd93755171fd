"""Which append or query each workgroup of the rotating appends is, on the host: every one once, and where the two kinds
alternate, each kind evenly over the eight XCDs (a workgroup runs on XCD index mod 8)."""
import os
import subprocess

import pytest

from tests.test_attention_shares import ROOT

PROGRAM = r"""
#include <cstdio>
#include "kernels.h"
int main() {
  long long appends, queries, alternate;
  while (std::scanf("%lld %lld %lld", &appends, &queries, &alternate) == 3) {
    int mix = 0;
    const long long groups = spexis::rotate_groups(appends, queries, alternate != 0, &mix);
    std::printf("%lld", groups);
    for (long long w = 0; w < groups; ++w) {
      const spexis::RotatePlace p = spexis::rotate_place((int)w, mix, (int)appends);
      std::printf(" %c%d", p.append ? 'a' : 'q', p.index);
    }
    std::printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    d = tmp_path_factory.mktemp("places")
    (d / "p.cpp").write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "paper_2609_34370_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(appends, queries, alternate):
        out = subprocess.run([str(d / "p")], input=f"{appends} {queries} {int(alternate)}", capture_output=True, text=True,
                             check=True).stdout.split()
        assert len(out) == int(out[0]) + 1
        return [(x[0], int(x[1:])) for x in out[1:]]

    return run


SIZES = [(1, 0), (8, 0), (777, 0), (1, 1), (1, 40), (40, 1), (5, 5), (16, 40), (100, 101), (640, 640), (640, 1280), (4096, 640),
         (4096, 1152), (2048, 4608), (2048, 2560), (1024, 160), (8192, 640), (900, 6300), (6300, 900), (512, 1536)]


@pytest.mark.parametrize("appends,queries", SIZES)
@pytest.mark.parametrize("alternate", [False, True])
def test_every_one_is_a_workgroup_once(places, appends, queries, alternate):
    got = places(appends, queries, alternate)
    for kind, n in (("a", appends), ("q", queries)):
        index = [i for k, i in got if k == kind]
        assert sorted(i for i in index if i < n) == list(range(n))   # others leave at once
        assert all(i >= 0 for i in index) and len(set(index)) == len(index)
    assert len(got) <= 2 * (appends + queries) + 8


@pytest.mark.parametrize("appends,queries", [s for s in SIZES if min(s) >= 100])
def test_both_kinds_lie_on_every_xcd_alike(places, appends, queries):
    """4096 appends and 640 queries used to alternate seven to one: every query on one XCD of the eight."""
    got = places(appends, queries, True)
    for kind, n in (("a", appends), ("q", queries)):
        by = [sum(k == kind and i < n for k, i in got[x::8]) for x in range(8)]
        assert max(by) <= n / 8 * 1.1 + 3, (kind, by)
        # and along the launch: the kind is as frequent in each quarter, up to where its last one lies
        last = max(w for w, (k, i) in enumerate(got) if k == kind and i < n) + 1
        quarters = [sum(k == kind and i < n for k, i in got[last * j // 4: last * (j + 1) // 4]) for j in range(4)]
        assert max(quarters) <= n / 4 * 1.25 + 8, (kind, quarters)


BLOCKS = r"""
#include <cstdio>
#include "kernels.h"
int main() {
  int seqs, blocks;
  while (std::scanf("%d %d", &seqs, &blocks) == 2) {
    for (int i = 0; i < seqs * blocks; ++i) {
      const spexis::RotateBlock b = spexis::rotate_block(i, seqs);
      std::printf("%d %d ", b.seq, b.nth);
    }
    std::printf("\n");
  }
}
"""


@pytest.mark.parametrize("seqs,blocks,heads", [(64, 2, 4), (128, 2, 4), (64, 2, 2), (100, 2, 1), (37, 4, 2), (512, 2, 8), (3, 40, 4)])
def test_the_blocks_that_get_rows_lie_on_every_xcd_alike(tmp_path, seqs, blocks, heads):
    """A step's few rows touch one block of a sequence, of the two that it has places for: with four heads the one used to
    be on XCDs 0 to 3 and the empty one on 4 to 7."""
    (tmp_path / "b.cpp").write_text(BLOCKS)
    r = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "paper_2609_34370_amd", "csrc"), str(tmp_path / "b.cpp"), "-o", str(tmp_path / "b")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([str(tmp_path / "b")], input=f"{seqs} {blocks}", capture_output=True, text=True, check=True).stdout
    v = [int(x) for x in out.split()]
    got = list(zip(v[::2], v[1::2]))
    assert sorted(got) == [(s, n) for s in range(seqs) for n in range(blocks)]
    for nth in range(blocks):
        at = [(i * heads + h) % 8 for i, g in enumerate(got) if g[1] == nth for h in range(heads)]
        by = [at.count(x) for x in range(8)]
        assert max(by) - min(by) <= 1, by
