"""A stored traffic figure is used only while the sources of the call's kernels are as they were when it was taken, the
headers that they include among them."""
import os
import re
import shutil

import pytest

from tests.test_bench_cli import ROOT, load_bench

CSRC = os.path.join("paper_2609_34370_amd", "csrc")


def included(name):
    """name and every header of csrc that it includes, itself or through another."""
    found, left = set(), [name]
    while left:
        n = left.pop()
        if n not in found and os.path.exists(os.path.join(ROOT, CSRC, n)):
            found.add(n)
            left += re.findall(r'^#include "([^"]+)"', open(os.path.join(ROOT, CSRC, n)).read(), re.M)
    return sorted(found)


@pytest.mark.parametrize("call", ["verify_attention", "accept"])
def test_every_source_of_a_call_counts(call, tmp_path, monkeypatch):
    bench = load_bench()
    shutil.copytree(os.path.join(ROOT, CSRC), tmp_path / CSRC)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    sources = bench.TRAFFIC_CALLS[call][2]
    names = {n for s in sources for n in included(s)}
    assert {"common.h", "kernels.h"} <= names
    before = bench._kernel_digest(sources)
    for n in sorted(names):
        path = tmp_path / CSRC / n
        text = path.read_text()
        path.write_text(text + "// another line\n")
        assert bench._kernel_digest(sources) != before, n
        path.write_text(text)
    assert bench._kernel_digest(sources) == before
    other = tmp_path / CSRC / "lookahead.hip"
    other.write_text(other.read_text() + "// another line\n")
    assert bench._kernel_digest(sources) == before
