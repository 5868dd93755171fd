"""What the compiler makes of the serving operators' kernels: no register spilled, no packed fp32 instruction, and no
kernel larger than the instruction cache (64 KB for two CUs)."""
import os
import re
import subprocess

import pytest

from paper_2609_34370_amd import build

SOURCES = ["attention8.hip", "rotate.hip", "logprobs.hip"]


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")
    jobs = {}
    for src in SOURCES:
        out = str(d / (src + ".s"))
        cmd = [build.HIPCC, *build.FLAGS, "-S", "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage",
               os.path.join(build.CSRC, src), "-o", out]
        jobs[src] = (out, subprocess.Popen(cmd, stderr=subprocess.PIPE, text=True))
    result = {}
    for src, (out, p) in jobs.items():
        remarks = p.communicate()[1]
        assert p.returncode == 0, remarks
        result[src] = (open(out).read(), remarks)
    return result


@pytest.mark.parametrize("src", SOURCES)
def test_code(compiled, src):
    asm, remarks = compiled[src]
    names = re.findall(r"Function Name: (\S+)", remarks)
    for kind in ("VGPRs Spill", "ScratchSize \\[bytes/lane\\]"):
        found = [int(x) for x in re.findall(kind + r": (\d+)", remarks)]
        assert names and len(found) == len(names) and not any(found), (kind, dict(zip(names, found)))
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)
    assert max(int(x) for x in re.findall(r"codeLenInByte = (\d+)", asm)) <= 65536
