"""The numbers of the units of a launch that holds shared prefixes and sequences, on the host: a prefix's partials lie in slots
of its units' numbers, so every one of them must be below the slots that the layout gives to prefixes."""
import os
import random
import subprocess

import pytest

from tests.test_attention_shares import ROOT

# For a batch: its sizes, of every segment (prefixes in front) whether it is a prefix, its row tiles and its key tiles.
# Prints merge, the slots of prefixes, units in all, and of every segment its first unit and its units.
PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "tiles.h"
using namespace spexis;
int main() {
  long seqs, groups, hq, hkv, dim, T, longest, keys;
  int ns;
  while (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld %d", &seqs, &groups, &hq, &hkv, &dim, &T, &longest, &keys, &ns) == 9) {
    const TileLayout l = tile_layout(seqs, groups, hq, hkv, dim, T, longest, keys);
    std::vector<std::vector<int>> seg(ns, std::vector<int>(2));
    std::vector<int> prefix(ns), tiles(ns), nt(ns);
    int64_t sum = 0;
    int rows = 0;
    for (int s = 0; s < ns; ++s) {
      if (std::scanf("%d %d %d", &prefix[s], &tiles[s], &nt[s]) != 3) return 1;
      sum += (int64_t)tiles[s] * nt[s];
      rows += tiles[s];
    }
    const int share = l.shares > 0 ? tile_attn_share(l.shares, tile_keys((int)dim), sum, rows) : INT32_MAX;
    for (int s = 0; s < ns; ++s) seg[s] = {nt[s], tiles[s] * tile_parts(nt[s], share)};
    std::printf("%d %ld %ld", (int)l.merge, (long)l.prefix_units, (long)l.units);
    int index = 0;
    for (int s = 0; s < ns; ++s) {
      int all = 0;
      const int at = tile_by_length((int)groups, l.shares, ns) ? tile_first_unit(seg, ns, s, &all) : index;
      std::printf(" %d %d", at, seg[s][1]);
      index += seg[s][1];
    }
    std::printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def numbers(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "p.cpp").write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "paper_2609_34370_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(batches):
        lines = []
        for (hkv, G, dim, groups, n, own) in batches:
            pre, segs = [0] * len(n), []
            for lo, hi, keys in groups:
                rows = sum(n[lo:hi]) * G if keys else 0
                segs.append((1, -(-rows // 128), -(-keys // (32 if dim == 128 else 64))))
                pre[lo:hi] = [keys] * (hi - lo)
            for b in range(len(n)):   # (their own keys begin at the prefix's end)
                segs.append((0, -(-n[b] * G // 128), -(-(own[b] + n[b]) // (32 if dim == 128 else 64))))
            most = max(p + o + x for p, o, x in zip(pre, own, n))
            lines.append(" ".join(map(str, (len(n), len(groups), G * hkv, hkv, dim, sum(n), max(n), most, len(segs),
                                            *(x for s in segs for x in s)))))
        out = subprocess.run([str(d / "p")], input="\n".join(lines), capture_output=True, text=True, check=True).stdout
        result = []
        for line, (*_, groups, n, _) in zip(out.splitlines(), batches):
            merge, slots, units, *x = map(int, line.split())
            result.append((merge, slots, units, x[0:2 * len(groups):2], x[1:2 * len(groups):2], x[0::2], x[1::2]))
        assert len(result) == len(batches)
        return result

    return run


def check(batch, got):
    merge, slots, units, first, count, firsts, counts = got
    assert all(a + c <= slots for a, c in zip(first, count) if c), batch
    # every unit has one segment, and they are as many as the launch holds at most
    assert sum(counts) <= units, batch
    at = 0
    for a, c in sorted((a, c) for a, c in zip(firsts, counts) if c):
        assert a == at, batch
        at += c


@pytest.mark.parametrize("hkv,G,dim,groups,n,own", [
    (32, 1, 64, [(0, 40, 512)], [5] * 40, [1000] * 40),
    (16, 2, 128, [(0, 60, 512)], [5] * 60, [1000] * 60),
    (24, 1, 128, [(0, 33, 512)], [5] * 33, [1000] * 33),
    (8, 4, 128, [(0, 62, 512)], [5] * 62, [16000] * 12 + [1000] * 50),
    (8, 4, 128, [(0, 62, 512)], [34] * 62, [1000] * 62),
    (16, 1, 64, [(0, 63, 512)], [9] * 63, [700] * 63),    # 64 segments
    (16, 1, 64, [(0, 64, 512)], [9] * 64, [700] * 64),    # and 65
])
def test_prefixes_shorter_than_what_follows(numbers, hkv, G, dim, groups, n, own):
    batch = (hkv, G, dim, groups, n, own)
    got = numbers([batch])[0]
    assert got[0]
    check(batch, got)


def test_any_batch(numbers):
    r = random.Random(1)
    batches = []
    for _ in range(6000):
        seqs = r.choice([r.randint(1, 63), r.randint(1, 63), r.randint(64, 90)])
        cuts = sorted(r.choices(range(seqs + 1), k=r.randint(2, 7)))
        groups = [(a, b, r.choice([0, 64, 512, 2048, 8192])) for a, b in zip(cuts, cuts[1:])]
        n = [r.choice([0, 1, 5, 9, 40, 130]) for _ in range(seqs)]
        n[0] = n[0] or 1
        batches.append((r.choice([1, 2, 4, 8, 16, 32]), r.choice([1, 2, 4, 7, 8]), r.choice([64, 128]), groups, n,
                        [r.choice([10, 1000, 16000]) for _ in range(seqs)]))
    merged = 0
    for batch, got in zip(batches, numbers(batches)):
        if got[0]:   # (otherwise prefixes are alone in their launch)
            merged += 1
            check(batch, got)
    assert merged > 2000


def test_prompts_of_any_lengths(numbers):
    """Without prefixes: every unit has one segment, the longest sequences first where they are few and their tiles whole."""
    r = random.Random(2)
    batches = []
    for _ in range(2000):
        seqs = r.choice([r.randint(1, 8), r.randint(1, 64), 8, 9])
        n = [r.choice([0, 1, 5, 200, 3000]) for _ in range(seqs)]
        n[0] = n[0] or 1
        batches.append((r.choice([1, 2, 8, 32]), r.choice([1, 4, 7]), r.choice([64, 128]), [], n, [r.choice([10, 1000, 16000]) for _ in range(seqs)]))
    ordered = 0
    for batch, got in zip(batches, numbers(batches)):
        check(batch, got)
        if not got[0] and len(batch[4]) <= 8:
            ordered += 1
            step = 32 if batch[2] == 128 else 64
            nt = [-(-(o + x) // step) for o, x in zip(batch[5], batch[4])]
            lengths = [k for _, k in sorted((a, k) for a, c, k in zip(got[5], got[6], nt) if c)]
            assert lengths == sorted(lengths, reverse=True)
    assert ordered > 100
