"""Rows before the first sequence's and behind the last one's are left as they were: which
rows of a group of tokens the append takes, over all sizes that the header allows, compiled
for the host. CPU only."""

import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2608_04048_amd", "csrc")
MOST = 1 << 26


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rows_of_a_group(tmp_path):
    exe = tmp_path / "rows"
    subprocess.run(["g++", "-O1", "-std=c++17", "-fwrapv", f"-I{CSRC}",
                    os.path.join(HERE, "csrc", "append_rows.cpp"), "-o", str(exe)], check=True)
    rng = random.Random(1)
    # token0, n, first, end, heads; far from the sequences on both sides, and across their ends
    cases = [(0, 8, MOST, MOST, 1 << 16), (0, 1, 1 << 15, MOST, 1 << 16),
             (0, 8, 40000, 50000, 60000), (40000, 8, 0, 1, 60000),
             (MOST - 8, 8, 0, 1, 1 << 16), (MOST - 1, 1, 0, MOST, 1 << 16),
             (8, 8, 3, 30, 40), (8, 8, 11, 13, 40), (8, 8, 16, 20, 40), (8, 8, 0, 8, 40)]
    for _ in range(20000):
        n = rng.randint(1, 8)
        a, b = sorted(int(2 ** rng.uniform(0, 26)) for _ in range(2))
        near = rng.choice((a, b, int(2 ** rng.uniform(0, 26))))
        cases.append((near // n * n, n, a, b, int(2 ** rng.uniform(0, 16))))
    out = subprocess.run([str(exe)], input="\n".join("%d %d %d %d %d" % c for c in cases),
                         capture_output=True, text=True, check=True, timeout=60).stdout
    got = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert len(got) == len(cases)
    for (token0, n, first, end, heads), (tokens, lo, hi) in zip(cases, got):
        want = [k for k in range(n) if first <= token0 + k < end]
        assert tokens == sum(token0 + k < end for k in range(n))
        assert list(range(lo, max(lo, hi), heads)) == [k * heads for k in want]
        assert not want or hi == (want[-1] + 1) * heads
