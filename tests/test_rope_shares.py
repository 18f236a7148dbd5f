"""How rows that turn by their positions are shared out over workgroups and launches (csrc/launch_rules.h), on the host: a launch counts its
threads in 32 bits, and a kernel's divisions are products below 2^22."""
import itertools
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2304_01089_amd", "csrc")
PROGRAM = r"""
#include <iostream>
#include "launch_rules.h"
int main() {
  long long T, heads, half, units;
  while (std::cin >> T >> heads >> half >> units) {
    const rptq::RopeShares s = rptq::rope_shares(T, static_cast<int>(heads), static_cast<int>(half), static_cast<int>(units));
    std::cout << s.rows << " " << s.heads << " " << s.head_groups << " " << s.launch_rows << "\n";
  }
}
"""


@pytest.fixture(scope="module")
def shares(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("shares")
    (at / "shares.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(at / "shares.cpp"), "-o", str(at / "shares")], check=True)

    def ask(queries):
        text = "".join("%d %d %d %d\n" % q for q in queries)
        out = subprocess.run([str(at / "shares")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [tuple(int(v) for v in line.split()) for line in out]
    return ask


def test_every_launch_can_be_made(shares):
    """Up to 2^40 rows, the most that a call may have; a launch of 2^26 rows at four a workgroup would have 2^32 threads."""
    rows = [1, 5, 1023, 1024, 4096, 8192, (1 << 26) - 1, 1 << 26, (1 << 26) + 5, 1 << 27, 1 << 31, (1 << 33) + 1, 1 << 40]
    heads = [(1, 1, 1), (1, 32, 4), (1, 512, 64), (32768, 1, 1), (129, 1, 508), (512, 64, 8), (65, 499, 501), (96, 512, 512)]   # (heads, pairs, pieces of a head)
    queries = [(T, n, half, units) for T, (n, half, units) in itertools.product(rows, heads)]
    for (T, n, half, units), (per, h, groups, most) in zip(queries, shares(queries)):
        assert per >= 1 and h >= 1 and (groups - 1) * h < n <= groups * h
        assert most >= per and most % per == 0
        part = min(T, most)
        assert -(-part // per) * groups * 256 < 1 << 32, (T, n)
        assert per * half <= 1024 and per * h * units < 1 << 22
    assert -(-(1 << 26) // shares([(1 << 26, 1, 32, 4)])[0][0]) * 256 == 1 << 32


def test_ordinary_calls_are_one_launch(shares):
    got = shares([(1, 24, 32, 4), (777, 25, 16, 10), (8192, 80, 64, 8), (4 << 20, 80, 64, 8)])
    assert [(r, h, g) for r, h, g, _ in got] == [(1, 24, 1), (1, 25, 1), (4, 80, 1), (4, 80, 1)]
    assert all(most >= T for (_, _, _, most), T in zip(got, (1, 777, 8192, 4 << 20)))
