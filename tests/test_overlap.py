"""Which arrays of a call share memory (csrc/overlap.h, plain C++; CPU), against byte for byte."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10392_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "overlap.h"

int main() {
  long long v[8];
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld", v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6, v + 7) == 8) {
    const unif::Block a{reinterpret_cast<const void*>(v[0]), v[1], v[2], v[3]},
        b{reinterpret_cast<const void*>(v[4]), v[5], v[6], v[7]};
    std::printf("%d%d\n", (int)unif::overlap(a, b), (int)unif::overlap(b, a));
  }
  return 0;
}
"""


def bytes_of(p, pitch, width, rows):
    return {p + r * pitch + i for r in range(rows) for i in range(width)} if p else set()


def test_against_every_byte(tmp_path):
    cxx = shutil.which(os.environ.get("CXX") or "g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    rng = random.Random(5)
    cases = []
    for _ in range(6000):
        pitch = rng.randint(1, 24)
        blocks = []
        for _ in range(2):
            own = pitch if rng.random() < 0.8 else rng.randint(1, 24)
            blocks.append((rng.randint(100, 260), own, rng.randint(1, own), rng.choice([0, 1, 1, 2, 5, 9])))
        cases.append(blocks)
    cases += [[(0, 8, 8, 4), (0, 8, 8, 4)], [(100, 8, 8, 4), (0, 8, 8, 4)], [(100, 8, 8, 1), (104, 100, 8, 1)],
              [(100, 40, 8, 1), (110, 20, 8, 5)], [(100, 16, 8, 6), (108, 16, 8, 6)], [(100, 16, 8, 6), (124, 16, 8, 6)],
              [(100, 16, 8, 6), (117, 999, 7, 1)], [(100, 16, 8, 6), (124, 999, 8, 1)], [(100, 16, 8, 6), (124, 999, 9, 1)]]
    src, exe = tmp_path / "o.cpp", tmp_path / "o"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], input="\n".join(" ".join(str(v) for b in c for v in b) for c in cases),
                       capture_output=True, text=True, check=True).stdout.split()
    assert len(r) == len(cases)
    exact = 0
    for (a, b), got in zip(cases, r):
        shares = bool(bytes_of(*a) & bytes_of(*b))
        assert got in ("00", "11"), (a, b)
        if a[1] == b[1] or a[3] <= 1 or b[3] <= 1:
            # (of the last row of one array, what is behind it counts as the next row's place)
            assert got == "11" or not shares, (a, b)
            exact += (got == "11") == shares
        else:
            assert not shares or got == "11", (a, b)
    assert exact > 0.95 * sum(a[1] == b[1] or a[3] <= 1 or b[3] <= 1 for a, b in cases)


def test_columns_of_one_array(tmp_path):
    """Side by side, in any order: they do not share memory, one row or many."""
    cxx = shutil.which(os.environ.get("CXX") or "g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "o.cpp", tmp_path / "o"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    cases = [((1000 + a, 64, w, ra), (1000 + b, 64, v, rb)) for a, w in ((0, 16), (16, 16), (40, 24))
             for b, v in ((0, 16), (16, 16), (40, 24)) if a != b for ra in (1, 2, 7) for rb in (1, 2, 7)]
    r = subprocess.run([str(exe)], input="\n".join(" ".join(str(v) for b in c for v in b) for c in cases),
                       capture_output=True, text=True, check=True).stdout.split()
    assert r == ["00"] * len(cases)
