"""What the library asks a device once is kept per kernel and device (csrc/per_device.h,
plain C++): an answer of one device does not stand for another's."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10392_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "per_device.h"

int main() {
  unif::PerDevice<unsigned> kept;
  int a = 0, b = 0, asked = 0;
  bool works = true;
  auto get = [&](const void* kernel, int device, unsigned answer) {
    unsigned v = 0;
    const bool ok = kept.get(kernel, device, &v, [&](unsigned* to) {
      ++asked;
      *to = answer;
      return works;
    });
    return ok ? (int)v : -1;
  };
  // each kernel on each device is asked once, and keeps its own answer
  if (get(&a, 0, 16) != 16 || get(&a, 0, 8) != 16 || asked != 1) return 1;
  if (get(&a, 1, 8) != 8 || get(&a, 1, 16) != 8 || get(&a, 0, 8) != 16 || asked != 2) return 2;
  if (get(&b, 1, 16) != 16 || get(&a, 1, 16) != 8 || asked != 3) return 3;
  // a failure is not kept
  works = false;
  if (get(&b, 0, 16) != -1 || asked != 4) return 4;
  works = true;
  if (get(&b, 0, 8) != 8 || get(&b, 0, 16) != 8 || asked != 5) return 5;
  return 0;
}
"""


def test_answers_are_kept_per_kernel_and_device(tmp_path):
    cxx = shutil.which(os.environ.get("CXX") or "g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "kept.cpp", tmp_path / "kept"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(src), "-o", str(exe), "-pthread"], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_balance_loss_keeps_no_answer_for_the_process():
    """Function-local statics of the launch code are all kept per device."""
    import re
    for name in sorted(os.listdir(CSRC)):
        if name in ("balance.cu", "block_norm.cu", "fp4_product.cu", "mxfp4.cu"):
            src = open(os.path.join(CSRC, name)).read()
            statics = re.findall(r"^\s+static (?!_assert|constexpr|const\b)(\S+)", src, re.M)
            assert all(s.startswith("PerDevice<") for s in statics), (name, statics)
