"""Rows of tensors of any number of dimensions (csrc/row_distance.h, plain C++; CPU), and the calls
that take such rows: rows that are one row in memory are refused, not taken for dense ones."""
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10392_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "row_distance.h"

// cols, then size and stride of each dimension in front
int main(int argc, char** argv) {
  int64_t sizes[8], strides[8], rows, distance;
  int n = 0;
  for (int i = 2; i + 1 < argc; i += 2, ++n) {
    sizes[n] = std::atoll(argv[i]);
    strides[n] = std::atoll(argv[i + 1]);
  }
  if (!unif::rows_at_one_distance(sizes, strides, n, std::atoll(argv[1]), &rows, &distance)) return 1;
  std::printf("%lld %lld", (long long)rows, (long long)distance);
  return 0;
}
"""


@pytest.fixture(scope="module")
def rows_of(tmp_path_factory):
    cxx = shutil.which(os.environ.get("CXX") or "g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("rows")
    (at / "rows.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, str(at / "rows.cpp"), "-o", str(at / "rows")], check=True)

    def run(t):
        args = [t.size(-1)] + [v for i in range(t.dim() - 1) for v in (t.size(i), t.stride(i))]
        r = subprocess.run([str(at / "rows")] + [str(v) for v in args], capture_output=True, text=True)
        return None if r.returncode else tuple(int(v) for v in r.stdout.split())
    return run


def test_rows_at_one_distance(rows_of):
    x = torch.empty(2, 3, 4, 50)
    assert rows_of(x) == (24, 50) and rows_of(x[0, 0, 0]) == (1, 50) and rows_of(x[:, :, :, :48]) == (24, 50)
    assert rows_of(x[:1, :, :1]) == (3, 200) and rows_of(x[:, :1, :1]) == (2, 600)
    assert rows_of(x[:, :, :3]) is None and rows_of(x[:, :2]) is None and rows_of(x.transpose(0, 1)) is None


def test_rows_that_are_one_row(rows_of):
    """Expanded tensors: one row in memory, or rows that repeat."""
    one, few = torch.empty(1, 64), torch.empty(1, 3, 64)
    assert rows_of(one.expand(1, 64)) == (1, 64)
    assert rows_of(one.expand(4, 64)) is None
    assert rows_of(one.expand(5, 4, 64)) is None
    assert rows_of(few.expand(2, 3, 64)) is None
    assert rows_of(few[:, :1].expand(1, 7, 64)) is None
    # an outer dimension at the distance that dense rows would have
    assert rows_of(torch.empty(900).as_strided((2, 4, 64), (256, 0, 1))) is None
    assert rows_of(torch.empty(900).as_strided((4, 64), (63, 1))) is None
    assert rows_of(torch.empty(900).as_strided((4, 64), (64, 1))) == (4, 64)


def test_no_rows(rows_of):
    for shape in ((0, 64), (3, 0, 64), (0, 3, 64), (2, 0, 3, 64), (2, 3, 0, 64)):
        assert rows_of(torch.empty(shape)) == (0, 64)
    assert rows_of(torch.empty(3, 0, 80)[..., :64]) == (0, 64)


@pytest.mark.gpu
def test_expanded_codes_are_refused():
    import paper_2608_10392_gb300 as pkg
    x = torch.ones(4, 64, device="cuda")
    q = pkg.fp8_quantize(x)
    scales = torch.ones(2, 2, 4, device="cuda")
    buffer = torch.zeros(64, 64, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
    one = buffer[:1]
    for codes, s in ((one.expand(4, 64), scales[0, 0]), (one.expand(2, 4, 64), scales[0]),
                     (buffer[:4].expand(2, 2, 4, 64), scales), (buffer.as_strided((2, 4, 64), (256, 0, 1)), scales[0])):
        with pytest.raises(ValueError, match="q.codes: need rows at one distance"):
            pkg.fp8_dequantize(pkg.Fp8(codes, s))
        with pytest.raises(ValueError, match="out.codes: need rows at one distance"):
            pkg.fp8_quantize(x.expand(codes.shape).contiguous(), out=pkg.Fp8(codes, s))
    with pytest.raises(Exception):  # the other calls on rows in 8 bits
        pkg.linear(pkg.Fp8(one.expand(4, 64), scales[0, 0]), q)
    w = torch.ones(64, device="cuda").bfloat16()
    with pytest.raises(Exception):
        pkg.BlockNorm(64, stream_dtype="f32", u_format="fp8").forward(
            x, u=pkg.Fp8(one.expand(4, 64), scales[0, 0]), pre_weight=w)
    assert (buffer.view(torch.uint8) == 0).all()
    # one row stays what it was: dense, wherever it lies
    assert torch.equal(pkg.fp8_dequantize(pkg.Fp8(q.codes[:1].expand(1, 64), q.scales[:1])), x[:1].bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(0, 50), (3, 0, 50), (0, 3, 50), (2, 3, 0, 64), (2, 0, 3, 64)])
def test_no_rows_of_any_dimensions(shape):
    from paper_2608_10392_gb300 import fp8_dequantize, fp8_quantize
    for dtype in (torch.float32, torch.bfloat16):
        q = fp8_quantize(torch.empty(shape, device="cuda", dtype=dtype))
        assert q.codes.shape == shape and q.scales.shape == shape[:-1]
        assert fp8_dequantize(q, dtype="f32").shape == shape
        assert fp8_quantize(torch.empty(shape, device="cuda", dtype=dtype), out=q) is q
