"""Rows to microscaled 4-bit floating point and back: codes, scale bytes and values
equal those of the definition in 64 bits, bit for bit (scaling by a power of two is
exact, so nothing is left to a tolerance); refusals."""
import ctypes as C
import math

import pytest
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def reference(x):
    """(codes [rows][cols] as numbers 0..15, scale bytes [rows][blocks]) by the
    definition, in 64 bits: nearest level, ties to the level of even code."""
    x = x.double().cpu()
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    codes = torch.zeros(rows, cols, dtype=torch.uint8)
    scales = torch.zeros(rows, blocks, dtype=torch.uint8)
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    for b in range(blocks):
        v = x[:, 32 * b:32 * b + 32]
        bad = ~torch.isfinite(v).all(1)
        most = torch.where(bad, 1.0, v.abs().amax(1))
        e = torch.frexp(most)[1].double() - 1  # floor(log2)
        e = torch.where(most == 0, -127.0, (e - 2).clamp(min=-127))
        scales[:, b] = torch.where(bad, 255.0, e + 127).to(torch.uint8)
        m = v.abs() / torch.exp2(e)[:, None]
        d = (m[:, :, None] - levels).abs()
        near = d.amin(2, keepdim=True)
        even = torch.tensor([0.0, 0.25] * 4, dtype=torch.float64)  # prefers even codes among the nearest
        code = torch.where(d == near, even, 9.0).argmin(2)
        code = torch.where(torch.signbit(v), code + 8, code)
        codes[:, 32 * b:32 * b + 32] = torch.where(bad[:, None], 0, code).to(torch.uint8)
    return codes, scales


def check(x, **kw):
    from paper_2608_10392_gb300 import mxfp4_dequantize, mxfp4_quantize
    rows, cols = x.shape
    q = mxfp4_quantize(x, **kw)
    codes, scales = reference(x)
    full = torch.zeros(rows, (cols + 31) // 32 * 32, dtype=torch.uint8)
    full[:, :cols] = codes
    assert torch.equal(q.codes.cpu(), full[:, 0::2] | full[:, 1::2] << 4)
    pitch = torch.zeros(rows, (cols + 255) // 256 * 8, dtype=torch.uint8)
    pitch[:, :scales.shape[1]] = scales
    assert torch.equal(q.scales.cpu(), pitch)
    table = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)
    size = torch.exp2(scales.double() - 127)
    size[scales == 255] = math.nan
    want = table[codes.long()] * size.repeat_interleave(32, 1)[:, :cols]
    for name, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        got = mxfp4_dequantize(q, dtype=name)
        assert got.dtype == dt
        assert torch.equal(torch.nan_to_num(got.cpu(), nan=77.0),
                           torch.nan_to_num(want.to(dt), nan=77.0))
    return q


def data(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    return x.to(dtype).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (17, 64), (2, 256),
                                       (9, 257), (33, 384), (7, 1000), (130, 1024), (4, 8192),
                                       (1, 100000), (2500, 96)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_codes_scales_and_values(rows, cols, dtype):
    check(data(rows, cols, dtype, rows + cols))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_every_tie_and_neighbour(dtype):
    """Blocks whose largest value is 4, 6 and just below 8, with every level, every
    middle of two levels and their neighbours, at scales from the least to the largest."""
    rows = []
    step = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -20
    points = sorted({v * s for a, b in zip(LEVELS, LEVELS[1:]) for v in (a, (a + b) / 2)
                     for s in (1 - step, 1.0, 1 + step)})
    for e in (-126, -100, -3, 0, 5, 60, 125):
        for most in (4.0, 5.0, 6.0, 7.0, 7.96875):
            for at in range(0, len(points), 31):
                p = points[at:at + 31]
                row = [most] + [v if i % 2 else -v for i, v in enumerate(p) if v <= most]
                rows.append([v * 2.0 ** e for v in row] + [0.0] * (32 - len(row)))
    check(torch.tensor(rows, dtype=torch.float64).to(dtype).cuda())


@pytest.mark.gpu
def test_zeros_small_values_infinities_and_nan():
    x = data(12, 96, torch.float32)
    x[0] = 0.0
    x[1] = -0.0
    x[2] = 1e-45                      # the least subnormal
    x[3, :32] = torch.finfo(torch.float32).tiny
    x[4] = torch.finfo(torch.float32).max
    x[5, 40] = float("nan")
    x[6, 3] = float("inf")
    x[7, 95] = float("-inf")
    x[8] *= 2.0 ** -140
    check(x)


@pytest.mark.gpu
@pytest.mark.parametrize("cols,pad,shift", [(256, 8, 0), (256, 3, 0), (64, 16, 1), (50, 7, 2)])
def test_strided_rows(cols, pad, shift):
    from paper_2608_10392_gb300 import mxfp4_dequantize
    x = data(40, cols, torch.bfloat16, 3)
    wide = torch.full((40, cols + pad + shift), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, shift:shift + cols] = x
    q = check(wide[:, shift:shift + cols])
    back = torch.full_like(wide, 5.0)
    mxfp4_dequantize(q, out=back[:, shift:shift + cols])
    assert torch.equal(back[:, shift:shift + cols], mxfp4_dequantize(q))
    assert (back[:, :shift] == 5).all() and (back[:, shift + cols:] == 5).all()


@pytest.mark.gpu
def test_leading_dimensions_out_and_no_rows():
    from paper_2608_10392_gb300 import Mxfp4, mxfp4_dequantize, mxfp4_quantize
    x = data(6, 320, torch.float32).view(2, 3, 320)
    q = mxfp4_quantize(x)
    assert q.codes.shape == (2, 3, 160) and q.scales.shape == (2, 3, 16)
    r = mxfp4_quantize(x, out=Mxfp4(torch.zeros_like(q.codes), torch.zeros_like(q.scales), 320))
    assert torch.equal(r.codes, q.codes) and torch.equal(r.scales, q.scales)
    assert mxfp4_dequantize(q).shape == (2, 3, 320)
    e = mxfp4_quantize(x[0, :0])
    assert e.codes.shape == (0, 160) and mxfp4_dequantize(e).shape == (0, 320)


@pytest.mark.gpu
def test_more_than_2_to_the_31_elements():
    """Offsets of the elements pass 32 bits (bf16 rows of 4.3 GB)."""
    from paper_2608_10392_gb300 import mxfp4_dequantize, mxfp4_quantize
    rows, cols = (1 << 31) // 4096 + 5, 4096
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-3:] = data(3, cols, torch.bfloat16)
    q = mxfp4_quantize(x)
    tail = check(x[-3:].clone())
    assert torch.equal(q.codes[-3:], tail.codes) and torch.equal(q.scales[-3:], tail.scales)
    assert not q.codes[:-3].any()
    back = mxfp4_dequantize(q)
    assert torch.equal(back[-3:], mxfp4_dequantize(tail)) and not back[:-3].any()


def test_refusals():
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    L = pkg.lib()
    p = C.c_void_p(4096)
    for f in (lambda x=p, dt=0, rows=4, cols=64, ld=64, c=p, s=p:
              L.unif_moe_mxfp4_quantize(x, dt, rows, cols, ld, c, s, None),
              lambda x=p, dt=0, rows=4, cols=64, ld=64, c=p, s=p:
              L.unif_moe_mxfp4_dequantize(c, s, rows, cols, x, dt, ld, None)):
        for k in (dict(x=None), dict(dt=2), dict(rows=-1), dict(cols=0), dict(cols=(1 << 24) + 1),
                  dict(ld=63), dict(c=None), dict(s=None), dict(c=C.c_void_p(4104)),
                  dict(s=C.c_void_p(4100))):
            assert f(**k) == -1, k
        assert f(rows=0, x=None) == 0
    with pytest.raises(ValueError, match="x"):
        pkg.mxfp4_quantize(torch.zeros(4, 64))  # not on the GPU
    with pytest.raises(ValueError, match="codes"):
        pkg.mxfp4_dequantize(pkg.Mxfp4(torch.zeros(4, 33, dtype=torch.uint8),
                                       torch.zeros(4, 8, dtype=torch.uint8), 64))
