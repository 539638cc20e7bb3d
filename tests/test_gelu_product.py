"""GELU in the 4-bit product's bf16 results (csrc/fp4_product.cu: gelu2) against v Phi(v)
in 64 bits, in relative terms: also where v is negative and GELU small.

CPU: the constants compiled into the kernel, in its arithmetic with an exact 2^, are
within 2^-18 of the value for v >= -4 and within 2^-12 down to v = -12.9, where Phi leaves
fp32's normal range (Phi is then taken as 0, the value below 2e-37).
GPU: products whose results are known exactly before GELU (sums of four 4-bit values of
different scales). The result is a value within 2^-11 of GELU (the function's bound and
the hardware's 2^, 2^-22), rounded to bf16 once: rounding keeps order, so it lies between
the roundings of the two ends of that range."""
import os
import re

import numpy as np
import pytest
from scipy.special import log_ndtr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "paper_2608_10392_gb300", "csrc", "fp4_product.cu")


def exact(v):
    v = np.asarray(v, dtype=np.float64)
    return v * np.exp(log_ndtr(v))


def test_constants_of_the_kernel():
    from gelu_log_fit import DEG, gelu_log
    src = open(SOURCE).read()
    body = src[src.index("uint32_t gelu2("):]
    found = {int(k): np.uint32(int(b, 16)).view(np.float32)
             for b, k in re.findall(r"UNIF_K2\((0x[0-9a-f]{8})\)\)?;\s*// q(\d+)", body)}
    assert sorted(found) == list(range(DEG + 1)), found
    c = [found[k] for k in range(DEG + 1)]
    for lo, hi, bound in ((-12.9, -4, 2.0 ** -12), (-4, 0, 2.0 ** -18), (0, 13, 2.0 ** -18)):
        v = np.linspace(lo, hi, 800001).astype(np.float32)
        v = v[v != 0]
        assert np.abs(gelu_log(v, c) / exact(v) - 1).max() < bound
    v = np.array([-1e30, -40, -14, -13, 0, 14, 40, 1e30, np.inf], dtype=np.float32)
    got = gelu_log(v, c)
    assert np.abs(got[:-1] - np.maximum(v, 0)[:-1]).max() < 2e-37 and got[-1] == np.inf
    assert np.isnan(gelu_log(np.array([np.nan], dtype=np.float32), c)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,cols,sizes,odd", [
    (128, 512, [300, 7, 93], False),    # channels as M, two channels a store
    (131, 512, [300, 7, 93], False),    # one channel a store
    (192, 512, [300, 0, 150], False),   # rows as M
    (192, 512, [300, 0, 150], True),    # rows of the output off 32 bytes
    (256, 2048, [200, 130], False)])    # pairs of CTAs
def test_small_values_of_gelu(n, cols, sizes, odd):
    import torch

    from paper_2608_10392_gb300 import Mxfp4, mxfp4_product, mxfp4_status
    g = torch.Generator().manual_seed(n + cols)
    rows, G, parts = sum(sizes), len(sizes), 4
    span = cols // parts  # channel j adds columns j % span + k span of a row
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6],
                         dtype=torch.float64)
    c = torch.randint(0, 16, (rows, cols), generator=g, dtype=torch.uint8)
    power = torch.tensor([1, -2, -5, -8]).repeat_interleave(span)  # of the parts' scales
    av = table[c.long()] * torch.exp2(power.double())
    a = Mxfp4((c[:, 0::2] | c[:, 1::2] << 4).cuda(),
              (power[::32] + 127).to(torch.uint8).repeat(rows, 1).cuda(), cols)
    w = torch.zeros(G, n, cols, dtype=torch.uint8)
    for j in range(n):
        w[:, j, j % span::span] = 2  # 1.0
    wq = Mxfp4((w[..., 0::2] | w[..., 1::2] << 4).cuda(),
               torch.full((G, n, cols // 32), 127, dtype=torch.uint8, device="cuda"), cols)
    v = av.view(rows, parts, span).sum(1)[:, torch.arange(n) % span].numpy()
    off = torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device="cuda")
    wide = torch.empty(rows, n + 3, dtype=torch.bfloat16, device="cuda")
    plain = mxfp4_product(a, wq, off, dtype="f32")
    assert np.array_equal(plain.double().cpu().numpy(), v)  # exact, so far
    got = mxfp4_product(a, wq, off, activation="gelu", out=wide[:, 3:] if odd else None)
    assert mxfp4_status() == 0
    got, want = got.double().cpu().numpy(), exact(v)
    near = v >= -12.9
    assert (v < -4).sum() > 1000
    ends = [torch.from_numpy(want * (1 + s * 2.0 ** -11)).bfloat16().double().numpy() for s in (-1, 1)]
    ok = (np.minimum(*ends) <= got) & (got <= np.maximum(*ends))
    assert ok[near].all(), (int((~ok[near]).sum()), v[near][~ok[near]][:5])
    assert (np.abs(got - want)[~near] < 2e-37).all()


@pytest.mark.gpu
def test_nan_through_gelu():
    """A NaN scale makes its row's results NaN, and no others."""
    import torch

    from paper_2608_10392_gb300 import Mxfp4, mxfp4_product
    for n in (128, 192):  # channels as M, rows as M
        c = torch.full((200, 16), 0x22, dtype=torch.uint8, device="cuda")  # all 1.0
        s = torch.zeros(200, 8, dtype=torch.uint8, device="cuda")
        s[:, 0] = 127
        w = Mxfp4(c[:1].repeat(n, 1), s[:1].repeat(n, 1), 32)
        s[3, 0] = 255
        got = mxfp4_product(Mxfp4(c, s, 32), w, activation="gelu")
        rest = [r for r in range(200) if r != 3]
        assert torch.isnan(got[3]).all() and (got[rest] == 32).all()
