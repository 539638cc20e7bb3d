"""The example that runs the operators round the layer together: training steps lower
the loss, and the 4-bit experts give the layer's output to the accuracy of 4 bits."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [dict(), dict(d=768, d_ff=1536, n_experts=6, n_blocks=8, tokens=777)],
                         ids=["vit_s", "wider"])
def test_sublayer_example(sizes, monkeypatch):
    monkeypatch.syspath_prepend(os.path.join(ROOT, "examples"))
    import sublayer
    losses, off = sublayer.main(steps=4, **sizes)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
    # an element of a 4-bit block is off by up to 1/4 of itself (about 0.11 rms over the block,
    # less for the largest); two operands of each of two products: 0.11 * sqrt(4) = 0.22
    assert 0.01 < off < 0.25, off


@pytest.mark.gpu
def test_tokens_of_several_passes_in_4_bits(monkeypatch):
    """More tokens than the layer takes in one pass: the 4-bit sublayer gives all of them,
    to the accuracy of 4 bits (0.25 as above; tokens that are left out are off by 1)."""
    monkeypatch.syspath_prepend(os.path.join(ROOT, "examples"))
    import sublayer
    import torch
    T = 12000
    s = sublayer.Sublayer(d=4096, d_ff=512, n_experts=2, n_blocks=4, tokens=T)
    assert s.layer.pass_tokens() < T
    x = torch.randn(T, s.d, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    _, y, _, closed = s.forward(x)
    y4, closed4 = s.forward_fp4(x, s.quantize())
    P = s.layer.pass_tokens()
    for part in (slice(0, P), slice(P, T)):
        off = float((y4[part].float() - y[part].float()).norm() / y[part].float().norm())
        assert 0.01 < off < 0.25, (part, off)
    assert closed4["u"].shape == closed["u"].shape
