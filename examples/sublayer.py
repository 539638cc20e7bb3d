"""One pre-norm Transformer sublayer round a UniF-MoE layer, trained for a few steps
and then served with its experts in 4 bits: the layer's own calls with the operators
round it (BlockNorm, balance_loss, mxfp4_quantize, mxfp4_product).

    python examples/sublayer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_10392_gb300 import (FEATURE_BACKWARD, FEATURES_DEFAULT, BlockNorm, Layer, Mxfp4,  # noqa: E402
                                    balance_loss, mxfp4_product, mxfp4_quantize, mxfp4_status)


class Sublayer:
    """out = x + scale * F(N(x)), F the layer; the next block's N'(out) comes with it.
    x is fp32, the branch bf16."""

    def __init__(self, d=384, d_ff=1536, n_experts=8, n_blocks=8, tokens=2048, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s, std: torch.randn(*s, generator=g, device="cuda") * std  # noqa: E731
        K = n_experts
        self.d, self.H, self.K, self.B = d, d_ff, K, n_blocks
        self.layer = Layer(d, d_ff, K, n_blocks, max_tokens=tokens,
                           features=FEATURES_DEFAULT | FEATURE_BACKWARD)
        base_up, base_down = r(d_ff, d, std=d ** -0.5), r(d, d_ff, std=d_ff ** -0.5)
        self.w = dict(router=r(d, K + 1, std=0.02),
                      up=base_up + r(K + 1, d_ff, d, std=0.05 * d ** -0.5),
                      down=base_down + r(K + 1, d, d_ff, std=0.05 * d_ff ** -0.5),
                      scale=torch.full((1, d), 0.5, device="cuda"),
                      norm=torch.ones(d, device="cuda"), next_norm=torch.ones(d, device="cuda"))
        self.opening = BlockNorm(d, stream_dtype="f32", pre_norm="rms")
        self.closing = BlockNorm(d, stream_dtype="f32", pre_norm="rms")
        self.load()

    def load(self):
        self.bf16 = {k: v.bfloat16() for k, v in self.w.items()}
        b = self.bf16
        self.layer.load_weights(b["router"], b["up"], b["down"])

    def forward(self, x, stats=False):
        b = self.bf16
        opened = self.opening.forward(x, pre_weight=b["norm"], stats=stats)
        counts = torch.empty(x.shape[0], dtype=torch.int32, device="cuda")
        y = self.layer.forward(opened["u"], residual_counts=counts)
        closed = self.closing.forward(x, y, gate=b["scale"], pre_weight=b["next_norm"], stats=stats)
        return opened, y, counts, closed

    def step(self, x, target, rate=0.02, balance_weight=0.01, z_weight=1e-4):
        """One step of gradient descent on 0.5 |u' - target|^2 / T with the router's
        losses; returns (loss, router's losses, tokens per expert)."""
        T, b = x.shape[0], self.bf16
        opened, y, counts, closed = self.forward(x, stats=True)
        u = opened["u"]
        off = closed["u"].float() - target
        loss = 0.5 * off.square().sum() / T
        # the router's losses from the decisions that the forward took
        wr = b["router"][:, 1:].float()
        routed = balance_loss(u.float() @ wr, self.layer.routing()["q"], counts,
                              balance_weight=balance_weight, z_weight=z_weight)
        grads = self.closing.backward(closed["out"], y, closed, du=(off / T).bfloat16(),
                                      gate=b["scale"], pre_weight=b["next_norm"])
        moe = self.layer.backward(u, grads["dy"])
        d_router = moe["dw_router"]
        d_router[:, 1:] += u.float().T @ routed["dlogits"]
        du = (moe["dx"] + routed["dlogits"] @ wr.T).bfloat16()
        first = self.opening.backward(x, None, opened, dout=grads["dx"], du=du,
                                      pre_weight=b["norm"])
        for name, grad in (("router", d_router), ("up", moe["dw_up"]), ("down", moe["dw_down"]),
                           ("scale", grads["d_gate"]), ("next_norm", grads["d_pre_weight"]),
                           ("norm", first["d_pre_weight"])):
            self.w[name] -= rate * grad
        self.load()
        return float(loss), routed["loss"], routed["counts"]

    def quantize(self):
        """The experts in 4 bits, one group of the layer's table for each (expert, block):
        up [G][M][d], down [G][d][M]."""
        E, B, M = self.K + 1, self.B, self.H // self.B
        up = self.bf16["up"].view(E * B, M, self.d)
        down = self.bf16["down"].view(E, self.d, B, M).transpose(1, 2).reshape(E * B, self.d, M)
        return mxfp4_quantize(up), mxfp4_quantize(down)

    def forward_fp4(self, x, experts):
        """The sublayer with 4-bit experts and activations, over the group table of the
        layer's routing. That table is in the handle after a bf16 forward of the same tokens
        and holds those of its last pass, so tokens are taken a pass at a time."""
        up, down = experts
        T, P = x.shape[0], self.layer.pass_tokens()
        y = torch.zeros(T, self.d, device="cuda")
        for lo in range(0, T, P):
            opened, _, _, _ = self.forward(x[lo:lo + P])
            _, offsets, token, weight = self.layer.groups()
            token, weight, offsets = token.long().cuda(), weight.cuda(), offsets.cuda()
            rows = opened["u"][token.clamp(min=0)]  # padding rows have weight 0
            h = mxfp4_product(mxfp4_quantize(rows), up, offsets, activation="gelu")
            part = mxfp4_product(mxfp4_quantize(h), down, offsets, dtype="f32")
            weight = torch.where(token < 0, 0.0, weight)
            y[lo:lo + P].index_add_(0, token.clamp(min=0), part * weight[:, None])
        y = y.bfloat16()
        return y, self.closing.forward(x, y, gate=self.bf16["scale"],
                                       pre_weight=self.bf16["next_norm"])


def main(tokens=2048, steps=5, **sizes):
    s = Sublayer(tokens=tokens, **sizes)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(tokens, s.d, generator=g, device="cuda")
    target = torch.randn(tokens, s.d, generator=g, device="cuda")
    losses = []
    for k in range(steps):
        loss, router, counts = s.step(x, target)
        losses.append(loss)
        print("step %d: loss %.4f, balance %.4f, z %.4f, tokens per expert %s"
              % (k, loss, float(router[1]), float(router[2]), counts.tolist()))
    _, y, _, closed = s.forward(x)
    experts = s.quantize()
    y4, closed4 = s.forward_fp4(x, experts)
    off = float((y4.float() - y.float()).norm() / y.float().norm())
    held = sum(t.numel() for e in experts for t in (e.codes, e.scales))
    print("4-bit experts: %.1f MB (bf16 %.1f), layer output off by %.3f of its norm, stream by %.4f"
          % (held / 1e6, 2 * (s.w["up"].numel() + s.w["down"].numel()) / 1e6, off,
             float((closed4["out"] - closed["out"]).norm() / closed["out"].norm())))
    if mxfp4_status() != 0:
        raise RuntimeError("a product gave up a wait")
    return losses, off


if __name__ == "__main__":
    main()
