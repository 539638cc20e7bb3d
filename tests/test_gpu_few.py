"""The layer for a few tokens (few_tokens, Layer.forward_few) against 64 bits: one token to 64,
layers of every kind of size, thresholds, masks, strides; decisions against the oracle's; the
handle's records left alone; refusals.

Tolerances. A pre-activation is a sum over d features, products exact, cut at every 16 (as
tests/test_gpu_linear.py derives): a = (d / 16 + 2) 2^-22 of its terms' sizes. h = w GELU: slope
1.13, GELU's own 2^-11, w within 2^-19 (an exponential of logits within 2e-6, a sum and a quotient),
rounded to bf16 by 2^-8. y sums h v over up to 8,256 channels a chain of 16 at a time in each of
a warp's 64, warps and CTAs in fp32: 40 steps of 2^-22 and the chain's c / 16 / 16 steps; rounded by 2^-8."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

F64 = torch.float64


def layer(d, H, K, B, seed, bias=False):
    g = torch.Generator().manual_seed(seed)
    up, down = torch.randn(H, d, generator=g) * d ** -0.5, torch.randn(d, H, generator=g) * H ** -0.5
    w = dict(up=(up + torch.randn(K + 1, H, d, generator=g) * 0.05 * d ** -0.5).bfloat16(),
             down=(down + torch.randn(K + 1, d, H, generator=g) * 0.05 * H ** -0.5).bfloat16(),
             router=(torch.randn(d, K + 1, generator=g) * 0.05).bfloat16(),
             bias=torch.randn(K + 1, generator=g) * 0.3 if bias else None)
    return w, g


def reference(w, x, r, B, mask):
    """(y, tolerance) in 64 bits with the decisions r."""
    up, down, x = w["up"].to(F64).cuda(), w["down"].to(F64).cuda(), x.to(F64).cuda()
    E, H, d = up.shape
    if mask is not None:
        x = torch.where(mask.cuda()[:, None] != 0, x, 0.0)
    shr = torch.from_numpy(((r.shr_mask[:, None] >> np.arange(B, dtype=np.uint64)) & np.uint64(1)).astype(np.float64)).cuda()
    em = torch.from_numpy(((r.expert_mask()[:, None] >> np.arange(E - 1, dtype=np.uint64)) & np.uint64(1)).astype(np.float64)).cuda()
    wt = torch.cat([(torch.from_numpy(r.alpha).cuda()[:, None] * shr)[:, None],
                    (torch.from_numpy(r.s).cuda() * em)[:, :, None] * (1 - shr[:, None])], 1)
    if mask is not None:
        wt = torch.where((mask.cuda() != 0)[:, None, None], wt, 0.0)
    y = torch.zeros(len(x), d, dtype=F64, device="cuda")
    tol = torch.zeros_like(y)
    chain = E * H / 64 / 16
    for e in range(E):
        z, size = x @ up[e].T, x.abs() @ up[e].abs().T
        we = wt[:, e].repeat_interleave(H // B, 1)
        h = we * z * torch.special.ndtr(z)
        off = we * 1.13 * (d / 16 + 2) * 2.0 ** -22 * size + h.abs() * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18)
        y += h @ down[e].T
        tol += off @ down[e].abs().T + (40 + chain) * 2.0 ** -22 * (h.abs() @ down[e].abs().T)
    return y, tol + 2.0 ** -8 * y.abs()


def check(d, H, K, B, T, seed=0, masked=False, bias=False, through="both", **th):
    import oracle
    from paper_2608_10392_gb300 import Layer, few_tokens, router_table
    oracle.build()
    w, g = layer(d, H, K, B, seed, bias)
    x = torch.randn(T, d, generator=g).bfloat16()
    mask = None
    if masked:
        mask = (torch.rand(T, generator=g) < 0.6).to(torch.uint8)
        x[mask == 0] = float("nan")
    mu = oracle.prototypes(w["up"][0], B, oracle.ROUND_BF16)
    r = oracle.route(x, w["router"], mu, K, B, oracle.Thresholds(**th), mask, w["bias"])
    want, tol = reference(w, x, r, B, mask)
    on = {k: None if v is None else v.cuda() for k, v in w.items()}
    xd, md = x.cuda(), None if mask is None else mask.cuda()
    table = router_table(on["router"], on["up"], B)
    assert torch.equal(table[:K + 1], on["router"].T)
    keys = on["up"][0].to(F64).view(B, H // B, d).mean(1)
    assert ((table[K + 1:].to(F64) - keys).abs() <= 2.0 ** -8 * keys.abs()).all()
    handle = Layer(d, H, K, B, max_tokens=max(T, 1), **th)
    handle.load_weights(on["router"], on["up"], on["down"], on["bias"])
    got = []
    for form in ("weights", "handle"):
        b, k = (torch.full((T,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        if form == "weights":
            y = few_tokens(xd, table, on["up"], on["down"], B, router_bias=on["bias"], mask=md, shared_counts=b,
                           residual_counts=k, **th)
        else:
            y = handle.forward_few(xd, mask=md, shared_counts=b, residual_counts=k)
        b, k = b.cpu().numpy(), k.cpu().numpy()
        # a decision closer to its border than the logits' fp32 error may fall either way
        clear = (np.nan_to_num(r.margin, nan=1.0).min(1) > 1e-5) if mask is None else (
            (np.nan_to_num(r.margin, nan=1.0).min(1) > 1e-5) | (mask.numpy() == 0))
        assert (b == np.where(mask.numpy() != 0, r.b, 0) if mask is not None else b == r.b)[clear].all()
        assert (k == np.where(mask.numpy() != 0, r.k, 0) if mask is not None else k == r.k)[clear].all()
        ok = torch.from_numpy(clear).cuda()
        err = (y.to(F64) - want).abs()
        assert y.dtype == torch.bfloat16 and (err <= tol)[ok].all(), float((err / tol.clamp(min=1e-30))[ok].max())
        if mask is not None:
            assert (y[md == 0] == 0).all()
        got.append(y)
    assert torch.equal(*got)  # (the same table, the same kernels)
    handle.close()
    return got[0]


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64])
@pytest.mark.parametrize("d,H,K,B", [(64, 128, 1, 2), (384, 1536, 8, 8), (320, 640, 5, 5)])
def test_against_64_bits(d, H, K, B, T):
    check(d, H, K, B, T, seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("d,H,K,B,T", [(768, 1024, 16, 16, 5), (1024, 4096, 32, 16, 1), (1024, 4096, 32, 16, 24),
                                       (128, 4096, 64, 64, 3), (128, 4096, 64, 64, 40), (1984, 256, 3, 4, 12),
                                       (64, 4096, 40, 2, 64), (448, 2304, 12, 12, 20)])
def test_other_layers(d, H, K, B, T):
    check(d, H, K, B, T, seed=d)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 20, 50])
@pytest.mark.parametrize("th", [dict(topk_fixed=2), dict(beta_fixed=0.7), dict(prefix_blocks=1), dict(alpha_fixed=0.0),
                                dict(alpha_fixed=1.0), dict(tau=0.2), dict(alpha_fixed=0.4, topk_fixed=1),
                                dict(topk_fixed=6), dict(beta_fixed=0.0), dict(beta_fixed=2.0)])
def test_thresholds_masks_and_bias(T, th):
    check(256, 768, 6, 6, T, seed=T, masked=True, bias=True, **th)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 8, 9, 40])
def test_weights_that_are_not_finite(T):
    """An expert's infinities and NaN reach the tokens that take it and no others."""
    from paper_2608_10392_gb300 import few_tokens, router_table
    d, H, K, B = 64, 256, 4, 4
    w, g = layer(d, H, K, B, 3)
    x = torch.randn(T, d, generator=g).bfloat16().cuda()
    on = {k: v.cuda() for k, v in w.items() if v is not None}
    table = router_table(on["router"], on["up"], B)
    k = dict(alpha_fixed=0.5, topk_fixed=1, prefix_blocks=True)
    want = few_tokens(x, table, on["up"], on["down"], B, **k)
    first = (x.to(F64) @ on["router"].to(F64))[:, 1:].argmax(1)
    e = int(first[0])
    takes = first == e
    if bool(takes.all()):
        x[1] = -x[0]
        want = few_tokens(x, table, on["up"], on["down"], B, **k)
        takes = (x.to(F64) @ on["router"].to(F64))[:, 1:].argmax(1) == e
    for name, value in (("up", math.nan), ("down", math.inf), ("down", math.nan)):
        bad = {n: on[n].clone() for n in ("up", "down")}
        bad[name][1 + e] = value
        y = few_tokens(x, table, bad["up"], bad["down"], B, **k)
        assert not takes.all() and torch.equal(y[~takes], want[~takes])
        assert not y[takes].isfinite().any()


@pytest.mark.gpu
def test_no_tokens_and_all_padding():
    from paper_2608_10392_gb300 import few_tokens, router_table
    w, g = layer(64, 256, 3, 4, 1)
    on = {k: None if v is None else v.cuda() for k, v in w.items()}
    table = router_table(on["router"], on["up"], 4)
    assert few_tokens(torch.empty(0, 64, device="cuda").bfloat16(), table, on["up"], on["down"], 4).shape == (0, 64)
    for T in (5, 40):
        x = torch.full((T, 64), float("nan"), device="cuda").bfloat16()
        y = few_tokens(x, table, on["up"], on["down"], 4, mask=torch.zeros(T, dtype=torch.bool, device="cuda"))
        assert (y == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 30])
def test_strides_place_and_repetition(T):
    from paper_2608_10392_gb300 import few_tokens, router_table
    w, g = layer(256, 512, 4, 4, 2)
    on = {k: None if v is None else v.cuda() for k, v in w.items()}
    table = router_table(on["router"], on["up"], 4)
    wide = torch.randn(T, 280, generator=g).bfloat16().cuda()
    x = wide[:, 8:264]
    want = few_tokens(x.contiguous(), table, on["up"], on["down"], 4)
    out = torch.full((T, 259), 3.0, device="cuda").bfloat16()
    few_tokens(x, table, on["up"], on["down"], 4, out=out[:, 1:257])
    assert torch.equal(out[:, 1:257], want) and (out[:, 0] == 3).all() and (out[:, 257:] == 3).all()
    y = x.contiguous()
    assert few_tokens(y, table, on["up"], on["down"], 4, out=y).data_ptr() == y.data_ptr() and torch.equal(y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 30])
def test_streams_graphs_and_two_calls_at_once(T):
    from paper_2608_10392_gb300 import few_tokens, router_table
    w, g = layer(256, 1024, 8, 8, 2)
    on = {k: None if v is None else v.cuda() for k, v in w.items()}
    table = router_table(on["router"], on["up"], 8)
    xs = [torch.randn(T, 256, generator=g).bfloat16().cuda() for _ in range(2)]
    run = lambda x, **s: few_tokens(x, table, on["up"], on["down"], 8, **s)  # noqa: E731
    want = [run(x) for x in xs]
    sides = [torch.cuda.Stream() for _ in xs]
    for _ in range(20):
        for s in sides:
            s.wait_stream(torch.cuda.current_stream())
        got = [run(x, stream=s) for x, s in zip(xs, sides)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, held = [], []
    for x in xs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(run(x))
    for gr in graphs * 3:
        gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


@pytest.mark.gpu
def test_between_a_forward_and_its_backward():
    """forward_few leaves what the last forward left: routing, groups, gradients."""
    from paper_2608_10392_gb300 import FEATURE_BACKWARD, FEATURES_DEFAULT, Layer
    w, g = layer(256, 512, 4, 4, 3)
    on = {k: v.cuda() for k, v in w.items() if v is not None}
    L = Layer(256, 512, 4, 4, max_tokens=200, features=FEATURES_DEFAULT | FEATURE_BACKWARD)
    L.load_weights(on["router"], on["up"], on["down"])
    x, dy = (torch.randn(200, 256, generator=g).bfloat16().cuda() for _ in range(2))
    few = torch.randn(7, 256, generator=g).bfloat16().cuda()
    L.forward(x)
    route, groups = L.routing(), L.groups()
    L.forward_few(few)
    assert all(torch.equal(a, b) for a, b in zip(route.values(), L.routing().values()))
    assert all(torch.equal(a, b) for a, b in zip(groups, L.groups()))
    got = L.backward(x, dy)
    assert torch.isfinite(got["dx"]).all()
    # the layer's own forward of the same tokens: the same decisions, sums in another order
    y, z = L.forward(few).float(), L.forward_few(few).float()
    assert (y - z).abs().max() <= 2e-2 * y.abs().max()
    L.close()


@pytest.mark.gpu
def test_a_serving_step():
    """norm -> the layer for a few tokens -> norm with 8-bit rows -> product onto the stream, a
    step of a server, in one graph: the same as the calls one by one."""
    from paper_2608_10392_gb300 import BlockNorm, fp8_quantize, few_tokens, linear, router_table
    w, g = layer(256, 512, 4, 4, 5)
    on = {k: v.cuda() for k, v in w.items() if v is not None}
    table = router_table(on["router"], on["up"], 4)
    x = torch.randn(6, 256, generator=g).cuda()
    ones = torch.ones(256, device="cuda").bfloat16()
    opening, closing = (BlockNorm(256, stream_dtype="f32", pre_norm="rms", u_format=f) for f in ("branch", "fp8"))
    proj = fp8_quantize((torch.randn(256, 256, generator=g) / 16).cuda())

    def step():
        y = few_tokens(opening.forward(x, pre_weight=ones)["u"], table, on["up"], on["down"], 4)
        r = closing.forward(x, y, pre_weight=ones)
        return linear(r["u"], proj, residual=r["out"], dtype="f32")

    want = step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, want) and torch.isfinite(want).all()


# ------------------------------------------------------------------ refusals

def test_refusals():
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    p = C.c_void_p(4096)
    nan = math.nan

    def call(**k):
        v = dict(T=4, d=64, H=256, K=4, B=4, tau=nan, alpha=nan, beta=nan, topk=0, x=p, ld=64, router=p, up=p, down=p,
                 out=p, ld_out=64, ws=p, bytes=1 << 30)
        v.update(k)
        desc = ops._FewDesc(v["T"], v["d"], v["H"], v["K"], v["B"], v["tau"], v["alpha"], v["beta"], v["topk"], 0)
        return L.unif_moe_few_forward(C.byref(desc), v["x"], v["ld"], v["router"], None, v["up"], v["down"], None,
                                      v["out"], v["ld_out"], None, None, v["ws"], v["bytes"], None)

    for k in (dict(T=-1), dict(d=0), dict(H=0), dict(K=0), dict(K=65), dict(B=1), dict(B=65), dict(topk=5),
              dict(topk=-1), dict(alpha=1.5), dict(alpha=-0.1), dict(beta=math.inf), dict(tau=-math.inf), dict(x=None),
              dict(router=None), dict(up=None), dict(down=None), dict(out=None), dict(ld=63), dict(ld=68),
              dict(ld_out=63), dict(x=C.c_void_p(4104)), dict(up=C.c_void_p(4112)), dict(down=C.c_void_p(4112)),
              dict(router=C.c_void_p(4104)), dict(ws=C.c_void_p(4104))):
        assert call(**k) == -1, k
    for k in (dict(d=96), dict(H=128, B=4), dict(H=255)):
        assert call(**k) == -2, k
    for k in (dict(T=65), dict(ws=None), dict(bytes=100)):
        assert call(**k) == -3, k
    assert call(T=0, x=None) == 0
    assert L.unif_moe_few_forward(None, p, 64, p, None, p, p, None, p, 64, None, None, p, 0, None) == -1
    assert L.unif_moe_forward_few(None, p, 64, 4, None, p, 64, None, None, p, 0, None) == -1
    assert L.unif_moe_forward_few_workspace(None, 4) == -1 and L.unif_moe_few_workspace(None) == -1
    assert L.unif_moe_router_table(64, 256, 4, 4, None, p, p, None) == -1
    assert L.unif_moe_router_table(64, 250, 4, 4, p, p, p, None) == -2
    x = torch.zeros(4, 64).bfloat16()
    with pytest.raises(ValueError, match="x: need a CUDA tensor"):
        pkg.few_tokens(x, x, x, x, 4)


@pytest.mark.gpu
def test_refusals_of_tensors_and_handles():
    import paper_2608_10392_gb300 as pkg
    w, g = layer(64, 256, 3, 4, 1)
    on = {k: v.cuda() for k, v in w.items() if v is not None}
    table = pkg.router_table(on["router"], on["up"], 4)
    x = torch.zeros(4, 64, device="cuda").bfloat16()
    for bad in ((x.float(), table, on["up"], on["down"]), (x, table[:7], on["up"], on["down"]),
                (x, table, on["up"][:2], on["down"]), (x, table, on["up"], on["down"][:, :32]),
                (x[:, :32], table, on["up"], on["down"]), (x, table, on["up"].float(), on["down"])):
        with pytest.raises(ValueError):
            pkg.few_tokens(*bad, 4)
    with pytest.raises(pkg.UnifMoeError, match="above 64"):
        pkg.few_tokens(torch.zeros(65, 64, device="cuda").bfloat16(), table, on["up"], on["down"], 4)
    L = pkg.Layer(64, 256, 3, 4, max_tokens=8)
    with pytest.raises(pkg.UnifMoeError, match="ERR_STATE"):
        L.forward_few(x)
    f = pkg.Layer(64, 256, 3, 4, dtype="f32", max_tokens=8)
    with pytest.raises(pkg.UnifMoeError, match="ERR_SHAPE"):
        f.forward_few(x)
    L.load_weights(on["router"], on["up"], on["down"])
    with pytest.raises(ValueError):
        L.forward_few(torch.zeros(4, 128, device="cuda").bfloat16())


@pytest.mark.gpu
def test_weights_in_another_layout_are_refused():
    """As many elements in another order: a router as columns, w_down as w_up's layout."""
    import paper_2608_10392_gb300 as pkg
    d, H, K, B = 64, 256, 3, 4
    w, g = layer(d, H, K, B, 1)
    on = {k: v.cuda() for k, v in w.items() if v is not None}
    with pytest.raises(ValueError, match=r"w_router: need \[64\]\[4\]"):
        pkg.router_table(on["router"].T.contiguous(), on["up"], B)
    with pytest.raises(ValueError, match="w_router"):
        pkg.router_table(on["router"].flatten(), on["up"], B)
    with pytest.raises(ValueError, match="contiguous"):
        pkg.router_table(on["router"].T.contiguous().T, on["up"], B)
    table = pkg.router_table(on["router"], on["up"], B)
    x = torch.zeros(4, d, device="cuda").bfloat16()
    for down in (on["down"].transpose(1, 2).contiguous(), on["down"].transpose(0, 1).contiguous(), on["down"].flatten(0, 1)):
        with pytest.raises(ValueError, match=r"w_down: need \[4\]\[64\]\[256\]"):
            pkg.few_tokens(x, table, on["up"], down, B)
    with pytest.raises(ValueError, match="contiguous"):
        pkg.few_tokens(x, table, on["up"], on["down"].transpose(1, 2).contiguous().transpose(1, 2), B)
    with pytest.raises(ValueError, match=r"router: need \[8\]\[64\]"):
        pkg.few_tokens(x, table.T.contiguous(), on["up"], on["down"], B)
    with pytest.raises(ValueError, match="router"):
        pkg.few_tokens(x, None, on["up"], on["down"], B)
    assert (pkg.few_tokens(x, table, on["up"], on["down"], B) == 0).all()


def test_results_over_operands_are_refused():
    """out, the counts and the workspace over each other and over all that the call reads, but for out over x. (Made-up
    addresses: each call is refused before anything is launched.)"""
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    T, d, H, K, B = 30, 64, 256, 3, 4
    desc = ops._FewDesc(T, d, H, K, B, math.nan, math.nan, math.nan, 0, 0)
    need = L.unif_moe_few_workspace(C.byref(desc))
    weights = (K + 1) * H * d * 2
    size = dict(x=T * d * 2, router=(1 + K + B) * d * 2, bias=4 * (K + 1), up=weights, down=weights, mask=T, out=T * d * 2,
                b=4 * T, k=4 * T, ws=need)
    places = {name: (i + 1) << 28 for i, name in enumerate(size)}
    for result in ("out", "b", "k", "ws"):
        for name in size:
            for shift in (0, -((size[result] - 1) // 16 * 16), (size[name] - 1) // 16 * 16):
                if name == result or (result, name) == ("out", "x"):
                    continue
                at = {**places, result: places[name] + shift}
                rc = L.unif_moe_few_forward(C.byref(desc), at["x"], d, at["router"], at["bias"], at["up"], at["down"],
                                            at["mask"], at["out"], d, at["b"], at["k"], at["ws"], need, None)
                assert rc == -1 and b"overlaps" in L.unif_moe_last_error(), (result, name, shift)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 30])
def test_out_over_x_a_row_further(T):
    from paper_2608_10392_gb300 import few_tokens, router_table
    w, g = layer(256, 512, 4, 4, 2)
    on = {k: None if v is None else v.cuda() for k, v in w.items()}
    table = router_table(on["router"], on["up"], 4)
    both = torch.randn(T + 1, 256, generator=g).bfloat16().cuda()
    x = both[:T].clone()
    want = few_tokens(x, table, on["up"], on["down"], 4)
    few_tokens(both[:T], table, on["up"], on["down"], 4, out=both[1:])
    assert torch.equal(both[1:], want) and torch.equal(both[0], x[0])


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,H,K,B,code", [(4, 96, 256, 3, 4, "ERR_SHAPE"), (4, 64, 128, 3, 4, "ERR_SHAPE"),
                                            (65, 64, 256, 3, 4, "ERR_CAPACITY"), (65, 96, 256, 3, 4, "ERR_CAPACITY")])
def test_refusals_have_the_code_of_the_call(T, d, H, K, B, code):
    import paper_2608_10392_gb300 as pkg
    t = lambda *s: torch.zeros(*s, device="cuda").bfloat16()  # noqa: E731
    with pytest.raises(pkg.UnifMoeError, match=code):
        pkg.few_tokens(t(T, d), t(1 + K + B, d), t(K + 1, H, d), t(K + 1, d, H), B)
    with pytest.raises(pkg.UnifMoeError, match="ERR_ARG"):
        pkg.few_tokens(t(4, 64), t(8, 64), t(4, 256, 64), t(4, 64, 256), 4, alpha_fixed=2.0)
