"""The norms round a block with gate and scaled residual (BlockNorm): forward and
backward against the formulas in 64 bits, gradients also against differences of
the 64-bit forward; widths, row counts, strides, gates and masks at which the
kernels take another path; refusals.

Tolerances. A value stored in bf16 is rounded once: 2^-8 of it covers the rounding
(2^-9) and a sum that falls on the other side of a rounding boundary. Before
that, everything is fp32: a sum over a row adds at most log2(1024) + 8 + 32
roundings of 2^-24 to terms no larger than the row's largest, and each result
passes about ten more operations, so 64 * 2^-24 ~ 4e-6 of the size of the terms
that it is made of bounds it; 2e-5 is used, of the sum of the absolute values of
those terms. A column sum adds at most 600 terms in a row (2,400 rows over the
fewest CTAs, see the row counts below) and a tree: 700 * 2^-24 ~ 4e-5 of the sum
of the absolute terms, with the terms' own 2e-5: 1e-4.
"""
import ctypes as C

import pytest
import torch

EPS = 1e-5
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(T, d, stream, branch, post, pre, gate_rows, bias, masked, seed, dev, scale=0.75):
    """Inputs (values of the storage types) and their 64-bit copies on the CPU."""
    g = torch.Generator().manual_seed(seed)

    def r(*shape, dtype, k=1.0, m=0.0):
        return (torch.randn(*shape, generator=g, dtype=torch.float64) * k + m).to(TYPES[dtype])

    v = dict(x=r(T, d, dtype=stream, m=0.3), y=r(T, d, dtype=branch, k=0.8, m=-0.2),
             dout=r(T, d, dtype=stream), du=r(T, d, dtype=branch))
    G = None if gate_rows is None else 1 if gate_rows == 0 else -(-T // gate_rows)
    v["gate"] = None if G is None else r(G, d, dtype=branch, k=0.5)
    for n, on in (("post", post != "none"), ("pre", pre != "none")):
        v[n + "_weight"] = r(d, dtype=branch, k=0.2, m=1.0) if on else None
        v[n + "_bias"] = r(d, dtype=branch, k=0.2) if on and bias else None
    mask = None
    if masked:
        mask = torch.rand(T, generator=g) < 0.6
        if masked == "all":
            mask[:] = False
        for n in ("x", "y", "dout", "du"):
            v[n][~mask] = float("nan")
    v["mask"] = mask
    on_gpu = {k: None if t is None else t.to(dev) for k, t in v.items()}
    exact = {k: None if t is None else (t if k == "mask" else t.double()) for k, t in v.items()}
    cfg = dict(T=T, d=d, post=post, pre=pre, gate_rows=gate_rows, scale=scale)
    return cfg, on_gpu, exact


def keep_of(cfg, e):
    return torch.ones(cfg["T"], dtype=torch.bool) if e["mask"] is None else e["mask"]


def norm64(v, kind):
    """(standardised rows, mean, 1 / sqrt) in 64 bits."""
    mean = v.mean(1) if kind == "layer" else torch.zeros(v.shape[0], dtype=torch.float64)
    c = v - mean[:, None]
    rstd = 1 / torch.sqrt(c.square().mean(1) + EPS)
    return c * rstd[:, None], mean, rstd


def gates(cfg, gate, rows):
    if gate is None:
        return torch.ones(1, cfg["d"], dtype=torch.float64)
    return gate[rows // cfg["gate_rows"]] if cfg["gate_rows"] else gate


def forward64(cfg, e, rows, x, y, p):
    z = y
    if cfg["post"] != "none":
        z = norm64(y, cfg["post"])[0] * p["post_weight"]
        z = z if p.get("post_bias") is None else z + p["post_bias"]
    out = cfg["scale"] * x + gates(cfg, p.get("gate"), rows) * z
    u = None
    if cfg["pre"] != "none":
        u = norm64(out, cfg["pre"])[0] * p["pre_weight"]
        u = u if p.get("pre_bias") is None else u + p["pre_bias"]
    return out, u


def layer_of(cfg, stream, branch):
    from paper_2608_10392_gb300 import BlockNorm
    return BlockNorm(cfg["d"], stream_dtype=stream, branch_dtype=branch, post_norm=cfg["post"],
                     pre_norm=cfg["pre"], gate_rows=cfg["gate_rows"] or 0,
                     res_scale=cfg["scale"], eps=EPS)


PARAMS = ("post_weight", "post_bias", "gate", "pre_weight")


def close(got, want, tol, what):
    got = got.double().cpu()
    bad = (got - want).abs() > tol
    assert not bad.any(), "%s: %d off, worst %.3g over its tolerance" % (
        what, int(bad.sum()), float(((got - want).abs() / tol.clamp(min=1e-300)).max()))


CASES = [
    # T, d, stream, branch, post, pre, gate_rows, bias, masked
    (1, 1024, "bf16", "bf16", "rms", "rms", 0, False, None),
    (7, 64, "f32", "f32", "layer", "layer", 1, True, None),
    (33, 48, "f32", "bf16", "rms", "layer", 5, True, "some"),
    (130, 128, "bf16", "bf16", "layer", "rms", None, True, None),
    (300, 256, "f32", "bf16", "none", "layer", 0, False, "some"),
    (2400, 384, "f32", "bf16", "layer", "layer", 197, True, "some"),
    (788, 768, "bf16", "bf16", "rms", "rms", 197, False, None),
    (515, 1024, "f32", "f32", "rms", "none", 0, True, None),
    (41, 2056, "bf16", "bf16", "layer", "layer", 3, True, "some"),
    (9, 8192, "f32", "bf16", "rms", "rms", 0, True, None),
    (5, 8192, "bf16", "bf16", "layer", "layer", 1, True, None),
    (12, 5000, "f32", "f32", "layer", "rms", 64, True, "some"),
    # widths that are no multiple of eight
    (65, 1, "f32", "f32", "rms", "rms", 0, True, None),
    (50, 37, "bf16", "bf16", "layer", "layer", 7, True, "some"),
    (21, 333, "f32", "bf16", "rms", "layer", 0, True, None),
    (19, 1001, "bf16", "bf16", "layer", "rms", 1000, True, None),
    (4, 7777, "f32", "f32", "layer", "layer", 2, True, None),
    # no valid row at all
    (40, 96, "bf16", "bf16", "layer", "layer", 8, True, "all"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_forward_against_64_bits(case):
    T, d, stream, branch = case[:4]
    cfg, v, e = make(*case, seed=3, dev="cuda")
    r = layer_of(cfg, stream, branch).forward(v["x"], v["y"], mask=v["mask"],
                                              pre_bias=v["pre_bias"], stats=True,
                                              **{k: v[k] for k in PARAMS})
    keep = keep_of(cfg, e)
    rows = torch.arange(T)[keep]
    out, u = forward64(cfg, e, rows, e["x"][keep], e["y"][keep], e)
    terms = (cfg["scale"] * e["x"][keep]).abs() + out.abs() + 1
    close(r["out"][keep.cuda()], out, ROUND[stream] * out.abs() + 2e-5 * terms, "out")
    assert not r["out"][~keep.cuda()].any()
    if cfg["pre"] == "none":
        assert r["u"] is None
    else:
        n, mean, rstd = norm64(out, cfg["pre"])
        terms = (rstd * (out.abs().amax(1) + 1))[:, None] * e["pre_weight"].abs() + u.abs()
        close(r["u"][keep.cuda()], u, ROUND[branch] * u.abs() + 2e-5 * terms, "u")
        assert not r["u"][~keep.cuda()].any()
        close(r["pre_mean"][keep.cuda()], mean, 2e-5 * (out.abs().mean(1) + 1), "mean")
        # d rstd = -rstd^3 d(var) / 2, and the variance is exact to 2e-5 of the squares
        close(r["pre_rstd"][keep.cuda()], rstd,
              2e-5 * rstd + 2e-5 * rstd ** 3 * (out.square().mean(1) + 1), "rstd")
        assert not r["pre_rstd"][~keep.cuda()].any()


def backward64(cfg, e):
    """Gradients by the formulas in 64 bits, and the sums of the absolute values of
    the terms of the parameters' gradients."""
    keep = keep_of(cfg, e)
    rows = torch.arange(cfg["T"])[keep]
    out, y, dout, du = (e[k][keep] for k in ("x", "y", "dout", "du"))
    p, g, size = e, {}, {}

    def through(a, n, rstd, kind):
        a = a - a.mean(1, keepdim=True) if kind == "layer" else a
        return rstd[:, None] * (a - n * (a * n).mean(1, keepdim=True))

    def total(name, terms):
        g[name], size[name] = terms.sum(0), terms.abs().sum(0)

    D = dout
    size["dx"] = D.abs()
    if cfg["pre"] != "none":
        n, _, rstd = norm64(out, cfg["pre"])
        total("d_pre_weight", du * n)
        total("d_pre_bias", du)
        a = du * p["pre_weight"]
        D = D + through(a, n, rstd, cfg["pre"])
        size["dx"] = size["dx"] + rstd[:, None] * (a.abs() + (1 + n.abs()) *
                                                   (a * n).abs().mean(1, keepdim=True)
                                                   + a.abs().mean(1, keepdim=True))
    g["dx"] = cfg["scale"] * D
    yn, rstd = y, torch.ones(len(y), dtype=torch.float64)
    if cfg["post"] != "none":
        yn, _, rstd = norm64(y, cfg["post"])
    if p["gate"] is not None:
        z = yn
        if cfg["post"] != "none":
            z = z * p["post_weight"] + (0 if p["post_bias"] is None else p["post_bias"])
        at = rows // cfg["gate_rows"] if cfg["gate_rows"] else torch.zeros_like(rows)
        g["d_gate"] = torch.zeros_like(p["gate"]).index_add_(0, at, D * z)
        size["d_gate"] = torch.zeros_like(p["gate"]).index_add_(0, at, size["dx"] * (z.abs() + 1))
    gate = gates(cfg, p["gate"], rows)
    D, size["dy"] = D * gate, size["dx"] * gate.abs()
    if cfg["post"] != "none":
        total("d_post_weight", D * yn)
        total("d_post_bias", D)
        # the terms of D, not D itself, bound its error
        size["d_post_weight"] = (size["dy"] * yn.abs()).sum(0)
        size["d_post_bias"] = size["dy"].sum(0)
        w = p["post_weight"].abs()
        s = size["dy"] * w
        size["dy"] = rstd[:, None] * (s + s.mean(1, keepdim=True)
                                      + (1 + yn.abs()) * (s * yn.abs()).mean(1, keepdim=True))
        D = through(D * p["post_weight"], yn, rstd, cfg["post"])
    g["dy"] = D
    size["dx"] = size["dx"] * abs(cfg["scale"])
    return keep, g, size


def statistics(cfg, e, dev="cuda"):
    keep = keep_of(cfg, e)
    s = {}
    for name, src, kind in (("post", e["y"], cfg["post"]), ("pre", e["x"], cfg["pre"])):
        mean, rstd = torch.zeros(cfg["T"]), torch.zeros(cfg["T"])
        if kind != "none" and keep.any():
            _, m, r = norm64(src[keep], kind)
            mean[keep], rstd[keep] = m.float(), r.float()
        s[name + "_mean"], s[name + "_rstd"] = mean.to(dev), rstd.to(dev)
    return s


def run_backward(cfg, v, e, stream, branch):
    return layer_of(cfg, stream, branch).backward(
        v["x"], v["y"], statistics(cfg, e), dout=v["dout"],
        du=v["du"] if cfg["pre"] != "none" else None, mask=v["mask"], **{k: v[k] for k in PARAMS})


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_backward_against_64_bits(case):
    stream, branch = case[2:4]
    cfg, v, e = make(*case, seed=5, dev="cuda")
    r = run_backward(cfg, v, e, stream, branch)
    keep, g, size = backward64(cfg, e)
    k = keep.cuda()
    close(r["dx"][k], g["dx"], ROUND[stream] * g["dx"].abs() + 2e-5 * size["dx"], "dx")
    close(r["dy"][k], g["dy"], ROUND[branch] * g["dy"].abs() + 4e-5 * size["dy"], "dy")
    assert not r["dx"][~k].any() and not r["dy"][~k].any()
    wanted = [n for n in g if n not in ("dx", "dy")]
    assert sorted(wanted) == sorted(n for n in r if n not in ("dx", "dy"))
    for n in wanted:
        close(r[n], g[n], 1e-4 * size[n] + 1e-30, n)


@pytest.mark.gpu
@pytest.mark.parametrize("post,pre", [("layer", "rms"), ("rms", "layer")])
def test_gradients_against_differences(post, pre):
    """Directional differences of the 64-bit forward: with h = 1e-5 the quotient is
    off by h^2 times third derivatives (~1e-9 of the terms); 1e-4 covers the fp32
    gradients, as in the formulas' test."""
    T, d = 37, 72
    cfg, v, e = make(T, d, "f32", "f32", post, pre, 10, True, None, seed=9, dev="cuda")
    from paper_2608_10392_gb300 import BlockNorm
    norm = layer_of(cfg, "f32", "f32")
    fwd = norm.forward(v["x"], v["y"], pre_bias=v["pre_bias"], stats=True, **{k: v[k] for k in PARAMS})
    r = norm.backward(fwd["out"], v["y"], fwd, dout=v["dout"], du=v["du"],
                      **{k: v[k] for k in PARAMS})
    rows = torch.arange(T)
    names = {"x": "dx", "y": "dy", "gate": "d_gate", "post_weight": "d_post_weight",
             "post_bias": "d_post_bias", "pre_weight": "d_pre_weight", "pre_bias": "d_pre_bias"}

    def loss(p):
        out, u = forward64(cfg, e, rows, p["x"], p["y"], p)
        return (out * e["dout"]).sum() + (u * e["du"]).sum()

    gen = torch.Generator().manual_seed(1)
    for name, grad in names.items():
        t = torch.randn(e[name].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        diff = (loss(dict(e, **{name: e[name] + h * t})) - loss(dict(e, **{name: e[name] - h * t}))) / (2 * h)
        terms = r[grad].double().cpu() * t
        assert abs(float(terms.sum() - diff)) <= 1e-4 * float(terms.abs().sum()), name


@pytest.mark.gpu
def test_opening_form():
    """Without y: the norm before the first block, and its gradient."""
    for d, stream, branch in ((384, "f32", "bf16"), (50, "bf16", "bf16")):
        cfg, v, e = make(70, d, stream, branch, "none", "layer", None, True, "some", seed=2,
                         dev="cuda", scale=1.0)
        norm = layer_of(cfg, stream, branch)
        r = norm.forward(v["x"], pre_weight=v["pre_weight"], pre_bias=v["pre_bias"], mask=v["mask"],
                         stats=True)
        assert r["out"] is v["x"]
        keep = keep_of(cfg, e)
        n, _, rstd = norm64(e["x"][keep], "layer")
        want = n * e["pre_weight"] + e["pre_bias"]
        terms = (rstd * (e["x"][keep].abs().amax(1) + 1))[:, None] * e["pre_weight"].abs() + want.abs()
        close(r["u"][keep.cuda()], want, ROUND[branch] * want.abs() + 2e-5 * terms, "u")
        g = norm.backward(v["x"], None, r, dout=v["dout"], du=v["du"],
                          pre_weight=v["pre_weight"], mask=v["mask"])
        _, want, size = backward64(cfg, e)
        close(g["dx"][keep.cuda()], want["dx"], ROUND[stream] * want["dx"].abs() + 2e-5 * size["dx"], "dx")
        assert g["dy"] is None
        close(g["d_pre_weight"], want["d_pre_weight"], 1e-4 * size["d_pre_weight"], "d_pre_weight")


@pytest.mark.gpu
@pytest.mark.parametrize("pad,shift", [(16, 0), (3, 0), (8, 1)])
def test_strides_and_alignment_change_no_value(pad, shift):
    """Rows apart by more than the width, and rows that start off 16 bytes, give
    what dense rows give to 2e-5 of the terms (another column order in the sums)."""
    T, d = 61, 256
    cfg, v, e = make(T, d, "bf16", "bf16", "rms", "layer", 0, True, None, seed=4, dev="cuda")
    norm = layer_of(cfg, "bf16", "bf16")
    params = {k: v[k] for k in PARAMS}

    def apart(t):
        wide = torch.full((T, d + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
        view = wide[:, shift:shift + d]
        view.copy_(t)
        return view

    r = norm.forward(v["x"], v["y"], pre_bias=v["pre_bias"], **params)
    o, u = apart(torch.zeros_like(v["x"])), apart(torch.zeros_like(v["x"]))
    s = norm.forward(apart(v["x"]), apart(v["y"]), pre_bias=v["pre_bias"], out=o, u=u, **params)
    for k in ("out", "u"):
        close(s[k], r[k].double().cpu(), 2.0 ** -7 * r[k].double().cpu().abs() + 1e-4, k)
    assert torch.isnan(o._base[:, shift + d:]).all()
    a = norm.backward(v["x"], v["y"], statistics(cfg, e), dout=v["dout"], du=v["du"], **params)
    b = norm.backward(apart(v["x"]), apart(v["y"]), statistics(cfg, e), dout=apart(v["dout"]),
                      du=apart(v["du"]), **params)
    _, _, size = backward64(cfg, e)
    for k in a:
        tol = (2.0 ** -7 if k in ("dx", "dy") else 0) * a[k].double().cpu().abs() + 1e-4 * size[k]
        close(b[k], a[k].double().cpu(), tol, k)


@pytest.mark.gpu
def test_in_place_and_repeatable():
    cfg, v, e = make(900, 384, "bf16", "bf16", "rms", "rms", 100, False, None, seed=6, dev="cuda")
    norm = layer_of(cfg, "bf16", "bf16")
    params = {k: v[k] for k in PARAMS}
    r = norm.forward(v["x"], v["y"], **params)
    x, y = v["x"].clone(), v["y"].clone()
    s = norm.forward(x, y, out=x, u=y, **params)
    assert torch.equal(s["out"], r["out"]) and torch.equal(s["u"], r["u"])
    assert s["out"] is x and s["u"] is y
    a = run_backward(cfg, v, e, "bf16", "bf16")
    b = run_backward(cfg, v, e, "bf16", "bf16")
    assert all(torch.equal(a[k], b[k]) for k in a)


# Forwards over enough rows that a CTA takes several after one another: each width class,
# rows that are no multiple of a CTA's, gates that change inside a CTA's rows.
MANY = [
    (39001, 48, "bf16", "bf16", "rms", "layer", 1, True, "some"),
    (19999, 128, "bf16", "bf16", "layer", "rms", 7, True, None),
    (9803, 200, "bf16", "bf16", "none", "layer", 197, False, "some"),
    (5005, 384, "bf16", "bf16", "rms", "none", 1, True, "some"),
    (2433, 1000, "bf16", "bf16", "layer", "layer", 0, True, "some"),
    (2501, 4096, "bf16", "bf16", "rms", "rms", 64, False, None),
    (3001, 320, "bf16", "bf16", "layer", "rms", 0, True, "all"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", MANY, ids=lambda c: "-".join(map(str, c)))
def test_forward_of_many_rows_against_64_bits(case):
    test_forward_against_64_bits(case)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(5003, 384), (39007, 64)])
def test_many_rows_in_place_and_without_a_branch(T, d):
    cfg, v, e = make(T, d, "bf16", "bf16", "rms", "rms", 100, False, "some", seed=6, dev="cuda")
    norm = layer_of(cfg, "bf16", "bf16")
    params = {k: v[k] for k in PARAMS}
    r = norm.forward(v["x"], v["y"], mask=v["mask"], **params)
    x, y = v["x"].clone(), v["y"].clone()
    norm.forward(x, y, mask=v["mask"], out=x, u=y, **params)
    assert torch.equal(x, r["out"]) and torch.equal(y, r["u"])
    # the stream's rows as they are, normed: what a few rows at a time give
    norm = layer_of(dict(cfg, post="none", gate_rows=None, scale=1.0), "bf16", "bf16")
    u = norm.forward(r["out"], pre_weight=v["pre_weight"])["u"]
    for lo in (0, T // 2, T - 40):
        part = norm.forward(r["out"][lo:lo + 40], pre_weight=v["pre_weight"])["u"].double().cpu()
        close(u[lo:lo + 40], part, 2.0 ** -7 * part.abs() + 1e-4, "u")


@pytest.mark.gpu
def test_another_stream_and_no_tokens():
    cfg, v, e = make(500, 768, "f32", "bf16", "layer", "layer", 0, True, None, seed=8, dev="cuda")
    norm = layer_of(cfg, "f32", "bf16")
    params = {k: v[k] for k in PARAMS}
    r = norm.forward(v["x"], v["y"], **params)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s = norm.forward(v["x"], v["y"], **params)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(s["out"], r["out"]) and torch.equal(s["u"], r["u"])
    none = dict(x=v["x"][:0], y=v["y"][:0])
    assert norm.forward(none["x"], none["y"], **params)["u"].shape == (0, 768)
    g = norm.backward(none["x"], none["y"], {k: t[:0] for k, t in statistics(cfg, e).items()},
                      dout=none["x"], du=none["y"], **params)
    assert g["dx"].shape == (0, 768)
    assert not any(g[k].any() for k in ("d_gate", "d_post_weight", "d_pre_bias"))


@pytest.mark.gpu
def test_large_values_stay_finite_and_nan_stays_in_its_row():
    """bf16 values up to 1e18 have squares within fp32; a NaN spoils its own row only."""
    T, d = 40, 512
    cfg, v, e = make(T, d, "bf16", "bf16", "none", "rms", None, False, None, seed=1, dev="cuda",
                     scale=1.0)
    norm = layer_of(cfg, "bf16", "bf16")
    x = v["x"] * 1e17
    x[7, 3] = float("nan")
    x[9, 100] = float("inf")
    u = norm.forward(x, torch.zeros_like(x), pre_weight=v["pre_weight"])["u"]
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[7] = bad[9] = True
    assert torch.isfinite(u[~bad]).all() and torch.isnan(u[7]).all() and torch.isnan(u[9, 100])


@pytest.mark.gpu
def test_stream_argument():
    """Calls on a stream that is not the current one, one after another without
    waiting: workspaces and outputs of one call are not handed to the next too early."""
    cfg, v, e = make(3000, 768, "bf16", "bf16", "rms", "rms", 100, False, None, seed=6, dev="cuda")
    norm = layer_of(cfg, "bf16", "bf16")
    params = {k: v[k] for k in PARAMS}
    s = statistics(cfg, e)
    want = norm.backward(v["x"], v["y"], s, dout=v["dout"], du=v["du"], **params)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [norm.backward(v["x"], v["y"], s, dout=v["dout"], du=v["du"], stream=side, **params)
           for _ in range(20)]
    outs = [norm.forward(v["x"], v["y"], stream=side.cuda_stream, **params) for _ in range(3)]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(g[k], want[k]) for k in want)
    first = norm.forward(v["x"], v["y"], **params)
    assert all(torch.equal(o["u"], first["u"]) for o in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [
    # a gate row per token: two rows a step, groups of lanes, other widths, wide rows
    (300, 384, "bf16", "bf16", "layer", "rms", 1, True, "some"),
    (301, 1024, "f32", "bf16", "rms", "none", 1, True, "some"),
    (200, 64, "f32", "f32", "layer", "layer", 1, True, "some"),
    (211, 200, "bf16", "bf16", "rms", "layer", 1, True, "some"),
    (90, 37, "bf16", "bf16", "layer", "layer", 1, True, "some"),
    (60, 333, "f32", "bf16", "rms", "layer", 1, True, "some"),
    (40, 5000, "bf16", "bf16", "layer", "layer", 1, True, "some"),
    # gate rows of which all tokens are padding
    (640, 128, "bf16", "bf16", "layer", "rms", 3, True, "some"),
    (600, 256, "f32", "f32", "rms", "rms", 4, True, "some"),
    (500, 384, "bf16", "bf16", "rms", "layer", 2, True, "some"),
    (400, 50, "f32", "bf16", "layer", "layer", 3, True, "some")],
    ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_gates_of_padding_take_no_part(case, value):
    """Gate rows of padding tokens alone may hold anything (made from their activations)."""
    T, d, stream, branch = case[:4]
    cfg, v, e = make(*case, seed=11, dev="cuda")
    gr = cfg["gate_rows"]
    used = torch.zeros(len(e["gate"]), dtype=torch.bool)
    used[torch.arange(T)[e["mask"]] // gr] = True
    assert not used.all()
    v["gate"][~used.cuda()] = value
    norm = layer_of(cfg, stream, branch)
    r = norm.forward(v["x"], v["y"], mask=v["mask"], pre_bias=v["pre_bias"],
                     **{k: v[k] for k in PARAMS})
    assert torch.isfinite(r["out"]).all() and (r["u"] is None or torch.isfinite(r["u"]).all())
    r = run_backward(cfg, v, e, stream, branch)
    keep, g, size = backward64(cfg, e)
    close(r["dy"][keep.cuda()], g["dy"], ROUND[branch] * g["dy"].abs() + 4e-5 * size["dy"], "dy")
    assert not r["dx"][~keep.cuda()].any() and not r["dy"][~keep.cuda()].any()
    for n in g:
        assert torch.isfinite(r[n]).all(), n
        if n not in ("dx", "dy"):
            close(r[n], g[n], 1e-4 * size[n] + 1e-30, n)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES + MANY, ids=lambda c: "-".join(map(str, c)))
def test_nothing_but_numbers(case):
    """No NaN or infinity in any result (a comparison with a tolerance lets NaN pass)."""
    stream, branch = case[2:4]
    cfg, v, e = make(*case, seed=21, dev="cuda")
    r = layer_of(cfg, stream, branch).forward(v["x"], v["y"], mask=v["mask"], pre_bias=v["pre_bias"],
                                              **{k: v[k] for k in PARAMS})
    r.update(run_backward(cfg, v, e, stream, branch))
    assert all(torch.isfinite(t).all() for t in r.values() if t is not None)


@pytest.mark.gpu
def test_statistics_and_results_of_absent_norms():
    """None, not memory that nothing has written."""
    cfg, v, e = make(30, 64, "f32", "f32", "rms", "layer", None, False, None, seed=2, dev="cuda")
    x, y, w = v["x"], v["y"], v["pre_weight"]

    def run(post, pre, y, **k):
        return layer_of(dict(cfg, post=post, pre=pre, gate_rows=None), "f32", "f32").forward(
            x, y, post_weight=w if post != "none" else None, pre_weight=w if pre != "none" else None,
            stats=True, **k)

    for post, pre, branch in (("none", "layer", y), ("rms", "none", y), ("none", "none", y),
                              ("layer", "rms", y), ("none", "rms", None)):
        r = run(post, pre, branch)
        for name, kind in (("post", post), ("pre", pre)):
            assert (r[name + "_rstd"] is None) == (kind == "none")
            assert (r[name + "_mean"] is None) == (kind == "none")
            if kind == "rms":
                assert not r[name + "_mean"].any()
    given = torch.full_like(x, 3.0)
    assert run("rms", "none", y, u=given)["u"] is None and (given == 3).all()


@pytest.mark.gpu
def test_any_true_value_asks_for_statistics_and_gradients():
    from paper_2608_10392_gb300 import balance_loss
    cfg, v, e = make(30, 64, "f32", "f32", "none", "rms", None, False, None, seed=2, dev="cuda")
    norm = layer_of(cfg, "f32", "f32")
    for yes, no in ((1, 0), ([1], []), ("yes", None)):
        assert "pre_rstd" in norm.forward(v["x"], pre_weight=v["pre_weight"], stats=yes)
        assert "pre_rstd" not in norm.forward(v["x"], pre_weight=v["pre_weight"], stats=no)
        q = torch.zeros(30, 1, dtype=torch.int32, device="cuda")
        assert balance_loss(v["x"], q, grad=yes)["dlogits"] is not None
        assert balance_loss(v["x"], q, grad=no)["dlogits"] is None


@pytest.mark.gpu
def test_sizes_beyond_32_bits_are_refused():
    from paper_2608_10392_gb300 import BlockNorm
    x, w = torch.ones(4, 64, device="cuda"), torch.ones(64, device="cuda")
    for k in (dict(width=64 + (1 << 32)), dict(width=64, gate_rows=(1 << 32) + 2)):
        norm = BlockNorm(stream_dtype="f32", branch_dtype="f32", **k)
        with pytest.raises(ValueError, match="32"):
            norm.forward(x, x, gate=torch.ones(2, 64, device="cuda"), pre_weight=w)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [
    (700, 384, "bf16", "bf16", "rms", "rms", 64, True, "some"),
    (400, 1000, "bf16", "bf16", "layer", "layer", 0, True, None),
    (300, 96, "bf16", "bf16", "layer", "rms", 1, True, "some"),
    (100, 333, "bf16", "bf16", "rms", "layer", None, False, None),
    (2500, 768, "bf16", "bf16", "none", "layer", 0, True, "some"),
    (500, 640, "f32", "bf16", "layer", "rms", 7, True, "some")],
    ids=lambda c: "-".join(map(str, c)))
def test_a_training_steps_chain(case):
    """The forward's own out and statistics into the backward, against the gradient of the
    whole in 64 bits, and the branch's statistics themselves. The statistics are those of
    the sum before its rounding to the stream's type, so that o^ = (out - m) r is off by
    r times a rounding of out (at most 2^-8 of it in bf16), which passes through the
    formulas."""
    T, d, stream, branch = case[:4]
    cfg, v, e = make(*case, seed=13, dev="cuda")
    keep = keep_of(cfg, e)
    k, rows = keep.cuda(), torch.arange(T)[keep]
    norm = layer_of(cfg, stream, branch)
    params = {n: v[n] for n in PARAMS}
    f = norm.forward(v["x"], v["y"], mask=v["mask"], pre_bias=v["pre_bias"], stats=True, **params)
    y = e["y"][keep]
    yn, ry = y, torch.ones(len(y), 1, dtype=torch.float64)
    if cfg["post"] != "none":
        yn, mean, rstd = norm64(y, cfg["post"])
        ry = rstd[:, None]
        close(f["post_mean"][k], mean, 2e-5 * (y.abs().mean(1) + 1), "post_mean")
        close(f["post_rstd"][k], rstd,
              2e-5 * rstd + 2e-5 * rstd ** 3 * (y.square().mean(1) + 1), "post_rstd")
        assert not f["post_rstd"][~k].any() and not f["post_mean"][~k].any()
    r = norm.backward(f["out"], v["y"], f, dout=v["dout"], du=v["du"], mask=v["mask"], **params)
    out = forward64(cfg, e, rows, e["x"][keep], y, e)[0]
    whole = torch.zeros(T, d, dtype=torch.float64)
    whole[keep] = out
    _, g, size = backward64(cfg, dict(e, x=whole))
    n, _, rstd = norm64(out, cfg["pre"])
    a, off = (e["du"][keep] * e["pre_weight"]).abs(), ROUND[stream] * out.abs() * rstd[:, None]
    more = {"d_pre_weight": (e["du"][keep].abs() * off).sum(0), "d_pre_bias": 0.0}
    D = rstd[:, None] * (off * (a * (n.abs() + off)).mean(1, keepdim=True)
                         + n.abs() * (a * off).mean(1, keepdim=True))
    more["dx"] = abs(cfg["scale"]) * D
    if e["gate"] is not None:
        z = yn
        if cfg["post"] != "none":
            z = z * e["post_weight"] + (0 if e["post_bias"] is None else e["post_bias"])
        at = rows // cfg["gate_rows"] if cfg["gate_rows"] else torch.zeros_like(rows)
        more["d_gate"] = torch.zeros_like(e["gate"]).index_add_(0, at, D * z.abs())
    D = D * gates(cfg, e["gate"], rows).abs()
    if cfg["post"] != "none":
        more["d_post_weight"], more["d_post_bias"] = (D * yn.abs()).sum(0), D.sum(0)
        D = D * e["post_weight"].abs()
        D = ry * (D + D.mean(1, keepdim=True) + yn.abs() * (D * yn.abs()).mean(1, keepdim=True))
    more["dy"] = D
    close(r["dx"][k], g["dx"], ROUND[stream] * (g["dx"].abs() + more["dx"]) + 2e-5 * size["dx"]
          + more["dx"], "dx")
    close(r["dy"][k], g["dy"], ROUND[branch] * (g["dy"].abs() + more["dy"]) + 4e-5 * size["dy"]
          + more["dy"], "dy")
    for name in g:
        assert torch.isfinite(r[name]).all(), name
        if name not in ("dx", "dy"):
            close(r[name], g[name], 1e-4 * size[name] + more[name] + 1e-30, name)


def test_refusals():
    """Bad descriptions and arguments are refused before anything runs (no GPU needed)."""
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300.operators import _BlockNormDesc as D
    L = pkg.lib()
    one = C.c_void_p(4096)

    def fwd(desc, x=one, y=one, w_post=one, gate=None, w_pre=one, out=one, u=one, ld=64):
        return L.unif_moe_block_norm_forward(
            None if desc is None else C.byref(desc), x, ld, y, 64, None, w_post, None, gate, w_pre,
            None, out, 64, u, 64, None, None, None, None, None)

    good = (4, 64, 0, 0, 2, 2, 0, 1.0, 1e-6)

    def bad(i, value):
        a = list(good)
        a[i] = value
        return D(*a)

    assert fwd(None) == -1
    for i, value in ((0, -1), (1, 0), (2, 2), (3, -1), (4, 3), (5, -1), (6, -1),
                     (7, float("inf")), (8, -1.0), (8, float("nan"))):
        assert fwd(bad(i, value)) == -1, (i, value)
    assert fwd(bad(1, 8193)) == -2 and b"width" in L.unif_moe_last_error()
    assert fwd(bad(0, 0x7fff0001)) == -2 and b"tokens" in L.unif_moe_last_error()
    assert fwd(D(4, 64, 1, 0, 2, 2, 0, 1.0, 1e-6)) == -1  # bf16 stream, fp32 branch
    assert fwd(D(*good), w_post=None) == -1
    assert fwd(D(*good), w_pre=None) == -1
    assert fwd(D(*good), x=None) == -1
    assert fwd(D(*good), u=None) == -1
    assert fwd(D(*good), y=None) == -1           # post norm without y
    assert fwd(D(*good), ld=63) == -1
    assert fwd(D(4, 64, 0, 0, 0, 0, 0, 1.0, 1e-6), y=None, out=None) == -1  # nothing to do
    assert L.unif_moe_block_norm_workspace(C.byref(bad(1, 0)), 0) == -1

    def bwd(desc, **k):
        a = dict(out=one, y=one, w_post=one, gate=None, w_pre=one, r_post=one, r_pre=one, dout=one,
                 du=one, dw_post=None, d_gate=None, ld=64)
        a.update(k)
        return L.unif_moe_block_norm_backward(
            C.byref(desc), a["out"], 64, a["y"], 64, None, a["w_post"], None, a["gate"], a["w_pre"],
            None, a["r_post"], None, a["r_pre"], a["dout"], a["ld"], a["du"], 64, one, 64,
            one if a["y"] else None, 64, a["dw_post"], None, a["d_gate"], None, None, None, 0, None)

    for k in (dict(w_post=None), dict(w_pre=None), dict(r_post=None), dict(r_pre=None),
              dict(du=None), dict(out=None), dict(y=None), dict(d_gate=one), dict(ld=1)):
        assert bwd(D(*good), **k) == -1, k
    assert bwd(D(4, 64, 0, 0, 1, 2, 0, 1.0, 1e-6)) == -1      # layer norm without its means
    assert bwd(D(4, 64, 0, 0, 0, 2, 0, 1.0, 1e-6), dw_post=one) == -1
    with pytest.raises(KeyError):
        pkg.BlockNorm(64, post_norm="batch")
    with pytest.raises(ValueError, match="x"):
        pkg.BlockNorm(64).forward(torch.zeros(2, 32), torch.zeros(2, 32), pre_weight=torch.ones(64))
