"""The dense products (linear, linear_backward) against 64 bits: sizes from one row to many,
odd widths, strides, masks, 8-bit rows, in-place residuals, gradients against the formula's
and against differences; refusals.

Tolerances. Products of two bf16 (or two 8-bit) values are exact in fp32. The tensor cores add
16 (32) of them to an fp32 sum and cut it: with S the sum of the terms' absolute values a
step loses at most 2^-22 S, so a sum over c columns is within (c / 16 + 2) 2^-22 S (the two:
sums of warps or parts). Scales, bias and residual are fp32 operations, 2^-23 of what they
give each: 4 in all. GELU has a slope of at most 1.13 and its own 2^-11 of the value in bf16
results, 2^-20 (normcdff and a product) in fp32 ones. A result is rounded once: 2^-8 in bf16."""
import ctypes as C
import math

import pytest
import torch

F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def gelu(z):
    return z * torch.special.ndtr(z)


def operand(rows, cols, g, pad=0, shift=0, scale=1.0):
    """bf16 rows, `pad` elements apart, `shift` elements into their buffer."""
    wide = torch.randn(rows, cols + pad + shift, generator=g, device="cuda").mul_(scale).bfloat16()
    return wide[:, shift:shift + cols]


def eight(rows, cols, g, pad=0, scale=1.0):
    from paper_2608_10392_gb300 import Fp8
    v = (torch.randn(rows, cols + pad, generator=g, device="cuda") * 60).clamp(-448, 448)
    return Fp8(v.to(torch.float8_e4m3fn)[:, :cols],
               scale / 60 * (0.5 + torch.rand(rows, generator=g, device="cuda")))


def value(x):
    if isinstance(x, torch.Tensor):
        return x.to(F64)
    return x.codes.to(F64) * x.scales.to(F64)[:, None]


def check(x, w, bias=None, act="none", residual=None, mask=None, dtype="bf16", keep=False, out=None, **kw):
    from paper_2608_10392_gb300 import linear, linear_status
    before = None if residual is None else residual.to(F64)
    got = linear(x, w, bias, activation=act, residual=residual, mask=mask, dtype=dtype, keep=keep, out=out, **kw)
    assert linear_status() == 0
    got, z_got = got if keep else (got, None)
    xv, wv = value(x), value(w)
    on = torch.ones(len(xv), dtype=torch.bool, device="cuda") if mask is None else mask != 0
    xv = torch.where(on[:, None], xv, 0.0)
    z = xv @ wv.T
    size = xv.abs() @ wv.abs().T
    step = 16 if isinstance(x, torch.Tensor) else 32
    tol = (xv.shape[1] / step + 2) * 2.0 ** -22 * size
    if bias is not None:
        z = z + bias.to(F64)
    tol = tol + 4 * 2.0 ** -23 * (size + z.abs())
    z_tol = tol + 2.0 ** -8 * z.abs()
    y = z
    if act == "gelu":
        y = gelu(z)
        tol = 1.13 * tol + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -20) * y.abs() + 2e-37
    if residual is not None:
        y = y + torch.where(on[:, None], before, 0.0)
        tol = tol + 2.0 ** -23 * (y.abs() + before.abs().nan_to_num())
    tol = tol + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * y.abs()
    assert got.shape == y.shape and got.dtype == TYPES[dtype]
    y, z = torch.where(on[:, None], y, 0.0), torch.where(on[:, None], z, 0.0)
    err = (got.to(F64) - y).abs()
    bad = ~(err <= torch.where(on[:, None], tol, 0.0))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(err.nan_to_num(1e9).max()))
    if keep:
        bad = ~((z_got.to(F64) - z).abs() <= torch.where(on[:, None], z_tol, 0.0))
        assert z_got.dtype == torch.bfloat16 and not bad.any(), int(bad.sum())
    return got


def inputs(T, cols, n, seed, kind="bf16", bias=None, residual=None, masked=False, dtype="bf16"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = operand if kind == "bf16" else eight
    r = dict(x=make(T, cols, g), w=make(n, cols, g, scale=cols ** -0.5))
    if bias:
        r["bias"] = torch.randn(n, generator=g, device="cuda").to(TYPES[bias])
    if residual:
        r["residual"] = (2 * torch.randn(T, n, generator=g, device="cuda")).to(TYPES[dtype])
    if masked:
        r["mask"] = torch.rand(T, generator=g, device="cuda") < 0.6
        if kind == "bf16":
            r["x"][~r["mask"]] = float("nan")
        else:
            r["x"].codes.view(torch.uint8)[~r["mask"]] = 0x7f  # NaN
        if residual:
            r["residual"][~r["mask"]] = float("nan")
    return r


SIZES = [(1, 1, 1), (1, 64, 16), (3, 7, 5), (7, 1024, 4096), (8, 4096, 1024), (9, 333, 77), (16, 384, 1536),
         (17, 100, 40), (32, 2000, 130), (33, 1, 1), (33, 64, 16), (64, 1023, 47), (100, 4096, 1024),
         (127, 768, 768), (128, 128, 256), (129, 65, 257), (300, 384, 1536), (1000, 1000, 1000), (2049, 72, 264),
         (5003, 1001, 777), (12608, 384, 1536), (9000, 520, 2064)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,cols,n", SIZES)
def test_against_64_bits(T, cols, n, kind):
    check(**inputs(T, cols, n, T + cols + n, kind))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,cols,n", [(5, 200, 33), (30, 512, 96), (70, 512, 96), (70, 200, 33), (700, 320, 528),
                                      (4000, 136, 600), (4000, 160, 608)])
@pytest.mark.parametrize("bias,act,residual,dtype,keep,masked", [
    ("bf16", "gelu", False, "bf16", True, False), ("f32", "none", True, "f32", False, True),
    ("bf16", "none", True, "bf16", False, True), (None, "gelu", True, "f32", True, True),
    ("f32", "gelu", True, "bf16", False, False)])
def test_epilogue(T, cols, n, kind, bias, act, residual, dtype, keep, masked):
    check(**inputs(T, cols, n, n + T, kind, bias, residual, masked, dtype), act=act, dtype=dtype, keep=keep)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,cols,n", [(33, 4096, 64), (129, 2000, 200), (250, 4096, 1024), (600, 8192, 264),
                                      (70, 1024, 40), (40, 8000, 4096)])
@pytest.mark.parametrize("bias,act,residual,dtype,keep,masked", [
    (None, "none", False, "bf16", False, False), ("bf16", "gelu", True, "bf16", True, True),
    ("f32", "gelu", True, "f32", True, False), ("f32", "none", True, "f32", False, True)])
def test_few_rows_and_long_reductions(T, cols, n, kind, bias, act, residual, dtype, keep, masked):
    """Tiles whose reduction several CTAs share."""
    check(**inputs(T, cols, n, n + T, kind, bias, residual, masked, dtype), act=act, dtype=dtype, keep=keep)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,cols,n", [(3, 300000, 20), (3, 32768, 20), (20, 32769, 40), (50, 200000, 24), (300, 100001, 48),
                                      (2000, 70000, 264)])
def test_very_long_reductions(T, cols, n, dtype, kind):
    """All terms positive, so that what an accumulator is cut by adds up: 2^-22 of what it holds each time (as
    above), half of it on average over the accumulation. These are short, whatever the length: 512 steps of
    four 32-byte sums for a bf16 result, 2^11 cuts, 2^-12; 22 steps for fp32 ones, or 32 of the few-row kernel, 2^7 cuts,
    2^-16; an fp32 addition each, 2^-24."""
    from paper_2608_10392_gb300 import linear, linear_status
    k = inputs(T, cols, n, n, kind)
    if kind == "bf16":
        k["x"].abs_(), k["w"].abs_()
    else:
        for q in (k["x"], k["w"]):
            q.codes.view(torch.uint8).bitwise_and_(0x7f)
    got = linear(k["x"], k["w"], dtype=dtype)
    assert linear_status() == 0
    want = value(k["x"]) @ value(k["w"]).T
    bound = 2.0 ** -12 + 2.0 ** -8 if dtype == "bf16" else 2.0 ** -16 + cols / (22 * 64) * 2.0 ** -24 + 2.0 ** -20
    assert float((got.to(F64) / want - 1).abs().max()) < bound


@pytest.mark.gpu
def test_every_row_padding_and_no_rows():
    from paper_2608_10392_gb300 import linear
    for T in (4, 200):
        k = inputs(T, 64, 48, 1, bias="f32", residual=True, masked=True)
        k["mask"][:] = False
        k["x"][:] = float("nan")
        k["residual"][:] = float("inf")
        assert (check(**k, act="gelu", keep=True) == 0).all()
    w = torch.ones(48, 64, device="cuda").bfloat16()
    assert linear(torch.empty(0, 64, device="cuda").bfloat16(), w).shape == (0, 48)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 40, 900])
@pytest.mark.parametrize("cols,n,pad,shift", [(128, 64, 8, 0), (128, 64, 8, 8), (128, 64, 3, 1), (100, 36, 4, 0),
                                              (64, 48, 1, 0), (96, 80, 0, 2)])
def test_strides(T, cols, n, pad, shift):
    g = torch.Generator(device="cuda").manual_seed(T + cols)
    x, w = operand(T, cols, g, pad, shift), operand(n, cols, g, pad, shift)
    for dtype in ("bf16", "f32"):
        wide = torch.full((T, n + pad + shift), 3.0, device="cuda", dtype=TYPES[dtype])
        res = torch.randn(T, n + pad + shift, generator=g, device="cuda").to(TYPES[dtype])[:, shift:shift + n]
        check(x, w, dtype=dtype, residual=res, out=wide[:, shift:shift + n])
        assert (wide[:, :shift] == 3).all() and (wide[:, shift + n:] == 3).all()
    q = eight(T, cols, g, pad=5)
    check(q, eight(n, cols, g, pad=3))


@pytest.mark.gpu
@pytest.mark.parametrize("T,n", [(6, 48), (50, 48), (600, 77), (3000, 512)])
def test_result_in_place_of_the_residual(T, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    x, w = operand(T, 96, g), operand(n, 96, g, scale=0.1)
    res = torch.randn(T, n, generator=g, device="cuda")
    want = check(x, w, residual=res.clone(), dtype="f32", act="gelu")
    got = check(x, w, residual=res, dtype="f32", act="gelu", out=res)
    assert got.data_ptr() == res.data_ptr() and torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [6, 50, 300])
def test_one_array_for_operands_and_result(T):
    """Columns of one array side by side; what would be written while it is read is refused."""
    from paper_2608_10392_gb300 import UnifMoeError, linear
    g = torch.Generator(device="cuda").manual_seed(T)
    wide = torch.randn(T, 64 + 48 + 48, generator=g, device="cuda").bfloat16()
    w = operand(48, 64, g)
    x, res, out = wide[:, :64], wide[:, 64:112], wide[:, 112:]
    before = wide[:, :112].clone()
    want = check(x.clone(), w, residual=res.clone())
    assert torch.equal(check(x, w, residual=res, out=out), want) and torch.equal(wide[:, :112], before)
    square = operand(64, 64, g)
    for k in (dict(x=x, w=square, out=x), dict(x=x, w=square, out=wide[:, 32:96]),
              dict(x=x[1:], w=w, out=wide[:-1, 60:108]), dict(x=x, w=w, residual=wide[:, 80:128], out=out),
              dict(x=x[1:], w=w, residual=out[1:], out=out[:-1]),
              dict(x=wide[:, :32], w=wide[:4, 64:96], out=wide[:, 66:70])):
        with pytest.raises(UnifMoeError, match="overlaps"):
            linear(**k)
    assert torch.equal(wide[:, :112], before)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """More than 2^31 elements of result: the last rows are as right as the first."""
    from paper_2608_10392_gb300 import linear
    g = torch.Generator(device="cuda").manual_seed(3)
    T, n = 70000, 32768
    x, w = operand(T, 64, g), operand(n, 64, g, scale=0.125)
    out = linear(x, w)
    for rows in (slice(0, 300), slice(T - 300, T)):
        z = x[rows].to(F64) @ w.to(F64).T
        assert ((out[rows].to(F64) - z).abs() <= 2.0 ** -8 * z.abs() + 1e-5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [6, 50, 3000])
def test_other_streams_and_graphs(T):
    from paper_2608_10392_gb300 import linear, linear_backward
    k = inputs(T, 200, 120, 2, bias="bf16")
    dout = torch.randn(T, 120, device="cuda").bfloat16()

    def both(**s):
        y, z = linear(k["x"], k["w"], k["bias"], activation="gelu", keep=True, **s)
        r = linear_backward(k["x"], k["w"], dout, z, activation="gelu", bias=True, **s)
        return y, r["dx"], r["dw"], r["dbias"]

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    k["x"].copy_(k["x"].flip(0))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    again = both()
    assert all(torch.equal(a, b) for a, b in zip(held, again)) and not torch.equal(held[0], want[0])


# ------------------------------------------------------------------ gradients

def check_backward(x, w, dout, z=None, act="none", mask=None, grad_dtype="f32", **kw):
    """dz is exact to 2^-20 (GELU's derivative, at most 1.13: 2e-6 of dout), rounded by 2^-8
    where it is not dout itself; sums as above over n columns (dx) or T rows (dw)."""
    from paper_2608_10392_gb300 import linear_backward, linear_status
    r = linear_backward(x, w, dout, z, activation=act, mask=mask, bias=True, grad_dtype=grad_dtype, **kw)
    assert linear_status() == 0
    on = torch.ones(len(x), dtype=torch.bool, device="cuda") if mask is None else mask != 0
    xv, d, wv = (torch.where(on[:, None], x.to(F64), 0.0), torch.where(on[:, None], dout.to(F64), 0.0), w.to(F64))
    dz, off = d, torch.zeros_like(d)
    if act == "gelu":
        zv = torch.where(on[:, None], z.to(F64), 0.0)
        dz = d * (torch.special.ndtr(zv) + zv * torch.exp(-zv * zv / 2) / math.sqrt(2 * math.pi))
        off = 2e-6 * d.abs()
    rounded = act != "none" or dout.dtype == torch.float32
    unit = 2.0 ** -8 * dz.abs() + off if rounded else off
    T, n = d.shape

    def close(got, want, tol, kind):
        assert got.dtype == TYPES[kind] and got.shape == want.shape
        tol = tol + (2.0 ** -8 if kind == "bf16" else 2.0 ** -23) * want.abs()
        bad = ~((got.to(F64) - want).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())

    size = dz.abs() @ wv.abs()
    close(r["dx"], dz @ wv, unit @ wv.abs() + (n / 16 + 2) * 2.0 ** -22 * size, "bf16")
    size = dz.abs().T @ xv.abs()
    # an accumulation runs over at most 1,024 rows; those are added in fp32
    close(r["dw"], dz.T @ xv, unit.T @ xv.abs() + (min(T, 1024) / 16 + T / 1024 + 66) * 2.0 ** -22 * size, grad_dtype)
    close(r["dbias"], dz.sum(0), off.sum(0) + (T / 32 + 64) * 2.0 ** -24 * dz.abs().sum(0), "f32")
    return r


def grads(T, cols, n, seed, act="none", masked=False, dtype="bf16", pad=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = dict(x=operand(T, cols, g, pad, shift), w=operand(n, cols, g, pad, shift, scale=cols ** -0.5), act=act)
    k["dout"] = (0.1 * torch.randn(T, n + pad, generator=g, device="cuda")).to(TYPES[dtype])[:, :n]
    if act != "none":
        k["z"] = operand(T, n, g, pad, shift, scale=2.0)
    if masked:
        k["mask"] = torch.rand(T, generator=g, device="cuda") < 0.6
        for name in ("x", "dout", "z"):
            if name in k:
                k[name][~k["mask"]] = float("nan")
    return k


@pytest.mark.gpu
@pytest.mark.parametrize("T,cols,n", [(1, 1, 1), (1, 64, 64), (5, 33, 7), (63, 128, 256), (64, 200, 120), (65, 65, 65),
                                      (300, 384, 1536), (1000, 768, 130), (1025, 72, 264), (5003, 333, 129),
                                      (12608, 384, 1536), (20000, 1024, 512), (40000, 128, 128),
                                      (50, 512, 4096), (200, 264, 2048)])
@pytest.mark.parametrize("act,masked,grad_dtype", [("none", False, "f32"), ("gelu", True, "bf16"),
                                                   ("gelu", False, "f32"), ("none", True, "f32")])
def test_gradients(T, cols, n, act, masked, grad_dtype):
    check_backward(**grads(T, cols, n, T + n, act, masked), grad_dtype=grad_dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("T,cols,n,act", [(64, 64, 64, "none"), (1300, 200, 136, "none"), (1300, 77, 130, "gelu"),
                                          (30001, 264, 200, "none"), (70000, 64, 72, "gelu")])
def test_gradients_of_long_padding(T, cols, n, act):
    """Runs of padding that are longer than a step of the reduction, at the ends and in between; all but
    one row; masks at any address."""
    k = grads(T, cols, n, T, act, True)
    for name in ("x", "dout", "z"):
        if name in k:
            k[name].copy_(torch.randn(k[name].shape, device="cuda"))
    row = torch.arange(T, device="cuda")
    for mask in (row >= T // 2, row < T // 3, (row // 100) % 3 == 1, row == T - 1, row == 0, row % 64 == 63):
        wide = torch.zeros(T + 1, dtype=torch.bool, device="cuda")
        wide[1:] = mask
        for m in (mask, wide[1:]):
            b = dict(k, mask=m, **{name: k[name].clone() for name in ("x", "dout", "z") if name in k})
            for name in ("x", "dout", "z"):
                if name in b:
                    b[name][~m] = float("nan")
            check_backward(**b)


@pytest.mark.gpu
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 1), (1, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_strided_rows(pad, shift, dtype):
    check_backward(**grads(300, 96, 80, 1, "gelu", False, dtype, pad, shift))
    check_backward(**grads(300, 96, 80, 1, "none", True, dtype, pad, shift))


@pytest.mark.gpu
def test_gradients_of_extreme_z():
    k = grads(70, 32, 48, 1, "gelu")
    k["z"][:, :8] = torch.tensor([0.0, -0.0, 13.0, -13.0, 40.0, -40.0, 1e30, -1e30], device="cuda").bfloat16()
    check_backward(**k)
    k["z"][:, 0], k["z"][:, 1] = float("inf"), -float("inf")
    from paper_2608_10392_gb300 import linear_backward
    r = linear_backward(k["x"], k["w"], k["dout"], k["z"], activation="gelu", bias=True)
    assert torch.isfinite(r["dx"]).all() and torch.isfinite(r["dw"]).all()
    # -inf is taken as -13, where the derivative is Phi - 13 phi > -13 0.4 e^-84.5 > -2e-36;
    # 70 rows of |x| < 6 and |dout| < 1 make less than 1e-33 of it
    assert (r["dw"][1].abs() < 1e-33).all() and torch.allclose(r["dbias"][0], k["dout"][:, 0].float().sum(), rtol=1e-5)


@pytest.mark.gpu
def test_no_rows_and_all_padding():
    from paper_2608_10392_gb300 import linear_backward
    w = torch.ones(48, 64, device="cuda").bfloat16()
    r = linear_backward(torch.empty(0, 64, device="cuda").bfloat16(), w, torch.empty(0, 48, device="cuda").bfloat16(),
                        bias=True)
    assert r["dx"].shape == (0, 64) and (r["dw"] == 0).all() and (r["dbias"] == 0).all()
    k = grads(90, 64, 48, 3, "gelu", True)
    k["mask"][:] = False
    r = check_backward(**k)
    assert all((r[name] == 0).all() for name in r)


@pytest.mark.gpu
def test_only_what_is_asked_for():
    from paper_2608_10392_gb300 import linear_backward
    k = grads(200, 96, 80, 5)
    whole = check_backward(**k)
    for ask in (dict(dw=False), dict(dx=False), dict(dx=False, dw=False, bias=True), dict(dx=False, dw=False)):
        r = linear_backward(k["x"], k["w"], k["dout"], **ask)
        for name, default in (("dx", True), ("dw", True), ("bias", False)):
            got = r["dbias" if name == "bias" else name]
            if ask.get(name, default):
                assert torch.equal(got, whole["dbias" if name == "bias" else name])
            else:
                assert got is None


@pytest.mark.gpu
def test_gradients_against_differences():
    """sum(out * c) for small changes of x and w, in 64 bits: the forward and the backward
    belong together. The difference quotient of step h is off by h^2 f''' / 6, far below the
    2^-8 that dz is rounded by."""
    from paper_2608_10392_gb300 import linear, linear_backward
    g = torch.Generator(device="cuda").manual_seed(11)
    T, cols, n = 50, 40, 24
    x, w, b = operand(T, cols, g), operand(n, cols, g, scale=0.2), torch.randn(n, generator=g, device="cuda")
    c = torch.randn(T, n, generator=g, device="cuda").bfloat16()
    _, z = linear(x, w, b, activation="gelu", keep=True)
    r = linear_backward(x, w, c, z, activation="gelu", bias=True)

    def f(xv, wv, bv):
        return (gelu(xv @ wv.T + bv) * c.to(F64)).sum()

    xv, wv, bv = x.to(F64), w.to(F64), b.to(F64)
    h = 1e-4
    for name, ref, at in (("dx", xv, (3, 7)), ("dx", xv, (49, 0)), ("dw", wv, (5, 39)), ("dbias", bv, (23,))):
        d = torch.zeros_like(ref)
        d[at] = h
        args = {"dx": [d, 0, 0], "dw": [0, d, 0], "dbias": [0, 0, d]}[name]
        num = (f(xv + args[0], wv + args[1], bv + args[2]) - f(xv - args[0], wv - args[1], bv - args[2])) / (2 * h)
        # z and dz rounded by 2^-8, each term of the sum at most |c| 1.13 times its factor
        size = {"dx": (c.to(F64).abs() @ wv.abs()), "dw": (c.to(F64).abs().T @ xv.abs()),
                "dbias": c.to(F64).abs().sum(0)}[name][at]
        assert abs(float(r[name][at]) - float(num)) <= 2.0 ** -6 * float(size)


@pytest.mark.gpu
def test_results_repeat():
    k = grads(9000, 520, 264, 9, "gelu")
    a, b = check_backward(**k), check_backward(**k)
    assert all(torch.equal(a[name], b[name]) for name in a)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,H,masked", [(1, 64, 128, False), (130, 64, 136, True), (1000, 384, 1536, True)])
def test_a_dense_ffn_in_training(T, d, H, masked):
    """Norm, two products, and back, against 64 bits from end to end. Tolerances: every tensor's own,
    from those of what it is made of by absolute values (a product's error |da| |b| + |a| |db|), sums
    2^-18 of their terms (1,000 rows or 1,536 columns, cut at every 16, stay below 100 2^-22), bf16 2^-8, GELU's slope
    1.13, that of its derivative 0.8, the derivative's own 2^-16; products of two errors, each below 2^-5 of its tensor
    where that counts: 2^-4 more in all."""
    from paper_2608_10392_gb300 import BlockNorm, linear, linear_backward, linear_status
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, d, generator=g, device="cuda")
    w0 = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16()
    w1, w2 = operand(H, d, g, scale=d ** -0.5), operand(d, H, g, scale=H ** -0.5)
    b1, b2 = (0.3 * torch.randn(n, generator=g, device="cuda") for n in (H, d))
    dy = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    mask = torch.rand(T, generator=g, device="cuda") < 0.7 if masked else None
    on = torch.ones(T, 1, device="cuda", dtype=F64) if mask is None else mask[:, None].to(F64)
    if masked:
        x[~mask], dy[~mask] = float("nan"), float("nan")
    norm = BlockNorm(d, "f32", pre_norm="rms")
    f = norm.forward(x, pre_weight=w0, mask=mask, stats=True)
    h, z = linear(f["u"], w1, b1, activation="gelu", mask=mask, keep=True)
    y = linear(h, w2, b2, residual=x, mask=mask, dtype="f32")
    r2 = linear_backward(h, w2, dy, mask=mask, bias=True)
    r1 = linear_backward(f["u"], w1, r2["dx"], z, activation="gelu", mask=mask, bias=True)
    r0 = norm.backward(x, None, f, dout=dy.float(), du=r1["dx"], pre_weight=w0, mask=mask)
    assert linear_status() == 0

    e, cut = 2.0 ** -8, 2.0 ** -18
    X, D = torch.where(on > 0, x.to(F64), 0.0), torch.where(on > 0, dy.to(F64), 0.0)
    W0, W1, W2 = (t.to(F64) for t in (w0, w1, w2))
    rstd = (X.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    u = X * rstd * W0
    u_off = (e + cut) * u.abs()
    Z = (u @ W1.T + b1.to(F64)) * on
    S = (u.abs() @ W1.abs().T + b1.abs().to(F64)) * on
    z_off = u_off @ W1.abs().T + cut * S          # before it is rounded, as GELU takes it
    phi = torch.exp(-Z * Z / 2) / math.sqrt(2 * math.pi)
    G = torch.special.ndtr(Z) + Z * phi
    Hh = gelu(Z) * on
    h_off = 1.13 * z_off + (e + 2.0 ** -11) * Hh.abs()
    Y = (Hh @ W2.T + b2.to(F64) + X) * on
    y_off = h_off @ W2.abs().T + cut * (Hh.abs() @ W2.abs().T + b2.abs() + X.abs())
    dh = D @ W2
    dh_off = e * dh.abs() + cut * (D.abs() @ W2.abs())
    dz = dh * G * on
    dz_off = (1.13 * dh_off + dh.abs() * (0.8 * (z_off + e * Z.abs()) + 2.0 ** -16)) * on
    dz_as = dz_off + e * dz.abs()                 # as the products take it
    du = dz @ W1
    du_off = dz_as @ W1.abs() + e * du.abs() + cut * (dz.abs() @ W1.abs())
    n = X * rstd
    back = lambda v: rstd * (v * W0 - n * (v * W0 * n).mean(1, keepdim=True)) * on
    size = lambda v: rstd * (v * W0.abs() + n.abs() * (v * W0.abs() * n.abs()).mean(1, keepdim=True)) * on
    dx = D + back(du)
    for got, want, off in ((y, Y, y_off), (r2["dw"], D.T @ Hh, D.abs().T @ h_off + cut * (D.abs().T @ Hh.abs())),
                           (r2["dbias"], D.sum(0), cut * D.abs().sum(0)), (r2["dx"], dh, dh_off),
                           (r1["dbias"], dz.sum(0), dz_off.sum(0) + cut * dz.abs().sum(0)),
                           (r1["dw"], dz.T @ u, dz_as.T @ u.abs() + dz.abs().T @ u_off + cut * (dz.abs().T @ u.abs())),
                           (r1["dx"], du, du_off), (r0["dx"], dx, size(du_off + cut * du.abs()) + cut * D.abs()),
                           (r0["d_pre_weight"], (du * n).sum(0), ((du_off + cut * du.abs()) * n.abs()).sum(0))):
        off = off * (1 + 2.0 ** -4) + 1e-12
        bad = ~((got.to(F64) - want).abs() <= off)
        assert not bad.any(), (int(bad.sum()), float(((got.to(F64) - want).abs() / off).max()))


@pytest.mark.gpu
def test_gradients_on_streams_and_in_graphs():
    from paper_2608_10392_gb300 import linear_backward
    k = grads(1500, 200, 136, 4, "gelu", True)
    args = (k["x"], k["w"], k["dout"], k["z"])

    def run(**s):
        return linear_backward(*args, activation="gelu", mask=k["mask"], bias=True, **s)

    want = run()
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [run(stream=s) for s in (first, second, first)]  # two at once, each with its own workspace
    torch.cuda.synchronize()
    assert all(torch.equal(r[n], want[n]) for r in got for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    flip = torch.rand(1500, device="cuda") < 0.5  # another batch and another mask in the same places
    for t in (k["x"], k["dout"], k["z"]):
        t.copy_(torch.where(flip[:, None], torch.randn(t.shape, device="cuda"), float("nan")))
    k["mask"].copy_(flip)
    graph.replay()
    torch.cuda.synchronize()
    want = run()
    assert all(torch.equal(held[n], want[n]) and torch.isfinite(held[n]).all() for n in want)


# ------------------------------------------------------------------ refusals

def test_refusals():
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    p = C.c_void_p(4096)

    def call(**k):
        v = dict(rows=4, cols=64, n=8, i=1, o=1, bt=1, act=0, x=p, ld_x=64, sx=None, w=p, ld_w=64, sw=None, res=None,
                 ld_r=8, out=p, ld=8, z=None, ld_z=8, ws=None, wb=0, status=p)
        v.update(k)
        d = ops._LinearDesc(v["rows"], v["cols"], v["n"], v["i"], v["o"], v["bt"], v["act"])
        return L.unif_moe_linear_forward(C.byref(d), v["x"], v["ld_x"], v["sx"], v["w"], v["ld_w"], v["sw"], None,
                                         v["res"], v["ld_r"], None, v["out"], v["ld"], v["z"], v["ld_z"], v["ws"],
                                         v["wb"], v["status"], None)

    for k in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(n=0), dict(cols=(1 << 24) + 1), dict(i=0),
              dict(i=3), dict(o=2), dict(bt=2), dict(act=2), dict(act=-1), dict(x=None), dict(w=None),
              dict(out=None), dict(status=None), dict(sx=p), dict(sw=p), dict(ld_x=63), dict(ld_w=63), dict(ld=7),
              dict(res=p, ld_r=7), dict(z=p, ld_z=7)):
        assert call(**k) == -1, k
    # rows that start off 16 bytes need a workspace
    odd = dict(rows=100, cols=63, ld_x=63)
    assert call(**odd) == -3 and call(**odd, ws=C.c_void_p(4100), wb=1 << 20) == -1
    assert call(rows=0, x=None) == 0
    d = ops._LinearDesc(100, 63, 8, 1, 1, 1, 0)
    assert L.unif_moe_linear_workspace(C.byref(d), p, 63, p, 64) >= 100 * 64 * 2
    assert L.unif_moe_linear_workspace(C.byref(d), p, 64, p, 64) == 0
    assert L.unif_moe_linear_workspace(None, p, 64, p, 64) == -1

    def back(**k):
        v = dict(i=1, rows=4, act=0, x=p, w=p, dout=p, z=None, ld_x=64, ld_w=64, ld_dout=8, ld_z=8, dt=1, gt=0, dx=p,
                 ld_dx=64, dw=p, ld_dw=64)
        v.update(k)
        d = ops._LinearDesc(v["rows"], 64, 8, v["i"], 1, 1, v["act"])
        g = ops._LinearGrad(v["x"], v["w"], v["dout"], v["z"], v["ld_x"], v["ld_w"], v["ld_dout"], v["ld_z"], v["dt"],
                            v["gt"], None, v["dx"], v["ld_dx"], v["dw"], v["ld_dw"], None)
        return L.unif_moe_linear_backward(C.byref(d), C.byref(g), None, 0, None, None)

    for k in (dict(i=2), dict(act=1), dict(x=None), dict(w=None), dict(dout=None), dict(dt=2), dict(gt=2),
              dict(ld_x=63), dict(ld_w=63), dict(ld_dout=7), dict(act=1, z=p, ld_z=7), dict(ld_dx=63),
              dict(ld_dw=63), dict(rows=-1), dict()):  # (the last: no status word)
        assert back(**k) == -1, k
    x = torch.zeros(4, 64).bfloat16()
    with pytest.raises(ValueError, match="x: need a CUDA tensor"):
        pkg.linear(x, x)
    with pytest.raises(ValueError, match="both in 8 bits"):
        pkg.linear(x, pkg.Fp8(x, x))
    with pytest.raises(KeyError):
        pkg.linear(x, x, activation="tanh")


@pytest.mark.gpu
def test_refusals_of_tensors():
    import paper_2608_10392_gb300 as pkg
    x, w = torch.zeros(4, 64, device="cuda").bfloat16(), torch.zeros(8, 64, device="cuda").bfloat16()
    for bad in (dict(bias=torch.zeros(7, device="cuda")), dict(bias=torch.zeros(8, device="cuda").half()),
                dict(residual=torch.zeros(4, 8, device="cuda")), dict(mask=torch.ones(3, device="cuda") > 0),
                dict(out=torch.zeros(4, 8, device="cuda")), dict(bias=torch.zeros(8))):
        with pytest.raises(ValueError):
            pkg.linear(x, w, **bad)
    with pytest.raises(ValueError, match="w:"):
        pkg.linear(x, w[:, :63])
    with pytest.raises(ValueError, match="z: the gradient"):
        pkg.linear_backward(x, w, torch.zeros(4, 8, device="cuda").bfloat16(), activation="gelu")


PLACES = {name: (i + 1) << 28 for i, name in enumerate(("x", "w", "sx", "sw", "bias", "res", "mask", "out", "z", "ws",
                                                          "status"))}


def test_results_over_operands_are_refused():
    """out and z over each other and over everything else of the call, whole or by their ends. (Made-up
    addresses: each call is refused before anything is launched.)"""
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()

    def refused(eight=False, cols=64, ld_x=64, ld_res=64, bytes_=0, **moved):
        at = {**PLACES, **moved}
        d = ops._LinearDesc(100, cols, 64, 2 if eight else 1, 1, 0, 1)
        rc = L.unif_moe_linear_forward(
            C.byref(d), at["x"], ld_x, at["sx"] if eight else None, at["w"], 64, at["sw"] if eight else None, at["bias"],
            at["res"], ld_res, at["mask"], at["out"], 64, at["z"], 64, at["ws"] if bytes_ else None, bytes_, at["status"],
            None)
        return rc == -1 and b"overlaps" in L.unif_moe_last_error()

    size = dict(x=12800, w=8192, sx=400, sw=256, bias=256, res=12800, mask=100, out=12800, z=12800, status=4)
    for result in ("out", "z"):
        for name in size:
            eight = name in ("sx", "sw")
            for shift in (0, -12800 + 2, (size[name] - 1) // 2 * 2):
                if name != result and not (result == "out" and name == "res" and shift == 0):  # (in its place)
                    assert refused(eight, **{result: PLACES[name] + shift}), (result, name, shift)
        # the workspace of rows that are laid out first
        assert refused(cols=63, ld_x=63, bytes_=1 << 20, **{result: PLACES["ws"] + 6400})
    assert refused(out=PLACES["res"], ld_res=72)  # the residual's place, with another stride


def backward_description(ops, at, act=1, rows=100, cols=64, n=64, gt=0, ld_x=64, **ask):
    """(descriptions of a backward of the arrays `at`; with ask[name] False that result is not asked for)"""
    d = ops._LinearDesc(rows, cols, n, 1, 1, 0, act)
    want = {name: at[name] if ask.get(name, True) else None for name in ("dx", "dw", "dbias")}
    return d, ops._LinearGrad(at["x"], at["w"], at["dout"], at["z"], ld_x, 64, 64, 64, 1, gt, at["mask"], want["dx"], 64,
                              want["dw"], 64, want["dbias"])


def test_gradients_over_operands_are_refused():
    """dx, dw and dbias over each other and over all that the call reads, whole or by their ends. (Made-up
    addresses: each call is refused before anything is launched.)"""
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    size = dict(x=12800, w=8192, dout=12800, z=12800, mask=100, dx=12800, dw=16384, dbias=256, status=4)
    places = {name: (i + 1) << 28 for i, name in enumerate(size)}
    for result in ("dx", "dw", "dbias"):
        for name in size:
            for shift in (0, -size[result] + 4, (size[name] - 1) // 4 * 4):
                if name == result:
                    continue
                at = {**places, result: places[name] + shift}
                d, g = backward_description(ops, at)
                assert L.unif_moe_linear_backward(C.byref(d), C.byref(g), None, 0, at["status"], None) == -1
                assert b"overlaps" in L.unif_moe_last_error(), (result, name, shift)


@pytest.mark.gpu
def test_gradients_over_what_is_not_read():
    """dx in the place of x without dw, dw in that of w without dx, dbias in that of z without an activation; over
    the workspace they are refused."""
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    k = grads(100, 64, 64, 3)
    x, w, dout = k["x"].contiguous(), k["w"].contiguous(), k["dout"].contiguous()
    want = pkg.linear_backward(x, w, dout, grad_dtype="bf16", bias=True)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for ask in (dict(dw=False), dict(dx=False), dict(dx=False, dw=False)):
        to = dict(x=x.clone(), w=w.clone(), dout=dout, z=torch.zeros(100, 64, device="cuda").bfloat16())
        place = dict(dx=to["x"], dw=to["w"], dbias=to["z"])
        at = {n: t.data_ptr() for n, t in to.items()}
        at.update({n: t.data_ptr() for n, t in place.items()}, mask=None)
        d, gr = backward_description(ops, at, act=0, gt=1, **ask)
        need = L.unif_moe_linear_backward_workspace(C.byref(d), C.byref(gr))
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        assert L.unif_moe_linear_backward(C.byref(d), C.byref(gr), ws.data_ptr(), need, status.data_ptr(),
                                          torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert int(status) == 0
        for name in ("dx", "dw"):
            if ask.get(name, True):
                assert torch.equal(place[name], want[name])
        assert torch.equal(place["dbias"].view(torch.float32).flatten()[:64], want["dbias"])
        d, gr = backward_description(ops, {**at, "dbias": ws.data_ptr()}, act=0, gt=1, **ask)
        assert need > 0 and L.unif_moe_linear_backward(C.byref(d), C.byref(gr), ws.data_ptr(), need, status.data_ptr(),
                                                       None) == -1
        assert b"overlaps" in L.unif_moe_last_error()


@pytest.mark.gpu
def test_columns_of_one_array_for_all_of_a_call():
    """What lies side by side is not refused: x, residual, out and z as columns of one array."""
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    g = torch.Generator(device="cuda").manual_seed(8)
    T = 200
    wide = torch.randn(T, 64 + 48 * 3, generator=g, device="cuda").bfloat16()
    x, res, out, z = wide[:, :64], wide[:, 64:112], wide[:, 112:160], wide[:, 160:]
    w, status = operand(48, 64, g), torch.zeros(1, dtype=torch.int32, device="cuda")
    want, z_want = pkg.linear(x.clone(), w, residual=res.clone(), activation="gelu", keep=True)
    before = wide[:, :112].clone()
    d = ops._LinearDesc(T, 64, 48, 1, 1, 1, 1)
    p = lambda t: t.data_ptr()  # noqa: E731
    need = pkg.lib().unif_moe_linear_workspace(C.byref(d), p(x), 208, p(w), 64)
    assert need == 0
    for to in (out, res):  # (the last: in place of the residual)
        assert pkg.lib().unif_moe_linear_forward(
            C.byref(d), p(x), 208, None, p(w), 64, None, None, p(res), 208, None, p(to), 208, p(z), 208, None, 0,
            p(status), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(to, want) and torch.equal(z, z_want) and int(status) == 0
        assert torch.equal(wide[:, :64], before[:, :64])
        if to is out:
            assert torch.equal(res, before[:, 64:])


@pytest.mark.gpu
@pytest.mark.parametrize("T,cols,n", [(5, 64, 64), (70, 64, 48), (300, 200, 136), (300, 77, 130), (3000, 512, 256),
                                      (64, 64, 4096)])
@pytest.mark.parametrize("act,dtype", [("none", "bf16"), ("none", "f32"), ("gelu", "bf16")])
def test_padding_rows_under_weights_that_are_not_finite(T, cols, n, act, dtype):
    """An infinity or NaN of the weights reaches dx of every row but padding, whose dx is 0 whether or not dz
    is laid out first; dw and dbias do not read the weights."""
    from paper_2608_10392_gb300 import linear, linear_backward, linear_status
    k = grads(T, cols, n, T + n, act, True, dtype)
    k["mask"][0], k["mask"][-1] = False, True
    for name in ("x", "dout", "z"):
        if name in k:
            k[name][0], k[name][-1] = float("nan"), 0.5
    ask = dict(activation=act, mask=k["mask"], bias=True)
    want = linear_backward(k["x"].nan_to_num(), k["w"], k["dout"].nan_to_num(), k["z"].nan_to_num() if "z" in k else None, **ask)
    w = k["w"].clone()
    w[3, 2], w[n // 2, cols - 1], w[n - 1, 0] = float("inf"), -float("inf"), float("nan")
    r = linear_backward(k["x"], w, k["dout"], k.get("z"), **ask)
    out = linear(k["x"], w, mask=k["mask"], dtype="f32")
    assert linear_status() == 0
    pad = ~k["mask"]
    assert (r["dx"][pad] == 0).all() and (out[pad] == 0).all()
    assert torch.equal(r["dw"], want["dw"]) and torch.equal(r["dbias"], want["dbias"])
    assert r["dx"][k["mask"]][:, 0].isnan().all()
    same = torch.ones(cols, dtype=torch.bool, device="cuda")
    same[[0, 2, cols - 1]] = False
    assert torch.equal(r["dx"][:, same], want["dx"][:, same])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "dx"])
def test_what_accumulations_lose_on_average(kind):
    """2^20 positive terms a sum, into bf16, in tiles whose reduction no CTAs share. Rounding is as often up as
    down, the cuts of an accumulator all go one way: the mean of the signed errors shows them. A cut loses at most
    2^-22 of what is held (as above), over an accumulation half of its sum is held on average: 2^11 cuts (512 steps
    of four) lose at most 2^11 2^-22 / 2 = 2^-12. In one unbroken accumulation there are 2^16 cuts (8 bits: 2^15), 32 (16)
    times as many. Of 128 x 128 results, spread over their binade by the scales of rows and channels, the mean of
    roundings by 2^-8 at most (2^-8 / sqrt(3) each) stays within five of its deviations, 2^-8 / sqrt(3) / 128."""
    from paper_2608_10392_gb300 import linear, linear_backward, linear_status
    g = torch.Generator(device="cuda").manual_seed(20)
    long, T, n, few = 1 << 20, 1280, 2048, 128

    def rows(count):
        if kind == "e4m3":
            q = eight(count, long, g)
            q.codes.view(torch.uint8).bitwise_and_(0x7f)
            return q
        r = torch.randn(count, long, generator=g, device="cuda").abs_()
        return r.mul_(1 + torch.rand(count, 1, generator=g, device="cuda")).bfloat16()

    def some(q, step):
        return value(type(q)(q.codes[::step], q.scales[::step]) if kind == "e4m3" else q[::step])

    x, w = rows(T), rows(n)
    want = some(x, T // few) @ some(w, n // few).T
    if kind == "dx":
        got = linear_backward(torch.empty(T, n, device="cuda").bfloat16(), w.T.contiguous(), x, dw=False)["dx"]
    else:
        got = linear(x, w)
    assert linear_status() == 0
    loss = 1 - got[::T // few, ::n // few].to(F64) / want
    assert loss.shape == (few, few) and float(loss.abs().max()) < 2.0 ** -8 + 2.0 ** -11
    assert abs(float(loss.mean())) < 2.0 ** -12 + 5 * 2.0 ** -8 / 3 ** 0.5 / few, float(loss.mean())
