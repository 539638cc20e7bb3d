"""Rows in 8-bit floating point: fp8_quantize and fp8_dequantize equal the definition in 64 bits
bit for bit (scaling by a power of two is exact), BlockNorm with u in 8 bits lies within half a
step of the 64-bit u; the run norm -> product -> 8 bits -> product; refusals."""
import ctypes as C
import math

import pytest
import torch

F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def levels():
    """The values 0 .. 448 of the codes 0x00 .. 0x7e."""
    c = torch.arange(127, dtype=torch.int64)
    e, m = c >> 3, (c & 7).to(F64)
    return torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.to(F64) - 10))


def reference(x):
    """(codes [rows][cols] uint8, scales [rows] fp32): the scale by trying every power of two,
    the nearest value, ties to the even code."""
    x = x.to(F64).cpu()
    scales = torch.zeros(len(x), dtype=torch.float32)
    codes = torch.zeros(x.shape, dtype=torch.uint8)
    lv = levels()
    mid = (lv[1:] + lv[:-1]) / 2
    for r, row in enumerate(x):
        if not torch.isfinite(row).all():
            scales[r] = math.nan
            continue
        e = next(e for e in range(-126, 128) if row.abs().max() <= 448 * 2.0 ** e)
        scales[r] = 2.0 ** e
        m = row.abs() / 2.0 ** e
        up, down = torch.bucketize(m, mid, right=True), torch.bucketize(m, mid)
        code = torch.where(up % 2 == 0, up, down)
        codes[r] = torch.where(torch.signbit(row), code + 128, code).to(torch.uint8)
    return codes, scales


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float().cpu(), nan=77.0), torch.nan_to_num(b.float().cpu(), nan=77.0))


def check(x, **kw):
    from paper_2608_10392_gb300 import fp8_dequantize, fp8_quantize
    q = fp8_quantize(x, **kw)
    codes, scales = reference(x)
    assert q.codes.shape == x.shape and torch.equal(q.codes.contiguous().view(torch.uint8).cpu(), codes)
    assert same(q.scales, scales)
    table = torch.cat([levels(), torch.tensor([math.nan], dtype=F64)])
    table = torch.cat([table, -table])
    want = table[codes.long()] * scales.to(F64)[:, None]
    for name, dt in TYPES.items():
        got = fp8_dequantize(q, dtype=name)
        assert got.dtype == dt and same(got, want.to(dt))
    return q


def data(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    return x.to(dtype).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 31), (5, 33), (17, 64), (2, 256), (9, 257), (33, 384),
                                       (7, 1000), (130, 1024), (3, 1025), (5, 1032), (4, 8192), (2, 8200), (2, 8191),
                                       (1, 100000), (1200, 96)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_codes_scales_and_values(rows, cols, dtype):
    check(data(rows, cols, dtype, rows + cols))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_every_level_tie_and_border(dtype):
    """Rows whose largest value is 448, just above, 256 and just below, with every level and
    every middle of two; all signs."""
    lv = levels()
    v = torch.cat([lv, (lv[1:] + lv[:-1]) / 2])
    v = torch.cat([v, -v])
    rows = [torch.cat([v[v.abs() <= top], torch.tensor([top], dtype=F64), torch.zeros(600 - int((v.abs() <= top).sum()),
                                                                                       dtype=F64)]) * 2.0 ** e
            for top in (448.0, 450.0, 256.0, 255.0, 224.0, 225.0) for e in (-20, 0, 9)]
    check(torch.stack(rows).to(dtype).cuda())


@pytest.mark.gpu
def test_extreme_rows():
    x = torch.zeros(9, 40, device="cuda")
    x[1, 3], x[2, 0], x[3, 39], x[4, 5] = math.inf, -math.inf, math.nan, 3.4e38
    x[5, 7], x[6, 7], x[7] = 1e-45, 1e-38, -0.0
    x[8, 0], x[8, 1] = 1e38, 1e-38
    q = check(x)
    assert float(q.scales[0]) == 2.0 ** -126


@pytest.mark.gpu
@pytest.mark.parametrize("pad,shift", [(8, 0), (16, 8), (3, 1), (1, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides_and_given_outputs(pad, shift, dtype):
    from paper_2608_10392_gb300 import Fp8, fp8_dequantize, fp8_quantize
    wide = data(21, 72 + pad + shift, dtype, pad)
    x = wide[:, shift:shift + 72]
    codes = torch.zeros(21, 72 + pad + shift, device="cuda", dtype=torch.uint8)
    out = Fp8(codes.view(torch.float8_e4m3fn)[:, shift:shift + 72], torch.empty(21, device="cuda"))
    assert fp8_quantize(x, out=out) is out
    want = check(x.contiguous())
    assert torch.equal(out.codes.contiguous().view(torch.uint8), want.codes.contiguous().view(torch.uint8))
    assert (codes[:, :shift] == 0).all() and (codes[:, shift + 72:] == 0).all()
    back = torch.full((21, 72 + pad + shift), 5.0, device="cuda")
    fp8_dequantize(out, dtype="f32", out=back[:, shift:shift + 72])
    assert same(back[:, shift:shift + 72], fp8_dequantize(want, dtype="f32"))
    assert (back[:, :shift] == 5).all() and (back[:, shift + 72:] == 5).all()


@pytest.mark.gpu
def test_more_dimensions_and_no_rows():
    from paper_2608_10392_gb300 import fp8_dequantize, fp8_quantize
    x = data(24, 50, torch.bfloat16)
    q, want = fp8_quantize(x.view(2, 3, 4, 50)), fp8_quantize(x)
    assert q.codes.shape == (2, 3, 4, 50) and q.scales.shape == (2, 3, 4)
    assert same(fp8_dequantize(q).view(24, 50), fp8_dequantize(want))
    e = fp8_quantize(x[:0])
    assert e.codes.shape == (0, 50) and fp8_dequantize(e).shape == (0, 50)


# ------------------------------------------------------------------ norms

EPS = 1e-5


def norm64(v, kind, w, b):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS) * w
    return v if b is None else v + b


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(1, 1), (3, 48), (40, 64), (9, 100), (17, 128), (5, 250), (33, 256), (300, 384),
                                 (7, 1000), (4, 1001), (130, 1024), (2500, 1024), (2440, 264), (3, 2048), (2, 8192)])
@pytest.mark.parametrize("stream,branch,post,pre,bias,masked", [
    ("f32", "bf16", "rms", "rms", False, False), ("bf16", "bf16", "none", "layer", True, True),
    ("f32", "f32", "layer", "rms", True, True), ("bf16", "bf16", "layer", "rms", False, False)])
def test_norm_with_8_bit_rows(T, d, stream, branch, post, pre, bias, masked):
    """u of the kernel is fp32, within 2e-5 of the size of its terms (tests/test_gpu_block_norm.py
    derives it), then rounded by half a step: 2^-4 of itself, or 2^-10 of the scale below
    2^-6 of it. The scale is the 64-bit one but where the row's largest value is that close to its
    border. out and the statistics are those of the norm without 8 bits, bit for bit."""
    from paper_2608_10392_gb300 import BlockNorm, fp8_dequantize
    g = torch.Generator().manual_seed(T + d)

    def r(*shape, dtype, k=1.0, m=0.0):
        return (torch.randn(*shape, generator=g) * k + m).to(TYPES[dtype]).cuda()

    x, y = r(T, d, dtype=stream, m=0.3), r(T, d, dtype=branch, k=0.8)
    p = dict(gate=r(1, d, dtype=branch, k=0.5), pre_weight=r(d, dtype=branch, k=0.2, m=1.0))
    if bias:
        p["pre_bias"] = r(d, dtype=branch, k=0.2)
    if post != "none":
        p["post_weight"] = r(d, dtype=branch, k=0.2, m=1.0)
    mask = None
    if masked:
        mask = (torch.rand(T, generator=g) < 0.6).cuda()
        x[~mask] = y[~mask] = float("nan")
    kw = dict(stream_dtype=stream, branch_dtype=branch, post_norm=post, pre_norm=pre, eps=EPS, res_scale=0.75)
    got = BlockNorm(d, u_format="fp8", **kw).forward(x, y, mask=mask, stats=True, **p)
    plain = BlockNorm(d, **kw).forward(x, y, mask=mask, stats=True, **p)
    for k in ("out", "post_mean", "post_rstd", "pre_mean", "pre_rstd"):
        assert (got[k] is None) == (plain[k] is None)
        assert got[k] is None or torch.equal(got[k], plain[k]), k
    on = torch.ones(T, dtype=torch.bool, device="cuda") if mask is None else mask
    q = {k: v.to(F64) for k, v in p.items()}
    z = y[on].to(F64)
    if post != "none":
        z = norm64(z, post, q["post_weight"], None)
    o = 0.75 * x[on].to(F64) + q["gate"] * z
    u = norm64(o, pre, q["pre_weight"], q.get("pre_bias"))
    tol = 2e-5 * (1 + u.abs() + o.abs() / torch.sqrt(o.square().mean(1, keepdim=True) + EPS))
    if d == 1 and pre == "layer":
        tol = tol + 1e-3  # (a variance of 0: rounding alone, by 1 / sqrt(eps))
    scale = got["u"].scales[on].to(F64)
    low, high = (torch.exp2(torch.ceil(torch.log2((u.abs() + s * tol).amax(1).clamp(min=1e-60) / 448)).clamp(min=-126))
                 for s in (-1, 1))
    assert ((scale >= low) & (scale <= high)).all()
    v = fp8_dequantize(got["u"], dtype="f32").to(F64)
    step = torch.maximum(2.0 ** -4 * u.abs(), 2.0 ** -10 * scale[:, None])
    assert ((v[on] - u).abs() <= step + 1.1 * tol).all()
    assert (v[~on] == 0).all() and (got["u"].codes.view(torch.uint8)[~on] == 0).all()


@pytest.mark.gpu
def test_norm_alone_strided_and_into_given_rows():
    """The norm before a stack's first block (no y), strided x, given codes."""
    from paper_2608_10392_gb300 import BlockNorm, Fp8, fp8_dequantize
    g = torch.Generator(device="cuda").manual_seed(4)
    for d, pad, shift in ((96, 8, 0), (96, 3, 1), (333, 0, 2)):
        x = torch.randn(50, d + pad + shift, generator=g, device="cuda")[:, shift:shift + d]
        w = torch.ones(d, device="cuda").bfloat16()
        codes = torch.zeros(50, d + pad + shift, device="cuda", dtype=torch.uint8)
        u = Fp8(codes.view(torch.float8_e4m3fn)[:, shift:shift + d], torch.empty(50, device="cuda"))
        n = BlockNorm(d, stream_dtype="f32", u_format="fp8")
        r = n.forward(x, u=u, pre_weight=w)
        want = n.forward(x.contiguous(), pre_weight=w)
        assert r["u"].codes.data_ptr() == u.codes.data_ptr() and same(fp8_dequantize(u), fp8_dequantize(want["u"]))
        assert (codes[:, :shift] == 0).all() and (codes[:, shift + d:] == 0).all()


@pytest.mark.gpu
def test_norm_of_rows_that_are_not_finite():
    from paper_2608_10392_gb300 import BlockNorm
    x = torch.ones(6, 400, device="cuda").bfloat16()
    x[2, 7], x[4, 0] = math.nan, math.inf
    r = BlockNorm(400, u_format="fp8").forward(x, pre_weight=torch.ones(400, device="cuda").bfloat16())
    bad = torch.isnan(r["u"].scales)
    assert bad.tolist() == [False, False, True, False, True, False]
    assert (r["u"].codes.view(torch.uint8)[bad] == 0).all()


# ------------------------------------------------------------------ together

@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 200])
def test_a_dense_ffn_in_8_bits(T):
    """norm -> 8-bit rows -> up with GELU -> 8-bit rows -> down onto the stream, against the same
    steps in 64 bits from the codes that the run produced: each product's own tolerance
    (tests/test_gpu_linear.py)."""
    from paper_2608_10392_gb300 import BlockNorm, fp8_dequantize, fp8_quantize, linear, linear_status
    g = torch.Generator(device="cuda").manual_seed(7)
    d, H = 256, 640
    x = torch.randn(T, d, generator=g, device="cuda")
    y = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    up = fp8_quantize(torch.randn(H, d, generator=g, device="cuda") * d ** -0.5)
    down = fp8_quantize(torch.randn(d, H, generator=g, device="cuda") * H ** -0.5)
    b1 = torch.randn(H, generator=g, device="cuda") * 0.1
    norm = BlockNorm(d, stream_dtype="f32", pre_norm="rms", u_format="fp8")
    r = norm.forward(x, y, pre_weight=torch.ones(d, device="cuda").bfloat16())
    h = linear(r["u"], up, b1, activation="gelu")
    hq = fp8_quantize(h)
    out = linear(hq, down, residual=r["out"], dtype="f32")
    assert linear_status() == 0

    def val(q):
        return q.codes.to(F64) * q.scales.to(F64)[:, None]

    z = val(r["u"]) @ val(up).T + b1.to(F64)
    want = z * torch.special.ndtr(z)
    size = val(r["u"]).abs() @ val(up).abs().T + b1.abs().to(F64)
    assert ((h.to(F64) - want).abs() <= 1.13 * (d / 32 + 6) * 2.0 ** -22 * size + (2.0 ** -8 + 2.0 ** -11) * want.abs()).all()
    want = r["out"].to(F64) + val(hq) @ val(down).T
    size = r["out"].abs().to(F64) + val(hq).abs() @ val(down).abs().T
    assert ((out.to(F64) - want).abs() <= (H / 32 + 8) * 2.0 ** -22 * size).all()
    # the whole run against 64 bits without any 8-bit step: rows and weights rounded by 2^-4 at
    # most, four times in a row; 2^-4 sqrt(4) of the branch's norm is far above their random sum
    o = x.to(F64) + y.to(F64)
    u = o / torch.sqrt(o.square().mean(1, keepdim=True) + 1e-6)
    full = o + (lambda t: t * torch.special.ndtr(t))(u @ val(up).T + b1.to(F64)) @ val(down).T
    assert float((out.to(F64) - full).norm() / (full - o).norm()) < 2.0 ** -3
    assert fp8_dequantize(hq).shape == (T, H)


@pytest.mark.gpu
def test_streams_and_graphs():
    from paper_2608_10392_gb300 import BlockNorm, fp8_dequantize, fp8_quantize
    x = data(300, 384, torch.bfloat16)
    w = torch.ones(384, device="cuda").bfloat16()
    norm = BlockNorm(384, u_format="fp8")

    def run(**s):
        q = fp8_quantize(x, **s)
        u = norm.forward(x, pre_weight=w, **s)["u"]
        return fp8_dequantize(q, **s), fp8_dequantize(u, dtype="f32", **s)

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b.flip(0)) for a, b in zip(held, want))


# ------------------------------------------------------------------ refusals

def test_refusals():
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    p = C.c_void_p(4096)

    def quantize(**k):
        v = dict(x=p, dt=1, rows=4, cols=64, ld=64, codes=p, ldc=64, scales=p)
        v.update(k)
        return L.unif_moe_fp8_quantize(v["x"], v["dt"], v["rows"], v["cols"], v["ld"], v["codes"], v["ldc"],
                                       v["scales"], None)

    def dequantize(**k):
        v = dict(x=p, dt=1, rows=4, cols=64, ld=64, codes=p, ldc=64, scales=p)
        v.update(k)
        return L.unif_moe_fp8_dequantize(v["codes"], v["ldc"], v["scales"], v["rows"], v["cols"], v["x"], v["dt"],
                                         v["ld"], None)

    for call in (quantize, dequantize):
        for k in (dict(x=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(rows=1 << 31), dict(cols=0),
                  dict(cols=(1 << 24) + 1), dict(dt=2), dict(ld=63), dict(ldc=63)):
            assert call(**k) == -1, k
        assert call(rows=0, x=None) == 0

    def norm(**k):
        v = dict(T=4, d=64, pre=2, x=p, u=p, ld_u=64, scales=p)
        v.update(k)
        desc = ops._BlockNormDesc(v["T"], v["d"], 1, 1, 0, v["pre"], 0, 1.0, 1e-6)
        return L.unif_moe_block_norm_forward_fp8(C.byref(desc), v["x"], 64, None, 64, None, None, None, None, p, None,
                                                 None, 64, v["u"], v["ld_u"], v["scales"], None, None, None, None, None)

    for k in (dict(pre=0), dict(scales=None), dict(u=None), dict(ld_u=63), dict(x=None)):
        assert norm(**k) == -1, k
    assert norm(T=0) == 0 and norm(d=8193, ld_u=8193) == -2
    with pytest.raises(ValueError, match="u_format"):
        pkg.BlockNorm(64, u_format="int8")
    with pytest.raises(ValueError, match="x: need a CUDA tensor"):
        pkg.fp8_quantize(torch.zeros(2, 2))


@pytest.mark.gpu
def test_refusals_of_tensors():
    import paper_2608_10392_gb300 as pkg
    x = torch.zeros(4, 64, device="cuda")
    q = pkg.fp8_quantize(x)
    for bad in (pkg.Fp8(q.codes[:, :32], q.scales), pkg.Fp8(q.codes[:3], q.scales), pkg.Fp8(q.codes, q.scales[:3]),
                pkg.Fp8(q.codes.view(torch.uint8), q.scales), pkg.Fp8(q.codes, None), pkg.Fp8(q.codes.T, q.scales)):
        with pytest.raises(ValueError):
            pkg.fp8_quantize(x, out=bad)
    for bad in (pkg.Fp8(q.codes, q.scales.double()), pkg.Fp8(q.codes[:, ::2], q.scales), pkg.Fp8(x, q.scales)):
        with pytest.raises(ValueError):
            pkg.fp8_dequantize(bad)
    with pytest.raises(ValueError, match="pre norm"):
        pkg.BlockNorm(64, stream_dtype="f32", post_norm="rms", pre_norm="none", u_format="fp8").forward(
            x, x.bfloat16(), post_weight=torch.ones(64, device="cuda").bfloat16())
    with pytest.raises(ValueError):
        pkg.linear(q, pkg.Fp8(q.codes, None))


def test_arrays_that_overlap_are_refused():
    """Codes or scales over the rows, whole or by their ends, in all three calls. (Made-up addresses: each
    call is refused before anything is launched.)"""
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    from paper_2608_10392_gb300 import operators as ops
    L = pkg.lib()
    T, d = 100, 64
    places = {name: (i + 1) << 28 for i, name in enumerate(("x", "y", "out", "codes", "scales", "mask"))}

    def calls(at, dt, norm):
        if not norm:
            yield L.unif_moe_fp8_quantize(at["x"], dt, T, d, d, at["codes"], d, at["scales"], None)
            yield L.unif_moe_fp8_dequantize(at["codes"], d, at["scales"], T, d, at["x"], dt, d, None)
        desc = ops._BlockNormDesc(T, d, dt, dt, 0, 2, 0, 1.0, 1e-6)
        yield L.unif_moe_block_norm_forward_fp8(C.byref(desc), at["x"], d, at["y"], d, at["mask"], None, None, None,
                                                0x70000000, None, at["out"], d, at["codes"], d, at["scales"], None, None,
                                                None, None, None)

    for dt, rows in ((0, T * d * 4), (1, T * d * 2)):
        size = dict(x=rows, y=rows, out=rows, codes=T * d, scales=4 * T, mask=T)
        for result in ("codes", "scales"):
            for name in size:
                for shift in (0, -((size[result] - 1) // 4 * 4), (size[name] - 1) // 4 * 4):
                    if name == result:
                        continue
                    at = {**places, result: places[name] + shift}
                    for rc in calls(at, dt, name in ("y", "out", "mask")):
                        assert rc == -1 and b"overlap" in L.unif_moe_last_error(), (dt, result, name, shift)


@pytest.mark.gpu
def test_codes_and_rows_side_by_side():
    """Rows and their codes as columns of one array."""
    from paper_2608_10392_gb300 import Fp8, UnifMoeError, fp8_dequantize, fp8_quantize
    wide = torch.zeros(50, 3 * 64, device="cuda").bfloat16()
    wide[:, :64] = data(50, 64, torch.bfloat16)
    x, want = wide[:, :64], check(wide[:, :64].contiguous())
    codes = wide.view(torch.float8_e4m3fn)[:, 128:192]
    out = fp8_quantize(x, out=Fp8(codes, torch.empty(50, device="cuda")))
    assert same(out.codes, want.codes) and same(out.scales, want.scales)
    back = fp8_dequantize(out, out=wide[:, 128:])
    assert same(back, fp8_dequantize(want)) and same(wide[:, :64], x)
    for bad in (wide.view(torch.float8_e4m3fn)[:, :64], wide.view(torch.float8_e4m3fn)[:, 127:191]):
        with pytest.raises(UnifMoeError, match="overlap"):
            fp8_quantize(x, out=Fp8(bad, out.scales))
