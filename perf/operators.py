"""The operators round the UniF-MoE layer, as cases to be measured.

Five calls: "norm_forward" and "norm_backward" (the norms after and before a
block, fused with the block's gate and the scaled residual sum), "balance"
(the router's balance and z losses with per-expert counts and the gradient of
the logits), "quantize" (rows to microscaled 4-bit floating point and back) and
"product" (4-bit rows, grouped by expert or by (expert, block), with 4-bit
weights). Sizes are those of the layers in the workloads package: tokens of
DeiT-S, ViT-B and BERT batches, widths 384, 768 and 1,024, 4 to 32 experts, 8
or 16 blocks; each call has a plain form in elementary torch operations.
"""
import math

import torch

own = False

F32, BF16 = torch.float32, torch.bfloat16
TYPES = {"f32": F32, "bf16": BF16}


# ------------------------------------------------------------------- cases

def _norm(name, call, T, d, stream, branch, post, pre, gate_rows, bias, padded, scale=1.0):
    """gate_rows: tokens that share a gate row (-1: no gate, 0: all of them)."""
    return dict(name=name, call=call, T=T, d=d, stream=stream, branch=branch, post=post, pre=pre,
                gate_rows=gate_rows, bias=bias, padded=padded, scale=scale)


def _balance(name, T, K, dtype, shared, top, padded):
    """shared: the logits are columns 1..K of [T][K + 1]; top: experts a token
    takes (0: its own number of them)."""
    return dict(name=name, call="balance", T=T, K=K, dtype=dtype, shared=shared, top=top,
                padded=padded)


def _quantize(name, rows, cols, dtype):
    return dict(name=name, call="quantize", rows=rows, cols=cols, dtype=dtype)


def _product(name, rows, groups, n, cols, act, dtype):
    return dict(name=name, call="product", rows=rows, groups=groups, n=n, cols=cols, act=act,
                dtype=dtype)


def listed():
    return [
        # eight single tokens of a server between two blocks of the wide model
        _norm("norms_tokens", "norm_forward", 8, 1024, "bf16", "bf16", "rms", "rms", 0, False, False),
        # the evaluation batch of 64 images between two DeiT-S blocks: per-channel scale of
        # the branch, residual stream in 32 bits
        _norm("norms_images", "norm_forward", 64 * 197, 384, "f32", "bf16", "none", "layer", 0,
              True, False),
        # a training step of ViT-B width with a gate per image and norms on both sides
        _norm("norms_train_gates", "norm_backward", 64 * 197, 768, "bf16", "bf16", "rms", "rms",
              197, False, False, 0.5),
        # a training step of the wide model: padded sequences, 32-bit residual stream
        _norm("norms_train_wide", "norm_backward", 65536, 1024, "f32", "bf16", "layer", "layer",
              0, True, True),
        # the small layer's router
        _balance("balance_small", 256, 4, "f32", False, 2, False),
        # the DeiT-S batch: the residual experts' columns of the router's product, each token
        # with the number of experts that its routing gave it
        _balance("balance_images", 64 * 197, 8, "bf16", True, 0, False),
        # the wide layer's 32 experts, padded sequences
        _balance("balance_wide", 65536, 32, "f32", True, 0, True),
        # one batch of activations on its way to a 4-bit product
        _quantize("fp4_images", 64 * 197, 384, "bf16"),
        # the 33 experts of the wide layer, from their 32-bit master weights
        _quantize("fp4_weights", 33 * 4096, 1024, "f32"),
        # a server's few tokens, each at its own experts
        _product("fp4_tokens_up", 24, 33, 4096, 1024, "gelu", "bf16"),
        # the ViT-B batch over its (expert, block) groups
        _product("fp4_blocks_up", 100003, 272, 192, 768, "gelu", "bf16"),
        # a large batch through the wide layer's down projections
        _product("fp4_wide_down", 131072, 33, 1024, 4096, "none", "f32"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["norm_forward", "norm_backward", "balance", "quantize", "product"])
    if call.startswith("norm"):
        d = _spread(rng, 48, 4096)
        d = d if rng.random() < 0.3 else max(64, d // 64 * 64)
        T = _spread(rng, 1, min(65536, 65536 * 1024 // d))
        stream, branch = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
        post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("rms", "none"),
                                ("rms", "rms"), ("layer", "layer"), ("layer", "rms")])
        c = _norm("", call, T, d, stream, branch, post, pre,
                  rng.choice([-1, 0, 0, 1, 64, 197]), rng.random() < 0.5, rng.random() < 0.3,
                  rng.choice([1.0, 0.5, 1.25]))
    elif call == "balance":
        K = _spread(rng, 2, 256)
        T = _spread(rng, 1, min(65536, 65536 * 32 // K))
        c = _balance("", T, K, rng.choice(["f32", "bf16"]), rng.random() < 0.5,
                     rng.choice([0, 1, 2, min(K, 8)]), rng.random() < 0.3)
        c["top"] = min(c["top"], K)
    elif call == "quantize":
        cols = _spread(rng, 1, 8192)
        cols = cols if rng.random() < 0.4 else max(32, cols // 32 * 32)
        c = _quantize("", _spread(rng, 1, min(131072, 33 * 4096 * 1024 // cols)), cols,
                      rng.choice(["f32", "bf16"]))
    else:
        cols = _spread(rng, 64, 4096)
        cols = cols if rng.random() < 0.3 else max(64, cols // 64 * 64)
        n = _spread(rng, 64, 4096)
        n = n if rng.random() < 0.3 else max(64, n // 64 * 64)
        groups = min(_spread(rng, 1, 300), max(1, (1 << 28) // (n * cols)))
        rows = _spread(rng, 1, min(100000, 100000 * 1024 * 2048 // (n * cols)))
        c = _product("", rows, groups, n, cols, rng.choice(["none", "gelu"]),
                     rng.choice(["bf16", "f32"]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _padding(T, g):
    """Sequences of 128 slots, a random number of them filled."""
    n = (T + 127) // 128
    lens = torch.randint(16, 129, (n,), generator=g, device="cuda")
    return (torch.arange(128, device="cuda") < lens[:, None]).reshape(-1)[:T].contiguous()


def _statistics(v, kind, eps):
    """The saved statistics of a norm over the rows of v, as its forward leaves them."""
    v = v.float()
    mean = v.mean(1) if kind == "layer" else torch.zeros_like(v[:, 0])
    var = (v - mean[:, None]).square().mean(1)
    return mean, torch.rsqrt(var + eps)


EPS = 1e-6


def _prepare_norm(case, g):
    T, d = case["T"], case["d"]
    f = dict(generator=g, device="cuda", dtype=F32)
    ts, tb = TYPES[case["stream"]], TYPES[case["branch"]]
    valid = _padding(T, g) if case["padded"] else None

    def rows(scale, dtype, shift=0.0):
        v = torch.randn(T, d, **f) * scale + shift
        if valid is not None:
            v[~valid] = float("nan")
        return v.to(dtype)

    def param(mean, scale):
        return (mean + scale * torch.randn(d, **f)).to(tb)

    post, pre = case["post"] != "none", case["pre"] != "none"
    s = dict(case=case, mask=None if valid is None else valid.to(torch.uint8))
    # a residual stream has a few channels much larger than the others
    loud = torch.where(torch.rand(d, generator=g, device="cuda") < 0.02, 8.0, 1.0)
    s["y"] = rows(0.7, tb, 0.1)
    s["post_weight"] = param(1.0, 0.1) if post else None
    s["post_bias"] = param(0.0, 0.1) if post and case["bias"] else None
    s["pre_weight"] = param(1.0, 0.1) if pre else None
    s["pre_bias"] = param(0.0, 0.1) if pre and case["bias"] else None
    gr = case["gate_rows"]
    G = 0 if gr < 0 else 1 if gr == 0 else (T + gr - 1) // gr
    s["gate"] = (0.3 + 0.3 * torch.randn(G, d, **f)).to(tb) if G else None
    stream = (rows(1.0, F32) * loud).to(ts)
    if case["call"] == "norm_forward":
        s["x"] = stream
    else:
        s["out"] = stream
        s["dout"] = rows(0.01, ts)
        s["du"] = rows(0.01, tb) if pre else None
        stats = dict(post_mean=None, post_rstd=None, pre_mean=None, pre_rstd=None)
        if post:
            stats["post_mean"], stats["post_rstd"] = _statistics(s["y"], case["post"], EPS)
        if pre:
            stats["pre_mean"], stats["pre_rstd"] = _statistics(s["out"], case["pre"], EPS)
        s["stats"] = stats
    return s


def _prepare_balance(case, g):
    T, K = case["T"], case["K"]
    z = torch.randn(T, K, generator=g, device="cuda") * 1.5
    z += torch.linspace(1.0, -1.0, K, device="cuda")  # some experts are more popular
    valid = _padding(T, g) if case["padded"] else None
    q = torch.sort(z, dim=1, descending=True, stable=True)[1].to(torch.int32)
    k = None
    if case["top"]:
        q = q[:, :case["top"]].contiguous()
    else:
        k = torch.randint(0, min(K, 6) + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    if valid is not None:
        z[~valid] = float("nan")
    z = z.to(TYPES[case["dtype"]])
    if case["shared"]:
        z = torch.cat([torch.zeros_like(z[:, :1]), z], 1)[:, 1:]
    return dict(case=case, logits=z, q=q, k=k, mask=None if valid is None else valid.to(torch.uint8))


def _prepare_quantize(case, g):
    x = torch.randn(case["rows"], case["cols"], generator=g, device="cuda")
    # rows of very different sizes, and a few large values within a row
    x *= torch.exp(1.5 * torch.randn(case["rows"], 1, generator=g, device="cuda"))
    x *= torch.where(torch.rand(x.shape, generator=g, device="cuda") < 0.01, 8.0, 1.0)
    return dict(case=case, x=x.to(TYPES[case["dtype"]]))


def _codes(g, rows, cols):
    """Rows in microscaled 4-bit form: two elements a byte (the first in the low half),
    a scale byte for each 32, rows of scales filled up to a multiple of 8 with 0."""
    blocks = (cols + 31) // 32
    codes = torch.randint(0, 256, (rows, blocks * 16), generator=g, device="cuda",
                          dtype=torch.uint8)
    if cols % 32:  # elements past the last one are 0
        codes[:, (cols + 1) // 2:] = 0
        if cols % 2:
            codes[:, cols // 2] &= 15
    scales = torch.zeros(rows, (blocks + 7) // 8 * 8, device="cuda", dtype=torch.uint8)
    scales[:, :blocks] = torch.randint(119, 124, (rows, blocks), generator=g, device="cuda",
                                       dtype=torch.uint8)
    return codes, scales


def _prepare_product(case, g):
    rows, G, n, cols = (case[k] for k in ("rows", "groups", "n", "cols"))
    a, a_scales = _codes(g, rows, cols)
    w, w_scales = _codes(g, G * n, cols)
    # uneven groups, about one in ten without rows
    share = torch.rand(G, generator=g, device="cuda", dtype=torch.float64).square() + 0.02
    share *= torch.rand(G, generator=g, device="cuda") < 0.9
    share[G // 2] += 0.02
    at = torch.cumsum(share, 0)
    ends = torch.round(at / at[-1] * rows).to(torch.int32)
    ends[-1] = rows
    offsets = torch.cat([torch.zeros_like(ends[:1]), ends])
    return dict(case=case, a=a, a_scales=a_scales, w=w.view(G, n, -1),
                w_scales=w_scales.view(G, n, -1), offsets=offsets,
                longest=int((offsets[1:] - offsets[:-1]).max()))


def prepare(case, seed):
    g = _generator(seed)
    if case["call"].startswith("norm"):
        return _prepare_norm(case, g)
    return {"balance": _prepare_balance, "quantize": _prepare_quantize,
            "product": _prepare_product}[case["call"]](case, g)


# ------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2608_10392_gb300 as pkg

    case = s["case"]
    if case["call"].startswith("norm"):
        norm = pkg.BlockNorm(case["d"], stream_dtype=case["stream"], branch_dtype=case["branch"],
                             post_norm=case["post"], pre_norm=case["pre"],
                             gate_rows=max(case["gate_rows"], 0), res_scale=case["scale"], eps=EPS)
        params = {k: s[k] for k in ("post_weight", "post_bias", "gate", "pre_weight")}
        if case["call"] == "norm_forward":
            r = norm.forward(s["x"], s["y"], **params, pre_bias=s["pre_bias"], mask=s["mask"])
            return {k: r[k] for k in ("out", "u")}
        r = norm.backward(s["out"], s["y"], s["stats"], dout=s["dout"], du=s["du"], **params,
                          mask=s["mask"])
        return {k: r[k] for k in _gradients(case)}
    if case["call"] == "balance":
        return pkg.balance_loss(s["logits"], s["q"], s["k"], mask=s["mask"],
                                balance_weight=W_BALANCE, z_weight=W_Z)
    if case["call"] == "quantize":
        q = pkg.mxfp4_quantize(s["x"])
        return pkg.mxfp4_dequantize(q, dtype=case["dtype"])
    a = pkg.Mxfp4(s["a"], s["a_scales"], case["cols"])
    w = pkg.Mxfp4(s["w"], s["w_scales"], case["cols"])
    return pkg.mxfp4_product(a, w, s["offsets"], activation=case["act"], dtype=case["dtype"])


# ------------------------------------------------------------- the plain forms

W_BALANCE, W_Z = 0.01, 0.001


def _gradients(case):
    names = ["dx", "dy"]
    if case["post"] != "none":
        names += ["d_post_weight"] + (["d_post_bias"] if case["bias"] else [])
    if case["gate_rows"] >= 0:
        names.append("d_gate")
    if case["pre"] != "none":
        names += ["d_pre_weight"] + (["d_pre_bias"] if case["bias"] else [])
    return names


def _gate_of(s, T):
    """The gate of every token, [T][d] or [1][d]."""
    gate, gr = s["gate"].float(), s["case"]["gate_rows"]
    return gate if gr == 0 else gate[torch.arange(T, device="cuda") // gr]


def _plain_forward(s):
    case = s["case"]
    ts, tb = TYPES[case["stream"]], TYPES[case["branch"]]

    def normed(v, kind, weight, bias):
        mean, rstd = _statistics(v, kind, EPS)
        v = (v - mean[:, None]) * rstd[:, None] * weight.float()
        return v if bias is None else v + bias.float()

    x, z = s["x"].float(), s["y"].float()
    if case["post"] != "none":
        z = normed(z, case["post"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        z = z * _gate_of(s, case["T"])
    out = case["scale"] * x + z
    u = None
    if case["pre"] != "none":
        u = normed(out, case["pre"], s["pre_weight"], s["pre_bias"])
    if s["mask"] is not None:
        pad = s["mask"][:, None] == 0
        out = out.masked_fill(pad, 0)
        u = None if u is None else u.masked_fill(pad, 0)
    return dict(out=out.to(ts), u=None if u is None else u.to(tb))


def _plain_backward(s):
    case, st = s["case"], s["stats"]
    T, d, gr = case["T"], case["d"], case["gate_rows"]
    ts, tb = TYPES[case["stream"]], TYPES[case["branch"]]
    pad = None if s["mask"] is None else s["mask"][:, None] == 0

    def clean(v):
        v = v.float()
        return v if pad is None else v.masked_fill(pad, 0)

    def standard(v, mean, rstd):
        return clean((v.float() - mean[:, None]) * rstd[:, None])

    def through(a, v, rstd, kind):
        """The gradient of a norm's input, from that of its standardised rows v."""
        if kind == "layer":
            a = a - a.mean(1, keepdim=True)
        return rstd[:, None] * (a - v * (a * v).mean(1, keepdim=True))

    r = {}
    D = clean(s["dout"])
    if case["pre"] != "none":
        o, du = standard(s["out"], st["pre_mean"], st["pre_rstd"]), clean(s["du"])
        D = D + clean(through(du * s["pre_weight"].float(), o, st["pre_rstd"], case["pre"]))
        r["d_pre_weight"], r["d_pre_bias"] = (du * o).sum(0), du.sum(0)
    r["dx"] = (case["scale"] * D).to(ts)
    post = case["post"] != "none"
    yn = standard(s["y"], st["post_mean"], st["post_rstd"]) if post else clean(s["y"])
    if gr >= 0:
        z = yn
        if post:
            z = z * s["post_weight"].float()
            z = z if s["post_bias"] is None else z + s["post_bias"].float()
        dg = D * z
        if gr == 0:
            r["d_gate"] = dg.sum(0, keepdim=True)
        else:
            G = s["gate"].shape[0]
            full = torch.zeros(G * gr, d, device="cuda")
            full[:T] = dg
            r["d_gate"] = full.view(G, gr, d).sum(1)
        D = D * _gate_of(s, T)
    if post:
        r["d_post_weight"], r["d_post_bias"] = (D * yn).sum(0), D.sum(0)
        D = clean(through(D * s["post_weight"].float(), yn, st["post_rstd"], case["post"]))
    r["dy"] = D.to(tb)
    return {k: r[k] for k in _gradients(case)}


def _plain_balance(s):
    z, q, k = s["logits"].float(), s["q"].long(), s["k"]
    T, K = z.shape
    chosen = torch.ones_like(q, dtype=torch.bool)
    if k is not None:
        chosen = torch.arange(q.shape[1], device="cuda") < k[:, None]
    valid = torch.ones(T, dtype=torch.bool, device="cuda")
    if s["mask"] is not None:
        valid = s["mask"] != 0
        z = z.masked_fill(~valid[:, None], 0)
        chosen = chosen & valid[:, None]
    n = valid.sum().clamp(min=1)
    counts = torch.zeros(K, dtype=torch.int32, device="cuda").index_add_(
        0, q.reshape(-1), chosen.reshape(-1).to(torch.int32))
    top = z.max(1, keepdim=True)[0]
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    p = e / total * valid[:, None]
    lse = (torch.log(total) + top) * valid[:, None]
    f = counts.float() / counts.sum().clamp(min=1)
    P = p.sum(0) / n
    balance, zloss = K * (f * P).sum(), lse.square().sum() / n
    dz = p / n * (W_BALANCE * K * (f - (p * f).sum(1, keepdim=True)) + 2 * W_Z * lse)
    return dict(loss=torch.stack([W_BALANCE * balance + W_Z * zloss, balance, zloss]),
                counts=counts, prob=P, dlogits=dz)


def _two_to(e, dtype):
    """2^e for whole numbers e >= -127, exactly (from its bits: pow may round)."""
    if dtype == torch.float64:
        return (e.long() + 1023 << 52).view(dtype)
    return torch.where(e > -127, e.int() + 127 << 23, 1 << 22).view(dtype)


def _plain_quantize(s):
    x = s["x"].float()
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    exponent = torch.frexp(x.abs().amax(2, keepdim=True))[1] - 3
    scale = _two_to(exponent.clamp(min=-127), F32)
    v = x / scale
    m = v.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    v = torch.sign(v) * torch.clamp(torch.round(m / step) * step, max=6.0)
    return (v * scale).view(rows, -1)[:, :cols].to(TYPES[s["case"]["dtype"]])


LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _read(codes, scales, cols, dtype):
    """The values of rows in microscaled 4-bit form."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda", dtype=dtype)
    two = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1)
    blocks = (cols + 31) // 32
    size = _two_to(scales.int() - 127, dtype)[..., :blocks]
    v = two.view(*codes.shape[:-1], blocks, 32) * size[..., None]
    return v.view(*codes.shape[:-1], blocks * 32)[..., :cols]


def _gelu(v):
    return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))


def _plain_product(s):
    case, at = s["case"], s["offsets"].long()
    a = _read(s["a"], s["a_scales"], case["cols"], F32)
    w = _read(s["w"], s["w_scales"], case["cols"], F32)
    r = torch.arange(case["rows"], device="cuda")
    g = torch.searchsorted(at[1:], r, right=True)
    spread = torch.zeros(case["groups"], s["longest"], case["cols"], device="cuda")
    spread[g, r - at[g]] = a
    y = torch.bmm(spread, w.transpose(1, 2))[g, r - at[g]]
    return (_gelu(y) if case["act"] == "gelu" else y).to(TYPES[case["dtype"]])


def run(state):
    if own:
        return _own(state)
    return {"norm_forward": _plain_forward, "norm_backward": _plain_backward,
            "balance": _plain_balance, "quantize": _plain_quantize,
            "product": _plain_product}[state["case"]["call"]](state)


# ---------------------------------------------------------------------- work

def work(case):
    if case["call"].startswith("norm"):
        T, d = case["T"], case["d"]
        bs, bb = (4 if case[k] == "f32" else 2 for k in ("stream", "branch"))
        pre, post = case["pre"] != "none", case["post"] != "none"
        gr = case["gate_rows"]
        gates = 0 if gr < 0 else d if gr == 0 else (T + gr - 1) // gr * d
        if case["call"] == "norm_forward":
            each = 2 * bs + bb + (bb if pre else 0)
            flops = 4 + 8 * (pre + post)
            extra = bb * gates
        else:
            each = 3 * bs + 2 * bb + (bb if pre else 0) - (0 if pre else bs)
            flops = 4 + 16 * (pre + post)
            extra = (bb + 4) * gates
        return {"bytes": T * d * each + extra, "flops": T * d * flops}
    if case["call"] == "balance":
        T, K = case["T"], case["K"]
        per = K * (2 if case["dtype"] == "bf16" else 4) + 4 * K + 4 * (case["top"] or 3)
        return {"bytes": T * per + 8 * K, "flops": 12 * T * K}
    if case["call"] == "quantize":
        n, b = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * (2 * b + 2 * 17 / 32), "flops": 6 * n}
    rows, n, cols = case["rows"], case["n"], case["cols"]
    used = min(rows, 0.9 * case["groups"])  # about one group in ten has no rows
    held = (rows + used * n) * cols * 17 / 32
    return {"bytes": held + rows * n * (2 if case["dtype"] == "bf16" else 4),
            "flops": 2 * rows * n * cols}


# --------------------------------------------------------------- in 64 bits

def _exact_norm(s):
    """The definition in 64 bits; gradients by differentiating it."""
    case = s["case"]
    T, gr = case["T"], case["gate_rows"]
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0

    def norm(v, kind, weight, bias):
        mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
        v = v - mean
        v = v * (v.square().mean(1, keepdim=True) + EPS) ** -0.5 * weight
        return v if bias is None else v + bias

    forward = case["call"] == "norm_forward"
    p = {k: s[k].double() for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")
         if s[k] is not None}
    y = s["y"][keep].double()
    x = s["x" if forward else "out"][keep].double()
    if not forward:
        # out as a leaf in the place of the sum: its gradient D is that of scale x + gate z
        leaves = dict(p, x=x, y=y)
        for v in leaves.values():
            v.requires_grad_(True)
    z = norm(y, case["post"], p["post_weight"], p.get("post_bias")) if "post_weight" in p else y
    if "gate" in p:
        z = z * (p["gate"] if gr == 0 else p["gate"][(torch.arange(T, device="cuda") // gr)[keep]])

    def whole(v, dtype=torch.float64):
        full = torch.zeros(T, v.shape[1], device="cuda", dtype=dtype)
        full[keep] = v.detach()
        return full

    if forward:
        out = case["scale"] * x + z
        u = norm(out, case["pre"], p["pre_weight"], p.get("pre_bias")) if "pre_weight" in p else None
        return dict(out=whole(out), u=None if u is None else whole(u))
    dout = s["dout"][keep].double()
    total = (x * dout).sum()
    if "pre_weight" in p:
        if "pre_bias" not in p:
            p["pre_bias"] = torch.zeros_like(p["pre_weight"])
        total = total + (norm(x, case["pre"], p["pre_weight"], p["pre_bias"])
                         * s["du"][keep].double()).sum()
    wanted = ["x"] + [k for k in ("pre_weight", "pre_bias") if k in p and p[k].requires_grad]
    first = dict(zip(wanted, torch.autograd.grad(total, [x if k == "x" else p[k] for k in wanted])))
    wanted = ["y"] + [k for k in ("post_weight", "post_bias", "gate") if k in p]
    second = dict(zip(wanted, torch.autograd.grad((z * first["x"]).sum(),
                                                  [y if k == "y" else p[k] for k in wanted])))
    r = dict(dx=whole(case["scale"] * first.pop("x")), dy=whole(second.pop("y")))
    r.update({"d_" + k: v for k, v in {**first, **second}.items()})
    return {k: r[k] for k in _gradients(case)}


def _exact_balance(s):
    case = s["case"]
    T, K = case["T"], case["K"]
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    z = s["logits"][keep].double().requires_grad_(True)
    q = s["q"][keep].long()
    k = torch.full((q.shape[0],), q.shape[1], device="cuda") if s["k"] is None else s["k"][keep]
    picked = q[torch.arange(q.shape[1], device="cuda")[None, :] < k[:, None]]
    counts = torch.bincount(picked, minlength=K).double()
    f = counts / max(1, picked.numel())
    n = max(1, z.shape[0])
    P = torch.softmax(z, 1).sum(0) / n
    balance, zloss = K * (f * P).sum(), torch.logsumexp(z, 1).square().sum() / n
    loss = W_BALANCE * balance + W_Z * zloss
    d = torch.zeros(T, K, device="cuda", dtype=torch.float64)
    d[keep] = torch.autograd.grad(loss, z)[0]
    return dict(loss=torch.stack([loss, balance, zloss]).detach(), counts=None, prob=P.detach(),
                dlogits=d)


def _exact_quantize(s):
    x = s["x"].double()
    rows, cols = x.shape
    levels = torch.tensor(LEVELS, device="cuda", dtype=torch.float64)
    # ties go to the level whose mantissa bit is 0: every second one
    middles = (levels[1:] + levels[:-1]) / 2
    got = torch.empty_like(x)
    for c in range(0, cols, 32):
        block = x[:, c:c + 32]
        most = block.abs().amax(1, keepdim=True)
        # 2^e <= most < 2^(e + 1), by comparisons: a logarithm may round across a power of two
        e = torch.floor(torch.log2(most.clamp(min=1e-60)))
        e = torch.where(_two_to(e + 1, x.dtype) <= most, e + 1, e)
        e = torch.where(_two_to(e, x.dtype) > most, e - 1, e)
        size = _two_to(torch.clamp(e - 2, min=-127), x.dtype)
        m = block.abs() / size
        up, down = torch.bucketize(m, middles, right=True), torch.bucketize(m, middles)
        code = torch.where(up % 2 == 0, up, down)
        got[:, c:c + 32] = torch.sign(block) * levels[code] * size
    return got


def _exact_product(s):
    case, at = s["case"], s["offsets"].tolist()
    y = torch.empty(case["rows"], case["n"], device="cuda", dtype=torch.float64)
    for g in range(case["groups"]):
        lo, hi = at[g], at[g + 1]
        if hi > lo:
            a = _read(s["a"][lo:hi], s["a_scales"][lo:hi], case["cols"], torch.float64)
            w = _read(s["w"][g], s["w_scales"][g], case["cols"], torch.float64)
            y[lo:hi] = a @ w.T
    return y * torch.special.ndtr(y) if case["act"] == "gelu" else y


def exact(case, seed):
    s = prepare(case, seed)
    if case["call"].startswith("norm"):
        return _exact_norm(s)
    return {"balance": _exact_balance, "quantize": _exact_quantize,
            "product": _exact_product}[case["call"]](s)
