"""Dense products, 8-bit rows and few-token layers, as cases to be measured.

Five calls: "linear" (rows times a weight matrix with bias, activation and residual
in the product's epilogue), "linear_fp8" (the same with rows and weights in 8-bit
floating point, a scale for each row and each output channel; the rows given in 8 bits
or brought there first), "linear_backward" (the gradients of rows, weights and bias),
"norm_fp8" (the norms and the residual sum between two blocks with the normalised rows
in 8 bits, and back) and "few" (a whole mixture-of-experts layer for at most 64
tokens). Sizes are those round the layers of the workloads package and of its wide
layer: widths 384, 768 and 1,024, hidden widths 1,536 and 4,096, up to 32 experts;
each call has a plain form in elementary torch operations.
"""
import math

import torch

own = False

F32, BF16, F8, F64 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float64
TYPES = {"f32": F32, "bf16": BF16}


# ------------------------------------------------------------------- cases

def _linear(name, T, cols, n, act="none", bias=True, residual="none", padded=False, keep=False,
            gap=0):
    """residual: "none", "bf16" or "f32" (the result's type with it, else bf16); keep: the
    result before the activation comes too; gap: unused elements between two rows."""
    return dict(name=name, call="linear", T=T, cols=cols, n=n, act=act, bias=bias,
                residual=residual, padded=padded, keep=keep, gap=gap)


def _fp8(name, T, cols, n, act="none", bias=True, residual="none", quantize=False):
    """quantize: the rows come in bf16 and go to 8 bits within the call."""
    return dict(name=name, call="linear_fp8", T=T, cols=cols, n=n, act=act, bias=bias,
                residual=residual, padded=False, quantize=quantize)


def _backward(name, T, cols, n, act="none", bias=True, padded=False):
    """The weights' gradient is bf16 through an activation, fp32 without one."""
    return dict(name=name, call="linear_backward", T=T, cols=cols, n=n, act=act, bias=bias,
                padded=padded)


def _norm(name, T, d, stream, post, pre, bias, gate, padded):
    return dict(name=name, call="norm_fp8", T=T, d=d, stream=stream, post=post, pre=pre,
                bias=bias, gate=gate, padded=padded)


def _few(name, T, d, H, K, B, padded=False, **options):
    """options: topk (0: by cumulative mass), beta (-1: adaptive), prefix."""
    c = dict(name=name, call="few", T=T, d=d, H=H, K=K, B=B, padded=padded, topk=0, beta=-1.0,
             prefix=False)
    c.update(options)
    return c


def listed():
    return [
        # one token of a server through the wide layer's 33 experts
        _few("few_one", 1, 1024, 4096, 32, 16),
        # a server's batch of single tokens, three of four slots in use
        _few("few_server", 24, 1024, 4096, 32, 16, padded=True),
        # four tokens through a dense up projection
        _linear("linear_tokens", 4, 1024, 4096, act="gelu"),
        # a batch of 64 images into a dense FFN of DeiT-S, in training
        _linear("linear_images", 64 * 197, 384, 1536, act="gelu", keep=True),
        # odd sizes all round, a padded batch onto a bf16 stream
        _linear("linear_odd", 5003, 1001, 777, residual="bf16", padded=True),
        # a large batch out of the wide FFN onto a 32-bit residual stream
        _linear("linear_wide", 65536, 4096, 1024, residual="f32"),
        # eight single tokens: rows to 8 bits, then down with the residual
        _fp8("fp8_tokens", 8, 4096, 1024, residual="bf16", quantize=True),
        # a large batch into the wide FFN, rows already in 8 bits
        _fp8("fp8_wide", 65536, 1024, 4096, act="gelu"),
        # the gradients of the DeiT-S batch through the activation
        _backward("back_images", 64 * 197, 384, 1536, act="gelu"),
        # padded sequences, the gradients of the wide down projection
        _backward("back_wide", 32768, 4096, 1024, padded=True),
        # eight single tokens between two blocks, on their way to an 8-bit product
        _norm("norm8_tokens", 8, 1024, "bf16", "none", "rms", False, False, False),
        # a large batch: 32-bit stream, norms on both sides, a gate
        _norm("norm8_wide", 65536, 1024, "f32", "rms", "rms", False, True, False),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    v = _spread(rng, lo, hi)
    return v if rng.random() < 0.3 else max(64, v // 64 * 64)


def draw(rng):
    call = rng.choice(["linear", "linear", "linear_fp8", "linear_backward", "norm_fp8", "few"])
    act, bias = rng.choice(["none", "gelu"]), rng.random() < 0.7
    residual = rng.choice(["none", "none", "bf16", "f32"])
    padded = rng.random() < 0.3
    if call == "few":
        B = rng.choice([4, 8, 8, 12, 16])
        M = 64 * rng.randint(1, 256 // 64)
        d = 64 * rng.choice([2, 5, 6, 6, 8, 12, 16])
        c = _few("", _spread(rng, 1, 64), d, B * M, rng.randint(2, 32), B, padded,
                 **rng.choice([{}, {}, {}, dict(topk=2), dict(beta=0.7), dict(prefix=True)]))
    elif call == "norm_fp8":
        d = _width(rng, 48, 4096)
        post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("rms", "rms"),
                                ("layer", "rms"), ("layer", "layer")])
        c = _norm("", _spread(rng, 1, min(65536, 65536 * 1024 // d)), d,
                  rng.choice(["f32", "bf16"]), post, pre, bias, rng.random() < 0.5, padded)
    else:
        cols, n = _width(rng, 32, 8192), _width(rng, 32, 8192)
        most = (1 << 38) if call != "linear_backward" else (1 << 37)
        T = _spread(rng, 1, min(65536, most // (cols * n)))
        if call == "linear":
            c = _linear("", T, cols, n, act, bias, residual, padded, rng.random() < 0.3,
                        rng.choice([0, 0, 0, 8, 3]))
        elif call == "linear_fp8":
            c = _fp8("", T, cols, n, act, bias, residual, rng.random() < 0.5)
        else:
            c = _backward("", T, cols, n, act, bias, padded)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 31)
    return g


def _padding(T, g):
    """Slots in use: of sequences of 128 a random number each, of fewer than 128 single
    tokens about three in four."""
    if T < 128:
        return torch.rand(T, generator=g, device="cuda") < 0.75
    n = (T + 127) // 128
    lens = torch.randint(16, 129, (n,), generator=g, device="cuda")
    return (torch.arange(128, device="cuda") < lens[:, None]).reshape(-1)[:T].contiguous()


def _rows(T, d, g, valid=None, loud=0.0, gap=0):
    """Activations: near unit size, a share `loud` of the channels much larger than the
    others, padding NaN."""
    x = torch.randn(T, d + gap, generator=g, device="cuda")
    if loud:
        x *= torch.where(torch.rand(d + gap, generator=g, device="cuda") < loud, 8.0, 1.0)
    if valid is not None:
        x[~valid] = float("nan")
    return x


def _eight(v, scale):
    """Values in 8 bits under a scale for each row, rows 16 bytes apart or a multiple."""
    rows, cols = v.shape
    wide = torch.zeros(rows, (cols + 15) // 16 * 16, device="cuda", dtype=F8)
    wide[:, :cols] = (v / scale[:, None]).clamp(-448, 448).to(F8)
    return wide[:, :cols]


def _prepare_linear(case, g):
    T, cols, n = case["T"], case["cols"], case["n"]
    f = dict(generator=g, device="cuda")
    valid = _padding(T, g) if case["padded"] else None
    s = dict(case=case, mask=None if valid is None else valid.to(torch.uint8))
    w = torch.randn(n, cols, **f) * cols ** -0.5
    s["bias"] = (0.3 * torch.randn(n, **f)).to(BF16) if case["bias"] else None
    x = _rows(T, cols, g, valid, 0.01, case.get("gap", 0))
    if case["call"] == "linear_fp8":
        s["w_scale"] = w.abs().amax(1) / 448
        s["w"] = _eight(w, s["w_scale"])
        if case["quantize"]:
            s["x"] = x.to(BF16)
        else:
            s["x_scale"] = x.abs().amax(1) / 448
            s["x"] = _eight(x, s["x_scale"])
    else:
        s["w"], s["x"] = w.to(BF16), x.to(BF16)[:, :cols]
    if case["call"] == "linear_backward":
        z = torch.randn(T, n, **f) * 1.2
        dout = 0.01 * torch.randn(T, n, **f)
        if valid is not None:
            z[~valid] = float("nan")
            dout[~valid] = float("nan")
        s["z"] = z.to(BF16) if case["act"] != "none" else None
        s["dout"] = dout.to(BF16)
    else:
        s["residual"] = None
        if case["residual"] != "none":
            s["residual"] = (2 * _rows(T, n, g, valid)).to(TYPES[case["residual"]])
    return s


EPS = 1e-6


def _prepare_norm(case, g):
    T, d = case["T"], case["d"]
    valid = _padding(T, g) if case["padded"] else None

    def param(mean, scale):
        return (mean + scale * torch.randn(d, generator=g, device="cuda")).to(BF16)

    s = dict(case=case, mask=None if valid is None else valid.to(torch.uint8))
    s["x"] = _rows(T, d, g, valid, 0.02).to(TYPES[case["stream"]])
    s["y"] = (0.7 * _rows(T, d, g, valid) + 0.1).to(BF16)
    post = case["post"] != "none"
    s["post_weight"] = param(1.0, 0.1) if post else None
    s["post_bias"] = param(0.0, 0.1) if post and case["bias"] else None
    s["gate"] = param(0.3, 0.3)[None] if case["gate"] else None
    s["pre_weight"] = param(1.0, 0.1)
    s["pre_bias"] = param(0.0, 0.1) if case["bias"] else None
    return s


def _decide(s, x, dtype):
    """The layer's routing in 64 bits: the weight of every (token, expert, block), and how
    far each token is from a decision that would change them."""
    case = s["case"]
    K, B = case["K"], case["B"]
    z = x.to(dtype) @ s["router"].to(dtype).T
    logits, u = z[:, 1:1 + K] + s["router_bias"][1:], z[:, 1 + K:]
    tau = (B - 1) / B ** 2
    alpha = tau + (1 - 2 * tau) * torch.sigmoid(z[:, :1] + s["router_bias"][:1])
    count = torch.round(B * alpha).clamp(0, B)
    margin = ((B * alpha - torch.floor(B * alpha) - 0.5).abs() / B)[:, 0]
    place = torch.arange(B, device="cuda")
    if case["prefix"]:
        shared = place < count
    else:
        order = torch.sort(u, dim=1, descending=True, stable=True)
        shared = torch.empty_like(u, dtype=torch.bool).scatter_(1, order[1], place < count)
        edge = torch.cat([order[0], order[0][:, -1:] - 1], 1)
        at = count.long()
        gap = (edge.gather(1, (at - 1).clamp(min=0)) - edge.gather(1, at))[:, 0]
        margin = torch.minimum(margin, torch.where((at[:, 0] > 0) & (at[:, 0] < B), gap, 1.0))
    share = torch.softmax(logits, 1)
    p, q = torch.sort(share, dim=1, descending=True, stable=True)
    if case["topk"]:
        k = torch.full_like(q[:, :1], min(case["topk"], K))
    else:
        beta = 1 - alpha if case["beta"] < 0 else torch.full_like(alpha, case["beta"])
        mass = torch.cumsum(p, 1)
        k = ((mass < beta).sum(1, keepdim=True) + 1).clamp(max=K)
        margin = torch.minimum(margin, (mass - beta).abs().amin(1))
    edge = torch.cat([p, torch.full_like(p[:, :1], -1.0)], 1)
    margin = torch.minimum(margin, (edge.gather(1, k - 1) - edge.gather(1, k))[:, 0])
    taken = torch.empty_like(share, dtype=torch.bool).scatter_(
        1, q, torch.arange(K, device="cuda") < k)
    weight = torch.cat([(alpha * shared)[:, None], (share * taken)[:, :, None] * ~shared[:, None]], 1)
    if s["mask"] is not None and len(x) == len(s["mask"]):
        weight = torch.where(s["mask"][:, None, None] != 0, weight, 0.0)
    return weight, margin


def _prepare_few(case, g):
    T, d, H, K, B = (case[k] for k in ("T", "d", "H", "K", "B"))
    f = dict(generator=g, device="cuda")
    up = torch.randn(H, d, **f) * d ** -0.5
    down = torch.randn(d, H, **f) * H ** -0.5
    s = dict(case=case, mask=None)
    s["up"] = (up + torch.randn(K + 1, H, d, **f) * (0.05 * d ** -0.5)).to(BF16)
    s["down"] = (down + torch.randn(K + 1, d, H, **f) * (0.05 * H ** -0.5)).to(BF16)
    # the router's rows: the shared demand's, the experts', the mean key of each block of
    # the shared expert
    router = (torch.randn(K + 1, d, **f) * 0.02).to(BF16)
    keys = s["up"][0].view(B, H // B, d).to(F64).mean(1).to(BF16)
    s["router"] = torch.cat([router, keys]).contiguous()
    s["router_bias"] = 0.3 * torch.randn(K + 1, **f)
    # tokens within 1e-5 of another decision, whose answer either side of it would be
    # right, are left out
    x = _rows(4 * T + 64, d, g).to(BF16)
    clear = _decide(s, x, F64)[1] > 1e-5
    s["x"] = x[torch.sort(~clear, stable=True)[1][:T]].contiguous()
    if case["padded"]:
        valid = _padding(T, g)
        s["x"][~valid] = float("nan")
        s["mask"] = valid.to(torch.uint8)
    return s


def prepare(case, seed):
    g = _generator(seed)
    return {"few": _prepare_few, "norm_fp8": _prepare_norm}.get(case["call"], _prepare_linear)(case, g)


# ------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2608_10392_gb300 as pkg

    case = s["case"]
    if case["call"] == "few":
        return pkg.few_tokens(s["x"], s["router"], s["up"], s["down"], case["B"],
                              router_bias=s["router_bias"], mask=s["mask"],
                              topk_fixed=min(case["topk"], case["K"]),
                              beta_fixed=case["beta"] if case["beta"] >= 0 else math.nan,
                              prefix_blocks=case["prefix"])
    if case["call"] == "norm_fp8":
        norm = pkg.BlockNorm(case["d"], stream_dtype=case["stream"], branch_dtype="bf16",
                             post_norm=case["post"], pre_norm=case["pre"], eps=EPS, u_format="fp8")
        r = norm.forward(s["x"], s["y"], mask=s["mask"],
                         **{k: s[k] for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")})
        return dict(out=r["out"], u=pkg.fp8_dequantize(r["u"]))
    if case["call"] == "linear_backward":
        r = pkg.linear_backward(s["x"], s["w"], s["dout"], s["z"], activation=case["act"],
                                mask=s["mask"], bias=case["bias"],
                                grad_dtype="bf16" if case["act"] != "none" else "f32")
        return {k: v for k, v in r.items() if v is not None}
    x, w = s["x"], s["w"]
    if case["call"] == "linear_fp8":
        x = pkg.fp8_quantize(x) if case["quantize"] else pkg.Fp8(x, s["x_scale"])
        w = pkg.Fp8(w, s["w_scale"])
    return pkg.linear(x, w, s["bias"], activation=case["act"], residual=s["residual"],
                      mask=s["mask"], dtype="f32" if case["residual"] == "f32" else "bf16",
                      keep=case.get("keep", False))


# ------------------------------------------------------------- the plain forms

def _two_to(e, dtype):
    """2^e for whole numbers -127 < e < 128, exactly (from its bits: pow may round)."""
    if dtype == F64:
        return (e.long() + 1023 << 52).view(dtype)
    return (e.int() + 127 << 23).view(dtype)


def _to_eight(v):
    """Rows as values of 8 bits under a scale 2^e of their own, the smallest (from 2^-126
    on) that leaves none above 448; in the type of v."""
    most = v.abs().amax(1, keepdim=True)
    m, e = torch.frexp(most)  # most = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = (e - 9 + (m > 0.875)).clamp(min=-126)
    scale = _two_to(torch.where(most > 0, e, torch.full_like(e, -126)), v.dtype)
    return (v / scale).float().to(F8).to(v.dtype) * scale


def _gelu(v):
    return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))


def _clean(s, v):
    """v with 0 in the place of padding rows."""
    return v if s["mask"] is None else v.masked_fill(s["mask"][:, None] == 0, 0)


def _plain_linear(s):
    case = s["case"]
    x, w = s["x"].float(), s["w"].float()
    if case["call"] == "linear_fp8":
        x = _to_eight(x) if case["quantize"] else x * s["x_scale"][:, None]
        w = w * s["w_scale"][:, None]
    z = x @ w.T
    z = z if s["bias"] is None else z + s["bias"].float()
    y = _gelu(z) if case["act"] == "gelu" else z
    y = y if s["residual"] is None else y + s["residual"].float()
    y = _clean(s, y).to(F32 if case["residual"] == "f32" else BF16)
    return (y, _clean(s, z).to(BF16)) if case.get("keep", False) else y


def _plain_backward(s):
    case = s["case"]
    x, d = _clean(s, s["x"].float()), _clean(s, s["dout"].float())
    if case["act"] == "gelu":
        z = _clean(s, s["z"].float())
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        d = d * (cdf + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5)
    r = dict(dx=(d @ s["w"].float()).to(BF16),
             dw=(d.T @ x).to(F32 if case["act"] == "none" else BF16))
    if case["bias"]:
        r["dbias"] = d.sum(0)
    return r


def _plain_norm(s):
    case = s["case"]

    def normed(v, kind, weight, bias):
        if kind == "layer":
            v = v - v.mean(1, keepdim=True)
        v = v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS) * weight.float()
        return v if bias is None else v + bias.float()

    z = s["y"].float()
    if case["post"] != "none":
        z = normed(z, case["post"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        z = z * s["gate"].float()
    out = _clean(s, s["x"].float() + z)
    u = _clean(s, normed(out, case["pre"], s["pre_weight"], s["pre_bias"]))
    return dict(out=out.to(TYPES[case["stream"]]), u=_to_eight(u).to(BF16))


def _plain_few(s):
    case = s["case"]
    x = _clean(s, s["x"].float())
    weight = _decide(s, x, F64)[0].float()
    h = _gelu(torch.einsum("td,ehd->teh", x, s["up"].float()))
    h = h.view(*weight.shape, -1) * weight[..., None]
    return torch.einsum("teh,edh->td", h.flatten(2), s["down"].float()).to(BF16)


def run(state):
    if own:
        return _own(state)
    return {"few": _plain_few, "norm_fp8": _plain_norm, "linear_backward": _plain_backward}.get(
        state["case"]["call"], _plain_linear)(state)


# ---------------------------------------------------------------------- work

def work(case):
    T = case["T"]
    if case["call"] == "few":
        # a token runs about half of the shared expert's blocks and the other half of about
        # a third of the experts (or of the fixed number)
        d, H, K, B = (case[k] for k in ("d", "H", "K", "B"))
        n = min(case["topk"], K) if case["topk"] else max(1.0, 0.32 * K)
        T = T * (0.75 if case["padded"] else 1.0)
        pairs = B * (1 - 0.5 ** T) + K * B * (1 - (1 - n / (2 * K)) ** T)
        each = 2 * d * (H // B)  # weights of a pair
        return {"bytes": 2 * each * pairs + 2 * d * (2 * T + 1 + K + B),
                "flops": 2 * each * T * (B + n * B) / 2}
    if case["call"] == "norm_fp8":
        n = T * case["d"]
        return {"bytes": n * (2 * (4 if case["stream"] == "f32" else 2) + 2 + 1 + 1 + 2) + 8 * T,
                "flops": n * (8 + 8 * (case["post"] != "none"))}
    cols, n = case["cols"], case["n"]
    if case["call"] == "linear_backward":
        through = case["act"] != "none"
        return {"bytes": 2 * (2 * T * cols + cols * n + T * n * (2 if through else 1))
                + cols * n * (2 if through else 4) + 4 * n * case["bias"],
                "flops": 4 * T * cols * n}
    size = 1 if case["call"] == "linear_fp8" else 2
    res = {"none": 2, "bf16": 4, "f32": 8}[case["residual"]]
    return {"bytes": size * cols * n + T * cols * (2 if case.get("quantize") else size)
            + T * n * (res + 2 * case.get("keep", False)) + 2 * n * case["bias"],
            "flops": 2 * T * cols * n}


# --------------------------------------------------------------- in 64 bits

def _phi(z):
    return torch.special.ndtr(z)


def _exact_linear(s):
    case = s["case"]
    T, n = case["T"], case["n"]
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    x, w = s["x"][keep].to(F64) if s["x"].dtype != F8 else s["x"].to(F64), s["w"].to(F64)
    if case["call"] == "linear_fp8":
        if case["quantize"]:
            # the scale by comparisons: the first of 2^-126, 2^-125, ... that is enough
            scales = _two_to(torch.arange(-126, 121, device="cuda"), F64)
            most = x.abs().amax(1)
            size = scales[torch.bucketize(most, 448 * scales)][:, None]
            x = (x / size).float().to(F8).to(F64) * size
        else:
            x = x * s["x_scale"].to(F64)[:, None]
        w = w * s["w_scale"].to(F64)[:, None]
    z = torch.zeros(T, n, device="cuda", dtype=F64)
    z[keep] = torch.addmm(torch.zeros(n, device="cuda", dtype=F64) if s["bias"] is None
                          else s["bias"].to(F64), x, w.T)
    y = z * _phi(z) if case["act"] == "gelu" else z.clone()
    if s["residual"] is not None:
        y[keep] += s["residual"][keep].to(F64)
    return (y, z) if case.get("keep", False) else y


def _exact_backward(s):
    case = s["case"]
    keep = torch.ones(case["T"], dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    x, w, d = s["x"][keep].to(F64), s["w"].to(F64), s["dout"][keep].to(F64)
    if case["act"] == "gelu":
        z = s["z"][keep].to(F64).requires_grad_(True)
        d = torch.autograd.grad((z * _phi(z)).sum(), z)[0] * d
    dx = torch.zeros(case["T"], case["cols"], device="cuda", dtype=F64)
    dx[keep] = torch.mm(d, w)
    r = dict(dx=dx, dw=torch.mm(d.T, x))
    if case["bias"]:
        r["dbias"] = d.sum(0)
    return r


def _exact_norm(s):
    case = s["case"]
    T = case["T"]
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0

    def norm(v, kind, weight, bias):
        mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
        v = weight.to(F64) * (v - mean) / ((v - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt()
        return v if bias is None else v + bias.to(F64)

    z = s["y"][keep].to(F64)
    if case["post"] != "none":
        z = norm(z, case["post"], s["post_weight"], s["post_bias"])
    z = z if s["gate"] is None else s["gate"].to(F64) * z
    out = torch.zeros(T, case["d"], device="cuda", dtype=F64)
    out[keep] = s["x"][keep].to(F64) + z
    u = norm(out[keep], case["pre"], s["pre_weight"], s["pre_bias"])
    scales = _two_to(torch.arange(-126, 121, device="cuda"), F64)
    size = scales[torch.bucketize(u.abs().amax(1), 448 * scales)][:, None]
    # the nearest of the values of 8 bits: steps of 2^-3 of the power of two below, 2^-9 at least
    m = (u / size).abs()
    step = torch.pow(2.0, torch.floor(torch.log2(m.clamp(min=2.0 ** -6))) - 3)
    full = torch.zeros_like(out)
    full[keep] = torch.sign(u) * torch.round(m / step) * step * size
    return dict(out=out, u=full)


def _exact_few(s):
    case = s["case"]
    T, B = case["T"], case["B"]
    x = s["x"].to(F64)
    if s["mask"] is not None:
        x[s["mask"] == 0] = 0
    K = case["K"]
    z = (x @ s["router"].to(F64).T).tolist()
    bias = s["router_bias"].tolist()
    tau = (B - 1) / B ** 2
    y = torch.zeros(T, case["d"], device="cuda", dtype=F64)
    w = torch.zeros(T, K + 1, B, dtype=F64)
    for t in range(T):
        if s["mask"] is not None and not s["mask"][t]:
            continue
        alpha = tau + (1 - 2 * tau) / (1 + math.exp(-z[t][0] - bias[0]))
        b = min(max(round(B * alpha), 0), B)
        u = z[t][1 + K:]
        shared = range(b) if case["prefix"] else sorted(range(B), key=lambda j: (-u[j], j))[:b]
        rest = [j for j in range(B) if j not in shared]
        logits = [z[t][1 + e] + bias[1 + e] for e in range(K)]
        total = sum(math.exp(v) for v in logits)
        order = sorted(range(K), key=lambda e: (-logits[e], e))
        beta = 1 - alpha if case["beta"] < 0 else case["beta"]
        w[t, 0, list(shared)] = alpha
        mass = 0.0
        for i, e in enumerate(order):
            p = math.exp(logits[e]) / total
            w[t, 1 + e, rest] = p
            mass += p
            if i + 1 == case["topk"] or (not case["topk"] and mass >= beta):
                break
    w = w.cuda()
    for e in range(K + 1):
        a = x @ s["up"][e].to(F64).T
        h = a * _phi(a) * w[:, e].repeat_interleave(case["H"] // B, 1)
        y += h @ s["down"][e].to(F64).T
    return y


def exact(case, seed):
    s = prepare(case, seed)
    return {"few": _exact_few, "norm_fp8": _exact_norm, "linear_backward": _exact_backward}.get(
        case["call"], _exact_linear)(s)
