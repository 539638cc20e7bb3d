"""Operators round the layer: thin ctypes binding of the handle-free entry points
of include/unif_moe.h, on torch tensors of the current device.

    norm = BlockNorm(1024, stream_dtype="f32", branch_dtype="bf16", post_norm="rms", pre_norm="rms")
    r = norm.forward(x, y, post_weight=g1, pre_weight=g2, stats=True)   # r["out"], r["u"], ...
    g = norm.backward(r["out"], y, r, dout=dout, du=du, post_weight=g1, pre_weight=g2)
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

__all__ = ["BlockNorm", "balance_loss", "Mxfp4", "mxfp4_quantize", "mxfp4_dequantize",
           "mxfp4_product", "mxfp4_status"]

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_CODES = {torch.float32: 0, torch.bfloat16: 1}
_ACTIVATIONS = {"none": 0, "gelu": 1}
_NORMS = {"none": 0, "layer": 1, "rms": 2}


class _BlockNormDesc(C.Structure):
    _fields_ = [("tokens", C.c_int), ("width", C.c_int), ("stream_dtype", C.c_int),
                ("branch_dtype", C.c_int), ("post_norm", C.c_int), ("pre_norm", C.c_int),
                ("gate_rows", C.c_int), ("res_scale", C.c_float), ("eps", C.c_float)]


EXPORTS = ["unif_moe_block_norm_forward", "unif_moe_block_norm_workspace",
           "unif_moe_block_norm_backward", "unif_moe_balance_workspace", "unif_moe_balance_loss",
           "unif_moe_mxfp4_quantize", "unif_moe_mxfp4_dequantize", "unif_moe_mxfp4_product"]


def declare(L: C.CDLL) -> None:
    """Argument and result types of the entry points."""
    P, I, I64 = C.c_void_p, C.c_int, C.c_int64
    D = C.POINTER(_BlockNormDesc)
    L.unif_moe_block_norm_forward.argtypes = ([D, P, I64, P, I64] + [P] * 6 + [P, I64, P, I64]
                                              + [P] * 5)
    L.unif_moe_block_norm_workspace.argtypes = [D, I]
    L.unif_moe_block_norm_backward.argtypes = ([D, P, I64, P, I64] + [P] * 9 + [P, I64] * 4
                                               + [P] * 6 + [I64, P])
    L.unif_moe_balance_workspace.argtypes = [I, I]
    L.unif_moe_balance_loss.argtypes = ([I, I, P, I, I64, P, I, I64, P, P, C.c_float, C.c_float]
                                        + [P] * 5 + [I64, P])
    L.unif_moe_mxfp4_quantize.argtypes = [P, I, I64, I, I64, P, P, P]
    L.unif_moe_mxfp4_dequantize.argtypes = [P, P, I64, I, P, I, I64, P]
    L.unif_moe_mxfp4_product.argtypes = [P, P, I64, I, P, P, I, I, P, I, P, I, I64, P, P]
    for name in EXPORTS:
        getattr(L, name).restype = I64 if name.endswith("_workspace") else C.c_int


_loaded = None


def _lib() -> C.CDLL:
    global _loaded
    if _loaded is None:
        from . import lib
        _loaded = lib()
    return _loaded


def _check(rc: int):
    if rc != 0:
        from . import _check as check
        check(rc)


def _stream(stream):
    if stream is None:  # the current stream's handle, without making a Stream object (3 us)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _rows(t: Optional[torch.Tensor], name: str, rows: int, width: int, dtype: torch.dtype):
    """(pointer, row stride) of a [rows][width] CUDA tensor whose rows are dense."""
    if t is None:
        return None, 0
    at = t.stride()
    if t.dtype is not dtype or t.shape != (rows, width) or not t.is_cuda \
            or (at[1] != 1 and width > 1):
        raise ValueError("%s: need a CUDA tensor [%d][%d] of %s with dense rows, got %s %s"
                         % (name, rows, width, dtype, tuple(t.shape), t.dtype))
    return t.data_ptr(), (at[0] if rows > 1 else max(at[0], width))


def _dense(t: Optional[torch.Tensor], name: str, count: int, dtype: torch.dtype):
    """Pointer of a contiguous CUDA tensor of `count` elements."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != count or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s: need a contiguous CUDA tensor of %d elements of %s, got %s %s"
                         % (name, count, dtype, tuple(t.shape), t.dtype))
    return t.data_ptr()


def _mask(mask: Optional[torch.Tensor], T: int):
    if mask is not None and mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    return _dense(mask, "mask", T, torch.uint8)


class BlockNorm:
    """The step between two blocks of a Transformer: the norm after a block, the
    block's gate, the scaled residual sum and the norm before the next block.

        z = N_post(y),  out = res_scale x + gate z,  u = N_pre(out)

    x, out: the residual stream [T][width] (stream_dtype "f32" or "bf16"); y, u and
    all parameters: branch_dtype. post_norm and pre_norm: "none", "layer" or
    "rms". gate_rows consecutive tokens share a row of the gate (0: all of them).
    Rows of the tensors may be strided; masked rows (mask 0) are not read and
    give 0."""

    def __init__(self, width: int, stream_dtype: str = "bf16", branch_dtype: str = "bf16",
                 post_norm: str = "none", pre_norm: str = "rms", gate_rows: int = 0,
                 res_scale: float = 1.0, eps: float = 1e-6):
        self.width, self.gate_rows = width, gate_rows
        self.stream, self.branch = DTYPES[stream_dtype], DTYPES[branch_dtype]
        self.post, self.pre = _NORMS[post_norm], _NORMS[pre_norm]
        self._args = (width, _CODES[self.stream], _CODES[self.branch], self.post, self.pre,
                      gate_rows, res_scale, eps)

    def _params(self, T, post_weight, post_bias, gate, pre_weight, pre_bias=None):
        d, tb = self.width, self.branch
        rows = 1 if self.gate_rows == 0 else -(-T // self.gate_rows)
        return (_dense(post_weight, "post_weight", d, tb), _dense(post_bias, "post_bias", d, tb),
                _dense(gate, "gate", rows * d, tb), _dense(pre_weight, "pre_weight", d, tb),
                _dense(pre_bias, "pre_bias", d, tb))

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, *,
                post_weight: Optional[torch.Tensor] = None,
                post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                pre_weight: Optional[torch.Tensor] = None,
                pre_bias: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None,
                stats: bool = False, stream=None) -> dict:
        """dict of out (x itself without y), u (None without pre norm) and, where
        `stats` asks for them, the statistics post_mean, post_rstd, pre_mean,
        pre_rstd [T] that backward takes. Without y: the norm before a stack's
        first block."""
        T, d = x.shape[0], self.width
        dev = x.device
        if y is not None and out is None:
            out = torch.empty(T, d, dtype=self.stream, device=dev)
        if self.pre and u is None:
            u = torch.empty(T, d, dtype=self.branch, device=dev)
        saved = torch.empty(4, T, dtype=torch.float32, device=dev) if stats else None
        px, ldx = _rows(x, "x", T, d, self.stream)
        py, ldy = _rows(y, "y", T, d, self.branch)
        po, ldo = _rows(out, "out", T, d, self.stream)
        pu, ldu = _rows(u, "u", T, d, self.branch)
        at = (None,) * 4
        if stats:
            s0 = saved.data_ptr()
            at = (s0, s0 + 4 * T, s0 + 8 * T, s0 + 12 * T)
        _check(_lib().unif_moe_block_norm_forward(
            _BlockNormDesc(T, *self._args), px, ldx, py, ldy, _mask(mask, T),
            *self._params(T, post_weight, post_bias, gate, pre_weight, pre_bias), po, ldo, pu, ldu,
            *at, _stream(stream)))
        r = dict(out=x if y is None else out, u=u)
        if stats:
            r.update(zip(("post_mean", "post_rstd", "pre_mean", "pre_rstd"), saved.unbind(0)))
        return r

    def backward(self, out: Optional[torch.Tensor], y: Optional[torch.Tensor], stats: dict, *,
                 dout: Optional[torch.Tensor] = None, du: Optional[torch.Tensor] = None,
                 post_weight: Optional[torch.Tensor] = None,
                 post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                 pre_weight: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                 stream=None) -> dict:
        """Gradients from those of out (None: none) and u, and the forward's out
        (x in the form without y), y and statistics: dict of dx (stream_dtype), dy
        (branch_dtype; None without y) and, in fp32, those of the parameters that
        there are: d_post_weight, d_post_bias, d_gate, d_pre_weight, d_pre_bias."""
        ref = du if dout is None else dout
        if ref is None:
            raise ValueError("dout and du are both None")
        T, d = ref.shape[0], self.width
        dev = ref.device
        L, desc = _lib(), _BlockNormDesc(T, *self._args)
        dx = torch.empty(T, d, dtype=self.stream, device=dev)
        dy = None if y is None else torch.empty(T, d, dtype=self.branch, device=dev)
        need = L.unif_moe_block_norm_workspace(desc, int(gate is not None))
        if need < 0:
            _check(-1)
        # one allocation: the parameters' gradients, each at 16 bytes, and the workspace
        names = (["d_post_weight", "d_post_bias"] if self.post else []) \
            + (["d_pre_weight", "d_pre_bias"] if self.pre else [])
        step = -(-d // 4) * 4
        gates = 0 if gate is None else gate.numel()
        g0 = len(names) * step
        w0 = g0 + -(-gates // 4) * 4
        flat = torch.empty(w0 + need // 4, dtype=torch.float32, device=dev)
        base = flat.data_ptr()
        at = {n: base + 4 * step * i for i, n in enumerate(names)}
        po, ldo = _rows(out, "out", T, d, self.stream) if self.pre else (None, 0)
        py, ldy = _rows(y, "y", T, d, self.branch)
        pdo, lddo = _rows(dout, "dout", T, d, self.stream)
        pdu, lddu = _rows(du, "du", T, d, self.branch)
        F, m1, r1, m2, r2 = torch.float32, None, None, None, None
        if self.post:
            r1 = _dense(stats["post_rstd"], "post_rstd", T, F)
            if self.post == 1:  # a layer norm's mean
                m1 = _dense(stats["post_mean"], "post_mean", T, F)
        if self.pre:
            r2 = _dense(stats["pre_rstd"], "pre_rstd", T, F)
            if self.pre == 1:
                m2 = _dense(stats["pre_mean"], "pre_mean", T, F)
        _check(L.unif_moe_block_norm_backward(
            desc, po, ldo, py, ldy, _mask(mask, T),
            *self._params(T, post_weight, post_bias, gate, pre_weight)[:4], m1, r1, m2, r2,
            pdo, lddo, pdu, lddu, dx.data_ptr(), d, None if dy is None else dy.data_ptr(), d,
            at.get("d_post_weight"), at.get("d_post_bias"),
            None if gate is None else base + 4 * g0, at.get("d_pre_weight"), at.get("d_pre_bias"),
            base + 4 * w0, need, _stream(stream)))
        # (as_strided makes a view in a third of the time of a slice and a view)
        r = {n: flat.as_strided((d,), (1,), i * step) for i, n in enumerate(names)}
        r["dx"], r["dy"] = dx, dy
        if gate is not None:
            r["d_gate"] = flat.as_strided((gates // d, d), (d, 1), g0)
        return r


def balance_loss(logits: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None, *,
                 mask: Optional[torch.Tensor] = None, balance_weight: float = 0.01,
                 z_weight: float = 0.0, grad: bool = True, stream=None) -> dict:
    """Balance and z losses of a router and the gradient of its logits: dict of
    loss [3] (weighted sum, balance, z), counts [K] (how often each expert was
    selected, int32), prob [K] (mean probabilities) and dlogits [T][K] (fp32; None
    without grad).

    logits [T][K] fp32 or bf16, rows may be strided; q [T][n] int32: the experts of
    a token, of which the first k[t] count (all without k): Layer.routing()'s q
    with the forward's residual_counts; mask [T]: 0 marks padding."""
    T, K = logits.shape
    dev = logits.device
    if logits.dtype not in _CODES:
        raise ValueError("logits: fp32 or bf16, got %s" % logits.dtype)
    pz, ld = _rows(logits, "logits", T, K, logits.dtype)
    n_q = q.shape[1]
    pq, ld_q = _rows(q, "q", T, n_q, torch.int32)
    L = _lib()
    need = L.unif_moe_balance_workspace(T, K)
    if need < 0:
        _check(-1)
    # one allocation: loss and prob, each at 16 bytes, and the workspace
    step = -(-K // 4) * 4
    flat = torch.empty(4 + step + need // 4, dtype=torch.float32, device=dev)
    counts = torch.empty(K, dtype=torch.int32, device=dev)
    at = flat.data_ptr()
    d = torch.empty(T, K, dtype=torch.float32, device=dev) if grad else None
    _check(L.unif_moe_balance_loss(
        T, K, pz, _CODES[logits.dtype], ld, pq, n_q, ld_q, _dense(k, "k", T, torch.int32),
        _mask(mask, T), balance_weight, z_weight, at, counts.data_ptr(), at + 16,
        None if d is None else d.data_ptr(), at + 16 + 4 * step, need, _stream(stream)))
    return dict(loss=flat.as_strided((3,), (1,)), counts=counts,
                prob=flat.as_strided((K,), (1,), 4), dlogits=d)


class Mxfp4(NamedTuple):
    """Rows in microscaled 4-bit floating point: codes [...][16 ceil(cols / 32)] uint8
    (two elements a byte, the even column in the low half), scales
    [...][8 ceil(cols / 256)] uint8 (byte b: columns 32 b .. 32 b + 31 by 2^(byte - 127)),
    both contiguous."""
    codes: torch.Tensor
    scales: torch.Tensor
    cols: int


def _mxfp4(t: Mxfp4, name: str):
    """(codes' pointer, scales' pointer, rows) of rows in 4 bits."""
    codes, scales, cols = t
    per, pitch = (cols + 31) // 32 * 16, (cols + 255) // 256 * 8
    if cols < 1 or codes.dim() < 1 or codes.shape[-1] != per:
        raise ValueError("%s: codes of %d columns are %d bytes a row, got %s"
                         % (name, cols, per, tuple(codes.shape)))
    rows = codes.numel() // per
    return (_dense(codes, name + ".codes", rows * per, torch.uint8),
            _dense(scales, name + ".scales", rows * pitch, torch.uint8), rows)


def mxfp4_quantize(x: torch.Tensor, out: Optional[Mxfp4] = None, stream=None) -> Mxfp4:
    """Rows x [...][cols] (fp32 or bf16; a 2-d x may have strided rows) to 4 bits: a
    block of 32 columns shares the scale 2^e, e = floor(log2 max |x|) - 2, elements
    round to nearest even and saturate at 6 2^e."""
    lead, cols = x.shape[:-1], x.shape[-1]
    if x.dim() != 2:
        if not x.is_contiguous():
            raise ValueError("x: more than two dimensions need a contiguous tensor")
        x = x.view(-1, cols)
    rows = x.shape[0]
    if x.dtype not in _CODES:
        raise ValueError("x: fp32 or bf16, got %s" % x.dtype)
    px, ld = _rows(x, "x", rows, cols, x.dtype)
    per, pitch = (cols + 31) // 32 * 16, (cols + 255) // 256 * 8
    if out is None:
        codes = torch.empty(*lead, per, dtype=torch.uint8, device=x.device)
        scales = torch.empty(*lead, pitch, dtype=torch.uint8, device=x.device)
        out = Mxfp4(codes, scales, cols)
        pc, ps = codes.data_ptr(), scales.data_ptr()
    else:
        pc, ps, n = _mxfp4(out, "out")
        if out.cols != cols or n != rows:
            raise ValueError("out: %d rows of %d columns, need %d of %d" % (n, out.cols, rows, cols))
    _check(_lib().unif_moe_mxfp4_quantize(px, _CODES[x.dtype], rows, cols, ld, pc, ps,
                                          _stream(stream)))
    return out


def mxfp4_dequantize(q: Mxfp4, dtype: str = "bf16", out: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """The values of rows in 4 bits, [...][cols] ("bf16" or "f32"); a 2-d out may have
    strided rows."""
    pc, ps, rows = _mxfp4(q, "q")
    if out is None:
        out = torch.empty(*q.codes.shape[:-1], q.cols, dtype=DTYPES[dtype], device=q.codes.device)
        po, ld = out.data_ptr(), q.cols
    else:
        po, ld = _rows(out, "out", rows, q.cols, DTYPES[dtype])
    _check(_lib().unif_moe_mxfp4_dequantize(pc, ps, rows, q.cols, po, _CODES[DTYPES[dtype]], ld,
                                            _stream(stream)))
    return out


_status_words = {}  # per device: set by a product whose kernel gave up a wait


def _status_word(device: torch.device) -> torch.Tensor:
    t = _status_words.get(device)
    if t is None:
        t = _status_words[device] = torch.zeros(1, dtype=torch.int32, device=device)
    return t


def mxfp4_status(device=None) -> int:
    """Waits for the device and returns ERR_TIMEOUT (-5) if a product's kernel gave up a
    wait since the last call (its output is incomplete), else 0."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None \
        else torch.device(device)
    torch.cuda.synchronize(device)
    word = _status_word(device)
    bad = int(word.item()) != 0
    word.zero_()
    return -5 if bad else 0


def mxfp4_product(a: Mxfp4, w: Mxfp4, offsets: Optional[torch.Tensor] = None, *,
                  activation: str = "none", dtype: str = "bf16",
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[r] = act(W_g a[r]) for the rows r of group g, [rows][n] ("bf16" or "f32").

    a: rows in 4 bits; w: codes [groups][n][...] or [n][...] (one group); offsets
    [groups + 1] int32 on the GPU: group g has the rows offsets[g] .. offsets[g + 1] - 1
    (None with one group: all rows; e.g. the offsets of Layer.groups()). Rows of no group
    are not written. activation: "none" or "gelu"."""
    pa, psa, rows = _mxfp4(a, "a")
    pw, psw, wn = _mxfp4(w, "w")
    if a.cols != w.cols:
        raise ValueError("a has %d columns, w %d" % (a.cols, w.cols))
    n = w.codes.shape[-2] if w.codes.dim() > 1 else 1
    groups = wn // n if n else 0
    if offsets is None and groups != 1:
        raise ValueError("offsets: needed with %d groups" % groups)
    dev = a.codes.device
    if out is None:
        out = torch.empty(rows, n, dtype=DTYPES[dtype], device=dev)
        po, ld = out.data_ptr(), n
    else:
        po, ld = _rows(out, "out", rows, n, DTYPES[dtype])
    _check(_lib().unif_moe_mxfp4_product(
        pa, psa, rows, a.cols, pw, psw, n, groups, _dense(offsets, "offsets", groups + 1, torch.int32),
        _ACTIVATIONS[activation], po, _CODES[DTYPES[dtype]], ld, _status_word(dev).data_ptr(),
        _stream(stream)))
    return out
