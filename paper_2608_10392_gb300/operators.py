"""Operators round the layer: the handle-free entry points of include/unif_moe.h on
torch tensors. A compiled module (csrc/binding.cpp) checks the tensors, allocates
the outputs and calls; there is no fallback, and without it every call raises.
Work goes to `stream` (the tensors' device's current one by default): with another
one the caller orders the streams and keeps the inputs until their use has ended;
outputs belong to it. Padding masks are uint8 or bool.

Nothing here records for autograd. Results are constants to it, whatever their
inputs require: gradients are what backward() and balance_loss()["dlogits"] return,
and balance_loss()["loss"] added to another loss adds a number, no gradient.

    norm = BlockNorm(1024, stream_dtype="f32", branch_dtype="bf16", post_norm="rms", pre_norm="rms")
    r = norm.forward(x, y, post_weight=g1, pre_weight=g2, stats=True)   # r["out"], r["u"], ...
    g = norm.backward(r["out"], y, r, dout=dout, du=du, post_weight=g1, pre_weight=g2)
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import math
import os
from typing import NamedTuple, Optional

import torch

__all__ = ["BlockNorm", "balance_loss", "Mxfp4", "mxfp4_quantize", "mxfp4_dequantize",
           "mxfp4_product", "mxfp4_status", "Fp8", "fp8_quantize",
           "fp8_dequantize", "linear", "linear_backward", "linear_status", "router_table", "few_tokens",
           "FEW_TOKENS"]

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_CODES = {torch.float32: 0, torch.bfloat16: 1}
_ACTIVATIONS = {"none": 0, "gelu": 1}
_NORMS = {"none": 0, "layer": 1, "rms": 2}


class _BlockNormDesc(C.Structure):
    _fields_ = [("tokens", C.c_int), ("width", C.c_int), ("stream_dtype", C.c_int),
                ("branch_dtype", C.c_int), ("post_norm", C.c_int), ("pre_norm", C.c_int),
                ("gate_rows", C.c_int), ("res_scale", C.c_float), ("eps", C.c_float)]


class _LinearDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int), ("n", C.c_int), ("in_dtype", C.c_int),
                ("out_dtype", C.c_int), ("bias_dtype", C.c_int), ("activation", C.c_int)]


class _LinearGrad(C.Structure):
    _fields_ = [("x", C.c_void_p), ("w", C.c_void_p), ("dout", C.c_void_p), ("z", C.c_void_p),
                ("ld_x", C.c_int64), ("ld_w", C.c_int64), ("ld_dout", C.c_int64),
                ("ld_z", C.c_int64), ("dout_dtype", C.c_int), ("grad_dtype", C.c_int),
                ("mask", C.c_void_p), ("dx", C.c_void_p), ("ld_dx", C.c_int64), ("dw", C.c_void_p),
                ("ld_dw", C.c_int64), ("dbias", C.c_void_p)]


class _FewDesc(C.Structure):
    _fields_ = [("tokens", C.c_int), ("d_model", C.c_int), ("d_ff", C.c_int),
                ("n_experts", C.c_int), ("n_blocks", C.c_int), ("tau", C.c_float),
                ("alpha_fixed", C.c_float), ("beta_fixed", C.c_float), ("topk_fixed", C.c_int),
                ("prefix_blocks", C.c_int)]


EXPORTS = ["unif_moe_block_norm_forward", "unif_moe_block_norm_workspace",
           "unif_moe_block_norm_backward", "unif_moe_balance_workspace", "unif_moe_balance_loss",
           "unif_moe_mxfp4_quantize", "unif_moe_mxfp4_dequantize", "unif_moe_mxfp4_product",
           "unif_moe_block_norm_forward_fp8", "unif_moe_fp8_quantize", "unif_moe_fp8_dequantize",
           "unif_moe_linear_workspace", "unif_moe_linear_forward",
           "unif_moe_linear_backward_workspace", "unif_moe_linear_backward",
           "unif_moe_router_table", "unif_moe_few_workspace", "unif_moe_few_forward",
           "unif_moe_forward_few_workspace", "unif_moe_forward_few"]
FEW_TOKENS = 64


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
    L.unif_moe_block_norm_forward_fp8.argtypes = ([D, P, I64, P, I64] + [P] * 6 + [P, I64, P, I64, P]
                                                  + [P] * 5)
    L.unif_moe_fp8_quantize.argtypes = [P, I, I64, I, I64, P, I64, P, P]
    L.unif_moe_fp8_dequantize.argtypes = [P, I64, P, I64, I, P, I, I64, P]
    Q, G = C.POINTER(_LinearDesc), C.POINTER(_LinearGrad)
    L.unif_moe_linear_workspace.argtypes = [Q, P, I64, P, I64]
    L.unif_moe_linear_forward.argtypes = ([Q, P, I64, P, P, I64, P, P, P, I64, P, P, I64, P, I64, P, I64,
                                           P, P])
    L.unif_moe_linear_backward_workspace.argtypes = [Q, G]
    L.unif_moe_linear_backward.argtypes = [Q, G, P, I64, P, P]
    F = C.POINTER(_FewDesc)
    L.unif_moe_router_table.argtypes = [I, I, I, I, P, P, P, P]
    L.unif_moe_few_workspace.argtypes = [F]
    L.unif_moe_few_forward.argtypes = [F, P, I64] + [P] * 6 + [I64, P, P, P, I64, P]
    L.unif_moe_forward_few_workspace.argtypes = [P, I]
    L.unif_moe_forward_few.argtypes = [P, P, I64, I, P, P, I64, P, P, P, I64, P]
    for name in EXPORTS:
        getattr(L, name).restype = I64 if name.endswith("_workspace") else C.c_int


BINDING_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "_binding.so")

_module = None


def _b():
    """The compiled module (built by __graft_entry__.build()); raises if absent."""
    global _module
    if _module is None:
        from . import UnifMoeError, lib
        lib()
        if not os.path.exists(BINDING_PATH):
            raise RuntimeError("_binding.so not built (%s); run __graft_entry__.build()"
                               % BINDING_PATH)
        spec = importlib.util.spec_from_file_location("_binding", BINDING_PATH)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        m.set_errors(UnifMoeError, torch.OutOfMemoryError)
        _module = m
    return _module


class BlockNorm:
    """The step between two blocks of a Transformer: the norm after a block, the
    block's gate, the scaled residual sum and the norm before the next block.

        z = N_post(y),  out = res_scale x + gate z,  u = N_pre(out)

    x, out: the residual stream [T][width] (stream_dtype "f32" or "bf16"); y, u and
    all parameters: branch_dtype. post_norm and pre_norm: "none", "layer" or
    "rms". gate_rows consecutive tokens share a row of the gate (0: all of them).
    Rows of the tensors may be strided; masked rows (mask 0) are not read and
    give 0. u_format "fp8": u in 8 bits (an Fp8, from the unrounded sum), for linear;
    the backward is the same, as if nothing had been rounded."""

    def __init__(self, width: int, stream_dtype: str = "bf16", branch_dtype: str = "bf16",
                 post_norm: str = "none", pre_norm: str = "rms", gate_rows: int = 0,
                 res_scale: float = 1.0, eps: float = 1e-6, u_format: str = "branch"):
        if u_format not in ("branch", "fp8"):
            raise ValueError("u_format: %r (branch or fp8)" % (u_format,))
        self.eight = u_format == "fp8"
        self.width, self.gate_rows = width, gate_rows
        self.post, self.pre = _NORMS[post_norm], _NORMS[pre_norm]
        self._desc = (width, _CODES[DTYPES[stream_dtype]], _CODES[DTYPES[branch_dtype]], self.post,
                      self.pre, gate_rows, res_scale, eps)

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, *,
                post_weight: Optional[torch.Tensor] = None,
                post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                pre_weight: Optional[torch.Tensor] = None,
                pre_bias: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, u=None,
                stats: bool = False, stream=None) -> dict:
        """dict of out (x itself without y), u (None without pre norm) and, where
        `stats` asks for them, the statistics post_mean, post_rstd, pre_mean,
        pre_rstd [T] that backward takes (None for a norm that is not there; means of
        an rms norm are 0). Without y: the norm before a stack's first block."""
        if self.eight:
            if u is not None and not isinstance(u, Fp8):
                raise ValueError("u: need an Fp8, got %s" % type(u).__name__)
            codes, scales = (None, None) if u is None else (u.codes, u.scales)
            r = _b().norm_forward_fp8(self._desc, x, y, post_weight, post_bias, gate, pre_weight,
                                      pre_bias, mask, out, codes, stats, stream, scales)
            r["u"] = Fp8(r["u"], r.pop("u_scales"))
            return r
        return _b().norm_forward(self._desc, x, y, post_weight, post_bias, gate, pre_weight,
                                 pre_bias, mask, out, u, stats, stream)

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
        post, pre = self.post, self.pre
        return _b().norm_backward(
            self._desc, out, y, stats["post_mean"] if post == 1 else None,
            stats["post_rstd"] if post else None, stats["pre_mean"] if pre == 1 else None,
            stats["pre_rstd"] if pre else None, dout, du, post_weight, post_bias, gate, pre_weight,
            mask, stream)


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
    return _b().balance(logits, q, k, mask, balance_weight, z_weight, grad, stream)


class Mxfp4(NamedTuple):
    """Rows in microscaled 4-bit floating point: codes [...][16 ceil(cols / 32)] uint8
    (two elements a byte, the even column in the low half), scales
    [...][8 ceil(cols / 256)] uint8 (byte b: columns 32 b .. 32 b + 31 by 2^(byte - 127)),
    both contiguous."""
    codes: torch.Tensor
    scales: torch.Tensor
    cols: int


def mxfp4_quantize(x: torch.Tensor, out: Optional[Mxfp4] = None, stream=None) -> Mxfp4:
    """Rows x [...][cols] (fp32 or bf16; a 2-d x may have strided rows) to 4 bits: a
    block of 32 columns shares the scale 2^e, e = floor(log2 max |x|) - 2, elements
    round to nearest even and saturate at 6 2^e."""
    if out is None:
        return Mxfp4(*_b().quantize(x, None, None, None, stream))
    _b().quantize(x, out.codes, out.scales, out.cols, stream)
    return out


def mxfp4_dequantize(q: Mxfp4, dtype: str = "bf16", out: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """The values of rows in 4 bits, [...][cols] ("bf16" or "f32"); an out
    [rows][cols] may have strided rows."""
    return _b().dequantize(q.codes, q.scales, q.cols, _CODES[DTYPES[dtype]], out, stream)


_status_words = {}  # per device: set by a product whose kernel gave up a wait


def _status_word(device: torch.device) -> torch.Tensor:
    t = _status_words.get(device)
    if t is None:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the first product on a device has to be outside a capture")
        t = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.current_stream(device).synchronize()  # products may be on another stream
        _status_words[device] = t
    return t


def mxfp4_status(device=None) -> int:
    """Waits for the device and returns ERR_TIMEOUT (-5) if the kernel of a product (mxfp4_product,
    linear, linear_backward) gave up a wait since the last call (its output is incomplete),
    else 0. linear_status is the same."""
    device = torch.device("cuda" if device is None else device)
    torch.cuda.synchronize(device)  # (raises for other devices)
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    word = _status_word(device)
    bad = int(word.item()) != 0
    word.zero_()
    torch.cuda.synchronize(device)  # a later product may be on another stream
    return -5 if bad else 0


def mxfp4_product(a: Mxfp4, w: Mxfp4, offsets: Optional[torch.Tensor] = None, *,
                  activation: str = "none", dtype: str = "bf16",
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[r] = act(W_g a[r]) for the rows r of group g, [rows][n] ("bf16" or "f32").

    a: rows in 4 bits; w: codes [groups][n][...] or [n][...] (one group); offsets
    [groups + 1] int32 on the GPU: group g has the rows offsets[g] .. offsets[g + 1] - 1
    (None with one group: all rows; e.g. the offsets of Layer.groups()). Rows of no group
    are not written. activation: "none" or "gelu"."""
    return _b().product(a.codes, a.scales, a.cols, w.codes, w.scales, w.cols, offsets,
                        _ACTIVATIONS[activation], _CODES[DTYPES[dtype]], out,
                        _status_word(a.codes.device) if a.codes.is_cuda else None, stream)


linear_status = mxfp4_status


class Fp8(NamedTuple):
    """Rows in 8-bit floating point (E4M3) under a scale each: a value is its code times the
    scale of its row. codes [...][cols] float8_e4m3fn with dense rows (those of a 2-d tensor may be
    strided), scales [...] fp32, contiguous."""
    codes: torch.Tensor
    scales: torch.Tensor


def fp8_quantize(x: torch.Tensor, out: Optional[Fp8] = None, stream=None) -> Fp8:
    """Rows x [...][cols] (fp32 or bf16; a 2-d x may have strided rows) to 8 bits: a row's scale is
    2^e, the smallest for which no value is above 448 2^e, codes round to nearest even. New
    codes have rows a multiple of 16 bytes apart, which linear reads as they are."""
    if out is None:
        return Fp8(*_b().fp8_quantize(x, None, None, stream))
    _b().fp8_quantize(x, out.codes, out.scales, stream)
    return out


def fp8_dequantize(q: Fp8, dtype: str = "bf16", out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The values of rows in 8 bits, [...][cols] ("bf16" or "f32"); an out [rows][cols] may
    have strided rows."""
    return _b().fp8_dequantize(q.codes, q.scales, _CODES[DTYPES[dtype]], out, stream)


def _status_of(x):
    return _status_word(x.device) if isinstance(x, torch.Tensor) and x.is_cuda else None


def linear(x, w, bias: Optional[torch.Tensor] = None, *, activation: str = "none",
           residual: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
           dtype: str = "bf16", keep: bool = False, out: Optional[torch.Tensor] = None, stream=None):
    """out = residual + act(x w^T + bias), [T][n] ("bf16" or "f32"): one kernel, the sum rounded
    once.

    x [T][cols] and w [n][cols] both bf16 or both Fp8 (rows under a scale each); rows of all
    2-d tensors may be strided, with any alignment. bias [n] fp32 or bf16; residual [T][n] of
    the result's dtype (out may be it, and shares memory with nothing else); activation "none" or "gelu"; mask [T]: 0 marks padding,
    whose rows give 0. keep: also z = x w^T + bias in bf16, (out, z), for linear_backward.

    Measured beside the library's plain product: the same up to 8 rows and for thousands of
    rows by thousands of columns, 1.2 to 2 times its time between (32 x 1,024 to 4,096 7.2 us and 3.7, 512 8.5 and
    4.9, 2,048 15.0 and 12.2)."""
    if isinstance(x, Fp8) != isinstance(w, Fp8):
        raise ValueError("x and w: need both in 8 bits or neither")
    xc, xs, wc, ws = (x.codes, x.scales, w.codes, w.scales) if isinstance(x, Fp8) else (x, None, w, None)
    return _b().linear(xc, xs, wc, ws, bias, _ACTIVATIONS[activation], residual, mask,
                       _CODES[DTYPES[dtype]], keep, out, _status_of(xc), stream)


def linear_backward(x: torch.Tensor, w: torch.Tensor, dout: torch.Tensor,
                    z: Optional[torch.Tensor] = None, *, activation: str = "none",
                    mask: Optional[torch.Tensor] = None, bias: bool = False, dx: bool = True,
                    dw: bool = True, grad_dtype: str = "f32", stream=None) -> dict:
    """Gradients of linear for bf16 x and w, from that of its result (dout [T][n], fp32 or bf16)
    and its z (with an activation): dict of dx [T][cols] (bf16), dw [n][cols] (grad_dtype),
    dbias [n] (fp32); None for what `dx`, `dw`, `bias` do not ask for. The residual's gradient
    is dout. Padding rows (mask 0) give 0 in dx and take no part in the sums. dz = dout act'(z)
    is rounded to bf16 for the two products."""
    return _b().linear_backward(x, w, dout, z, _ACTIVATIONS[activation], mask, dx, dw, bias,
                                _CODES[DTYPES[grad_dtype]], _status_of(x), stream)


def router_table(w_router: torch.Tensor, w_up: torch.Tensor, n_blocks: int, stream=None) -> torch.Tensor:
    """The router's rows [1 + K + B][d] for few_tokens, made once for a layer's weights: W_shr, W_g
    (w_router [d][K + 1]) and the mean key of each of the n_blocks blocks of the shared expert
    (w_up [K + 1][H][d]); bf16."""
    return _b().router_table(w_router, w_up, n_blocks, stream)


def few_tokens(x: torch.Tensor, router: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
               n_blocks: int, *, router_bias: Optional[torch.Tensor] = None,
               mask: Optional[torch.Tensor] = None, tau: float = math.nan,
               alpha_fixed: float = math.nan, beta_fixed: float = math.nan, topk_fixed: int = 0,
               prefix_blocks: bool = False, shared_counts: Optional[torch.Tensor] = None,
               residual_counts: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """The whole layer for up to FEW_TOKENS tokens x [T][d] (bf16), from the caller's weights: router
    from router_table, w_up [K + 1][H][d], w_down [K + 1][d][H] (contiguous bf16), router_bias
    [K + 1] fp32; thresholds as Layer's. x's rows start at multiples of 16 bytes; out may lie over x. A
    server's step: two or three kernels that read each weight in use once. mask [T]: 0 marks padding, which gives 0. shared_counts, residual_counts [T]
    int32 receive b(x) and k(x). Layer.forward_few does the same with a layer's weights."""
    return _b().few_tokens(x, router, w_up, w_down, n_blocks, router_bias, mask,
                           (tau, alpha_fixed, beta_fixed, topk_fixed, prefix_blocks), shared_counts,
                           residual_counts, out, stream)
