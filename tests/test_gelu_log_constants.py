"""GELU and its derivative beside the dense products and the few-token layer (csrc/gelu_log.cuh), in
the kernels' arithmetic with an exact 2^ (CPU).

gelu2: |error| <= 2^-12.5 of GELU down to v = -12.9, where Phi leaves fp32's normal range (Phi then
counts as 0, the value below 2e-37). Of Phi the polynomial's own is 2^-12.8; nine multiply-adds of a
power up to 2^6.97 in size add at most 2^-24 2^6.97 ln 2 (1 + 1/2 + ...) < 2^-16.
gelu_grad2: the polynomial of the 4-bit product, Phi within 2^-18 of itself for v >= -4; the
derivative adds v phi(v), a few roundings of 2^-24 and one exponential: within 2^-16 absolute everywhere."""
import os
import re

import numpy as np
from scipy.special import log_ndtr, ndtr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10392_gb300", "csrc")


def constants(path, start, letter, degree):
    src = open(os.path.join(CSRC, path)).read()
    body = src[src.index(start):]
    found = {}
    for bits, k in re.findall(r"UNIF_K2\((0x[0-9a-f]{8})\)\)?;\s*// %s(\d+)" % letter, body):
        found.setdefault(int(k), np.uint32(int(bits, 16)).view(np.float32))
    assert sorted(found) == list(range(degree + 1)), found
    return [found[k] for k in range(degree + 1)]


def test_gelu():
    from gelu_log_fit import gelu_log
    c = constants("gelu_log.cuh", "void gelu2(", "g", 8)
    v = np.concatenate([np.linspace(-12.9, 0, 800001), np.linspace(0, 13, 400001)]).astype(np.float32)
    v = v[v != 0]
    want = v.astype(np.float64) * np.exp(log_ndtr(v.astype(np.float64)))
    assert np.abs(gelu_log(v, c) / want - 1).max() < 2.0 ** -12.5
    v = np.array([-1e30, -40, -14, -13, 0, 14, 40, 1e30, np.inf], dtype=np.float32)
    got = gelu_log(v, c)
    assert np.abs(got[:-1] - np.maximum(v, 0)[:-1]).max() < 2e-36 and got[-1] == np.inf
    assert np.isnan(gelu_log(np.array([np.nan], dtype=np.float32), c)).all()


def test_derivative():
    from gelu_log_fit import DEG
    c = constants("gelu_log.cuh", "void gelu_grad2(", "q", DEG)
    assert c == constants("fp4_product.cu", "uint32_t gelu2(", "q", DEG)
    f32, f64 = np.float32, np.float64
    v = np.linspace(-20, 20, 400001).astype(f32)
    x = np.maximum(-np.abs(v), f32(-13))
    q = np.full_like(x, c[-1])
    for k in c[-2::-1]:
        q = (q.astype(f64) * x + f64(k)).astype(f32)
    p = np.exp2(q.astype(f64)).astype(f32)
    e = np.exp2(((x * x).astype(f32) * f32(-0.72134752044448170)).astype(f64)).astype(f32)
    d = ((x * f32(0.39894228040143268)).astype(f64) * e + p).astype(f32)
    d = np.where(v > 0, f32(1) - d, d)
    z = v.astype(f64)
    want = ndtr(z) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    assert np.abs(d - want).max() < 2.0 ** -16
