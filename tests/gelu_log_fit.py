"""Generates the polynomial of the 4-bit product's GELU for bf16 results.

GELU(v) = v Phi(v) with Phi the standard normal CDF. With x = -|v|, Phi(x) = 2^Q(x), where
Q(x) = log2(Phi(x)) = log2(erfcx(-x / sqrt 2) / 2) - x^2 / (2 ln 2) is smooth (erfcx(z) =
exp(z^2) erfc(z)); then GELU(v) = max(v, 0) + x Phi(x), which keeps the relative accuracy
of Phi(x) for every negative v. Q is approximated by a polynomial of degree 11 on
[-X_MAX, 0]: its largest error over BOUNDS is the least (Lawson's algorithm), with each
coefficient rounded to fp32 and the rest fitted again to what is left.

Run:  python tests/gelu_log_fit.py   (prints the constants that csrc/fp4_product.cu holds;
tests/test_gelu_product.py checks them)
"""
import numpy as np
from scipy.special import erfcx

from gelu_fit import _fit_rounded

DEG, X_MAX = 11, 13.0
LOG2_E_HALF = 0.72134752044448170  # 1 / (2 ln 2)


def fit():
    """Coefficients of Q, lowest first."""
    x = np.sort((np.cos(np.linspace(0, np.pi, 6002)) - 1) * (X_MAX / 2))[:-1]
    bounds = np.where(x >= -4, 2.0 ** -18, 2.0 ** -12)  # relative errors of Phi
    q = np.log2(0.5 * erfcx(-x / np.sqrt(2))) - x * x * LOG2_E_HALF
    return _fit_rounded(x, q, 1 / bounds, DEG)


def gelu_log(v, coef):
    """The kernel's arithmetic in fp32 (fused multiply-adds rounded once) with an exact 2^."""
    f32, f64 = np.float32, np.float64
    v = v.astype(f32)
    x = np.maximum(-np.abs(v), f32(-X_MAX))
    q = np.full_like(x, f32(coef[-1]))
    for c in coef[-2::-1]:
        q = (q.astype(f64) * x + f64(f32(c))).astype(f32)
    p = np.exp2(q.astype(f64)).astype(f32)
    p[p < f32(2.0 ** -126)] = 0  # a power below fp32's normal range is 0
    return (np.maximum(v, f32(0)).astype(f64) + x.astype(f64) * p).astype(f32)


if __name__ == "__main__":
    from scipy.special import log_ndtr
    coef = fit()
    for k, c in enumerate(coef):
        print("  0x%08x  // q%d = %.9g" % (np.float32(c).view(np.uint32), k, np.float32(c)))
    for lo, hi in ((-12.9, -8), (-8, -4), (-4, -1), (-1, 0), (0, 1), (1, 13)):
        v = np.linspace(lo, hi, 400001).astype(np.float32)
        v = v[v != 0]
        want = v.astype(np.float64) * np.exp(log_ndtr(v.astype(np.float64)))
        print("// v in [%g, %g]: relative error %.2e" % (lo, hi, np.abs(gelu_log(v, coef) / want - 1).max()))
