"""The polynomial of the dense products' GELU (csrc/gelu_log.cuh: gelu2) is the fit that its comment
names: degree 8, the same weight everywhere (CPU)."""
import numpy as np

from gelu_fit import _fit_rounded
from gelu_log_fit import LOG2_E_HALF, X_MAX
from test_gelu_log_constants import constants


def test_constants_are_the_fit():
    from scipy.special import erfcx
    x = np.sort((np.cos(np.linspace(0, np.pi, 6002)) - 1) * (X_MAX / 2))[:-1]
    q = np.log2(0.5 * erfcx(-x / np.sqrt(2))) - x * x * LOG2_E_HALF
    fit = _fit_rounded(x, q, np.ones_like(x), 8)
    held = [float(c) for c in constants("gelu_log.cuh", "void gelu2(", "g", 8)]
    # (the last bits of the coefficients are the machine's; the polynomials differ by less than fp32's steps of a
    # power up to 2^7)
    got, want = (np.polynomial.polynomial.polyval(x, c) for c in (held, fit))
    assert np.abs(got - want).max() < 2.0 ** -17
    assert np.abs(want - q).max() < 2.0 ** -12.8 / np.log(2)
