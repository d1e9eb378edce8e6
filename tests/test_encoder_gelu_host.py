"""The normal distribution that gelu of 16-bit results is formed with, from the coefficients that the kernels have, against
erfc: the fit in 64 bits, and as it is evaluated in float."""
import os
import re

import numpy as np
import pytest

from conftest import ROOT

erfc = pytest.importorskip("scipy.special").erfc


@pytest.fixture(scope="module")
def fit():
    """(factor of t, coefficients from the highest power)."""
    with open(os.path.join(ROOT, "paper_2607_03574_amd", "csrc", "product.h")) as f:
        body = f.read().split("sizeof(T) == 2) {", 1)[1].split("q = q * t * e;", 1)[0]
    factor = float(re.search(r"rcpf\(1\.0f \+ ([\d.]+)f \* fabsf", body).group(1))
    first = float(re.search(r"float q = ([\d.]+)f;", body).group(1))
    rest = [float(sign + v) for sign, v in re.findall(r"q = q \* t ([+-]) ([\d.]+)f;", body)]
    assert len(rest) == 6
    return factor, [first, *rest]


def test_fit(fit):
    x = np.linspace(0.0, 13.0, 100001)
    t = 1.0 / (1.0 + fit[0] * x)
    found = np.polyval(fit[1], t) * t * np.exp(-0.5 * x * x)
    want = 0.5 * erfc(x * 0.5 ** 0.5)
    assert np.max(np.abs(found / want - 1.0)) <= 9.2e-7


def test_fit_in_float(fit):
    """The argument of the exponential is rounded as x^2 / 2 and as its product with log2 e, each off by 2^-24 of at most x^2 / 2
    in a power of e; the seven steps of the polynomial, t, and three products by a few units of 2^-24 more."""
    f = np.float32
    x = np.linspace(0.0, 13.0, 200001).astype(f)
    once = lambda v: v.astype(f).astype(np.float64)         # a fused operation, rounded once
    t = once(1.0 / once(1.0 + float(f(fit[0])) * x.astype(np.float64)))
    power = once(once(once(-0.5 * x.astype(np.float64)) * x) * float(f(1.44269504)))
    e, q = once(np.exp2(power)), np.full(x.shape, float(f(fit[1][0])))
    for c in fit[1][1:]:
        q = once(q * t + float(f(c)))
    found = once(once(q * t) * e)
    want = 0.5 * erfc(x.astype(np.float64) * 0.5 ** 0.5)
    there = want >= 2.0 ** -126
    off = np.abs(found / want - 1.0)
    assert np.all((off <= 9.2e-7 + (x.astype(np.float64) ** 2 + 14.0) * 2.0 ** -24)[there])
