"""The 8-bit experts' GeLU, its constants read from the kernel source: the fit against the function it stands for, and the
kernel's formula in fp32 against 64 bits, relative to the value on the left as well, where GeLU is small."""
import math
import os
import re

import numpy as np
import pytest
from scipy.special import erfc, erfcx

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2109_10465_amd", "csrc", "fp8_gemm.hip")
f = np.float32


def constants():
    text = open(SRC).read()
    body, = re.findall(r"constexpr float TAIL\[\d\] = \{([^}]*)\}", text)
    at, = re.findall(r"\bTAIL_AT = ([0-9.]+)f", text)
    lh, = re.findall(r"\bLOG2E_HALF = (-[0-9.]+)f", text)
    return [f(v.strip().rstrip("f")) for v in body.split(",")], f(at), f(lh)


C, AT, LH = constants()


def test_fit():
    t = np.linspace(0.0, 13.2, 400001)
    u = 1.0 / (1.0 + float(AT) * t)
    got = sum(float(c) * u ** i for i, c in enumerate(C))
    # the fit's 1.5e-6, and the roundings of its coefficients
    assert np.abs(got / (0.5 * erfcx(t / math.sqrt(2.0))) - 1.0).max() <= 1.6e-6
    assert LH == f(-math.log2(math.e) / 2.0)


def fma(a, b, c):
    return f(np.asarray(a, np.longdouble) * np.asarray(b, np.longdouble) + np.asarray(c, np.longdouble))


def kernel_form(z):
    t = np.minimum(np.abs(z), f(16))
    u = f(1.0 / fma(AT, t, f(1)).astype(np.float64))
    r = np.full_like(u, C[-1])
    for c in C[-2::-1]:
        r = fma(r, u, c)
    e = f(np.exp2(f(f(t * LH) * t).astype(np.float64)))
    return fma(-t, f(r * e), np.where(z <= 0, f(0), z))


@pytest.mark.parametrize("lo,hi", [(0, 1e-3), (1e-3, 1), (1, 3), (3, 5), (5, 7), (7, 10), (10, 12.5)])
def test_error(lo, hi):
    t = f(np.random.default_rng(1).uniform(lo, hi, 200000))
    for z in (t, -t):
        z64 = z.astype(np.float64)
        exact = z64 * 0.5 * erfc(-z64 / math.sqrt(2.0))
        off = np.abs(kernel_form(z).astype(np.float64) - exact)
        # of z Phi(-|z|): the fit's 1.6e-6; 2^-24 for each of about 8 operations; three roundings of the exponent -z^2 log2(e) / 2,
        # which are an error of z^2 / 2 times as much.  |z| Phi(-|z|) is below 0.17; on the right z's own rounding is on top
        share = 1.6e-6 + (8 + 1.5 * z64 ** 2) * 2.0 ** -24
        assert (off <= share * np.abs(z64) * 0.5 * erfc(np.abs(z64) / math.sqrt(2.0)) + 2.0 ** -23 * np.abs(exact)).all()
        assert off.max() <= 0.17 * share.max() + 2.0 ** -23 * hi


def test_ends():
    z = f([np.inf, -np.inf, 0.0, -0.0, 1e30, -1e30, 20.0, -20.0])
    assert kernel_form(z).tolist() == [np.inf, 0.0, 0.0, 0.0, float(f(1e30)), 0.0, 20.0, 0.0]
    assert np.isnan(kernel_form(f([np.nan]))).all()
