"""The polynomial of the 8-bit products' gelu: the errors that its comment states, from the coefficients as they stand in the source (no GPU)."""
import re

import numpy as np
from scipy.special import erfcx, ndtr

from test_asm_distances import CSRC

SOURCE = (CSRC / "f8_epilogue.h").read_text()


def coefficients():
    """the highest first, and what s is multiplied with, as fp32 numbers"""
    body = SOURCE[SOURCE.index("float gelu(float v)"): SOURCE.index("float gelu_tanh(float v)")]
    k = re.search(r"fmaf\(s, ([\d.]+)f, 1\.0f\)", body).group(1)
    first = re.search(r"float q = fmaf\(t, (-?[\d.]+)f, (-?[\d.]+)f\)", body).groups()
    c = [np.float32(v) for v in (*first, *re.findall(r"q = fmaf\(t, q, (-?[\d.]+)f\)", body))]
    assert len(c) == 8
    return c, np.float32(k)


def stated(pattern):
    return float(re.search(pattern, SOURCE).group(1))


def test_the_polynomial():
    c, k = coefficients()
    s = np.linspace(0, 14, 140001)
    t = 1 / (float(k) * s + 1)
    q = np.zeros_like(t)
    for v in c:
        q = q * t + float(v)
    off = np.abs(q * t / (erfcx(s / np.sqrt(2)) / 2) - 1).max()   # erfcx: 1e-15
    assert 0.99 * stated(r"the polynomial's ([\d.e-]+)") <= off <= stated(r"the polynomial's ([\d.e-]+)")


def test_in_fp32():
    """with the reciprocal and the exponential off by a unit either way: half steps of the value, beside what the exponent's rounding does"""
    c, k = coefficients()
    f, d = np.float32, np.float64
    v = np.concatenate([np.linspace(-13, 13, 400000), -np.logspace(-30, 0, 5000), np.logspace(-30, 0, 5000)]).astype(f)
    s, most = np.abs(v), 0.0
    for rcp in (-1, 0, 1):
        t = (1 / (s.astype(d) * k + 1).astype(f).astype(d)).astype(f)
        t = np.nextafter(t, f(np.inf) * rcp) if rcp else t
        q = (t.astype(d) * c[0] + c[1]).astype(f)
        for a in c[2:]:
            q = (t.astype(d) * q.astype(d) + a).astype(f)
        for exp in (-1, 0, 1):
            e = np.exp2((s * s * f(-0.72134752044448170368)).astype(d)).astype(f)
            e = np.nextafter(e, f(np.inf) * exp) if exp else e
            p = q * t * e
            y = v * np.where(v > 0, f(1) - p, p)
            want = v.astype(d) * ndtr(v.astype(d))
            off = np.abs(y - want) / np.abs(want) - np.where(v < 0, 2.0**-23 * s.astype(d) ** 2, 0)
            most = max(most, off.max() * 2**24)
    assert most <= stated(r"in fp32 (\d+) half steps")
