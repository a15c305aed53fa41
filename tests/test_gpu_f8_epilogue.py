"""The 8-bit product with bias, activation and residual after it, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_f8_forced import PAIRS
from test_gpu_f8 import BF16, DEV, EPS, F16, F32, acts, np64, rng, weight

pytestmark = pytest.mark.gpu
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu", "silu_gated"]


def sum_off(x8, w, dtype):
    """how far the sums may be off: as in test_gpu_f8.tolerance, without the output's rounding"""
    steps = 128 + -(-x8.shape[1] // 128) + 8
    a, b = np.abs(x8), np.abs(w)
    off = steps * 2.0**-23 * (a @ b.T)
    if dtype is not F32:
        most = lambda v: np.pad(v, ((0, 0), (0, -v.shape[1] % 8))).reshape(len(v), -1, 8).max(axis=2)
        off += 7 * 2.0**-13 * (most(a) @ most(b).T)
    return off


def sigmoid(v):
    return np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))


def activate(v, off, act):
    """(value, how far off) for arguments that are off by `off`: the functions' slopes are 1.13 at most; their own error 2^-20 of the value, and what a rounding of the argument
    of the exponential or of erfc, 2^-21 of it, does"""
    if act is None:
        return v, off
    if act == "relu":
        return np.maximum(v, 0), off
    if act == "silu_gated":
        (g, u), (og, ou) = np.split(v, 2, axis=1), np.split(off, 2, axis=1)
        silu = g * sigmoid(g)
        return silu * u, 1.1 * og * np.abs(u) + np.abs(silu) * ou + 1.1 * og * ou + 2.0**-21 * np.abs(silu * u)
    if act == "silu":
        return v * sigmoid(v), 1.13 * off + 2.0**-21 * np.abs(v * sigmoid(v))
    if act == "gelu":
        from scipy.special import ndtr
        h = v * ndtr(v)
        return h, 1.13 * off + 2.0**-20 * np.abs(h) + 2.0**-21 * v * v * np.exp(-v * v / 2) / math.sqrt(2 * math.pi) + 2.0**-126
    arg = 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v**3)
    s = sigmoid(arg)
    return v * s, 1.13 * off + 2.0**-20 * np.abs(v * s) + 2.0**-21 * np.abs(v * arg) * s * (1 - s) + 2.0**-126


def check(y, x8, w, dtype, bias, act, residual):
    a, off = x8 @ w.T, sum_off(x8, w, dtype)
    if bias is not None:
        a = a + np64(bias)
        off = off + 2.0**-24 * np.abs(a)
    h, off = activate(a, off, act)
    if residual is not None:
        h = h + np64(residual)
        off = off + 2.0**-24 * np.abs(h)
    off = off + EPS[dtype] * (np.abs(h) + off) + (2.0**-25 if dtype is F16 else 0)
    got = np64(y)
    if dtype is F16:   # beyond fp16's range both are infinite, near its end either may be
        far = np.abs(h) + off >= 65504
        assert (got[far] * np.sign(h[far]) >= 65504 - 2 * off[far]).all()
        got, h, off = got[~far], h[~far], off[~far]
    assert np.isfinite(got).all()
    d = np.abs(got - h)
    assert (d <= off).all(), f"{(d / off).max():.2f} times what it may be"


SHAPES = [  # tokens, out (half of it gated: those, and twice as many rows), in
    (1, 1, 1), (1, 128, 128), (1, 512, 512), (1, 1056, 2001), (2, 130, 127), (3, 100, 129), (5, 256, 4096), (15, 257, 640), (16, 384, 256), (17, 96, 300),
    (31, 1000, 1111), (57, 1056, 2001), (64, 512, 1024), (65, 129, 513), (127, 255, 1152), (128, 128, 128), (129, 384, 2048), (200, 1056, 1040), (255, 640, 777),
    (257, 513, 1280), (300, 1024, 4096), (513, 384, 384), (300, 256, 8192),
]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,cols,inn", SHAPES)
def test_epilogue(tokens, cols, inn, dtype, act):
    g = rng(tokens * 7 + cols + inn)
    out = 2 * cols if act == "silu_gated" else cols
    for scales, with_bias, with_residual in (("e8m0", True, tokens % 2 == 0), ("f32", tokens % 3 == 0, True)):
        q, s = weight(g, out, inn, scales)
        x = acts(g, tokens, inn, dtype) * 0.003
        bias = torch.randn(out, generator=g, device=DEV).to(BF16 if tokens % 2 else dtype) if with_bias else None
        residual = torch.randn((tokens, cols), generator=g, device=DEV).to(dtype) if with_residual else None
        if act is None and bias is None:
            residual = torch.randn((tokens, cols), generator=g, device=DEV).to(dtype)
        y = B.linear_f8(x, q, s, bias=bias, activation=act, residual=residual)
        assert y.dtype is dtype and tuple(y.shape) == (tokens, cols)
        x8, _ = O.quantise_rows(np64(x))
        check(y, x8, O.weight_values(np64(q), np64(s)), dtype, bias, act, residual)


@pytest.mark.parametrize("act", ["gelu_tanh", "silu_gated"])
@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("kernel,y", PAIRS)
def test_every_kernel(kernel, y, scales, act):
    """tiles with empty rows and columns, columns that end inside a block and inside 16 bytes, in one slice and in three"""
    dtype = {0: F16, 1: F32, 2: BF16}[y]
    g = rng(kernel)
    out, inn, tokens = (1280, 1803, 300)
    cols = out // 2 if act == "silu_gated" else out - 9
    q, s = weight(g, out if act == "silu_gated" else cols, inn, scales)
    x = acts(g, tokens, inn, dtype) * 0.003
    bias, residual = torch.randn(q.shape[0], generator=g, device=DEV), torch.randn((tokens, cols), generator=g, device=DEV).to(dtype)
    x8, _ = O.quantise_rows(np64(x))
    w = O.weight_values(np64(q), np64(s))
    try:
        for k in (kernel, kernel + 3 * 1024) if kernel > 64 else (kernel,):
            B.set_option(B.OPT_F8_KERNEL, k)
            for n in (tokens, 7):
                check(B.linear_f8(x[:n], q, s, bias=bias, activation=act, residual=residual[:n]), x8[:n], w, dtype, bias, act, residual[:n])
    finally:
        B.set_option(B.OPT_F8_KERNEL, 0)
