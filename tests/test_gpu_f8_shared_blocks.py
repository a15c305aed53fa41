"""Gates and values that share a block of 128, in every kernel that leaves their sums and the join behind it, against the definition in 64 bits."""
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_f8_forced import PAIRS
from test_gpu_f8 import BF16, DEV, F16, F32, acts, np64, rng, weight
from test_gpu_f8_epilogue import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("cols", [133, 600, 654, 1025])
@pytest.mark.parametrize("kernel,y", [p for p in PAIRS if p[0] > 64])
def test_every_kernel(kernel, y, cols, scales):
    """values that begin with any multiple of four or none, tiles with empty rows and columns, columns that end inside a block and inside 16 bytes, in one slice and in three"""
    dtype = {0: F16, 1: F32, 2: BF16}[y]
    g = rng(kernel + cols)
    inn, tokens = 1803, 300
    q, s = weight(g, 2 * cols, inn, scales)
    x = acts(g, tokens, inn, dtype) * 0.003
    bias, residual = torch.randn(2 * cols, generator=g, device=DEV), torch.randn((tokens, cols), generator=g, device=DEV).to(dtype)
    x8, _ = O.quantise_rows(np64(x))
    w = O.weight_values(np64(q), np64(s))
    try:
        for slices in (1, 3):
            B.set_option(B.OPT_F8_KERNEL, kernel + 1024 * slices)
            for n in (tokens, 7, 1):
                y = B.linear_f8(x[:n], q, s, bias=bias, activation="silu_gated", residual=residual[:n])
                check(y, x8[:n], w, dtype, bias, "silu_gated", residual[:n])
    finally:
        B.set_option(B.OPT_F8_KERNEL, 0)


@pytest.mark.parametrize("dtype", [F16, F32], ids=["f16", "f32"])
def test_many_rows(dtype):
    """2048 x 14000 by the built-in choice; every 37th row is looked at"""
    g = rng(5)
    inn, cols, tokens = 640, 7000, 2048
    q, s = weight(g, 2 * cols, inn, "f32")
    x = acts(g, tokens, inn, dtype) * 0.003
    y = B.linear_f8(x, q, s, activation="silu_gated")
    take = torch.arange(0, tokens, 37, device=DEV)
    check(y[take], O.quantise_rows(np64(x[take]))[0], O.weight_values(np64(q), np64(s)), dtype, None, "silu_gated", None)
