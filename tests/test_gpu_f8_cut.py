"""16-bit outputs against the rule of the 8-bit matrix instruction itself: of eight neighbouring columns each product is cut to a multiple of 2^-13 of the power of
two in the largest one (the largest has 8 significant bits and stays whole), what is added to these sums is fp32.  Also where loud products
cancel, so that y is far smaller than they are."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, EPS, F16, acts, np64, rng, weight

pytestmark = pytest.mark.gpu


def bound(xq, ex, wq, s, dtype, want):
    """xq, wq: e4m3 values; ex: exponents of the rows' blocks; s: scales of the weight's"""
    tokens, inn = xq.shape
    steps = 128 + -(-inn // 128) + 8
    cut, size = np.zeros_like(want), np.zeros_like(want)
    for c in range(0, inn, 8):
        p = np.abs(xq[:, None, c : c + 8] * wq[None, :, c : c + 8])
        scale = np.ldexp(1.0, ex[:, c // 128])[:, None] * np.repeat(s[:, c // 128], 128)[None, : len(wq)]
        most = p.max(axis=2)
        unit = np.where(most > 0, np.ldexp(1.0, np.frexp(most)[1] - 1 - 13), 0)
        cut += 7 * unit * scale
        size += p.sum(axis=2) * scale
    return cut + steps * 2.0**-23 * size + EPS[dtype] * np.abs(want) + (2.0**-25 if dtype is F16 else 0)


@pytest.mark.parametrize("cancel", [False, True])
@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("tokens,out,inn", [(3, 64, 512), (16, 70, 1000), (40, 130, 1111), (200, 260, 640)])
def test_cut_of_eight_columns(tokens, out, inn, dtype, scales, cancel):
    g = rng(tokens)
    q, s = weight(g, out, inn, scales)
    x = acts(g, tokens, inn, dtype) * 0.01
    if cancel:   # every second pair of columns: one loud value, weights of opposite signs
        x[:, 0 : inn - 1 : 4] *= 30
        x[:, 1:inn:4] = x[:, 0 : inn - 1 : 4]
        raw = q.view(torch.uint8)
        raw[:, 1:inn:4] = raw[:, 0 : inn - 1 : 4] ^ 0x80
    x8, ex = O.quantise_rows(np64(x))
    xq = x8 / np.repeat(np.ldexp(1.0, ex), 128, axis=1)[:, :inn]
    want = x8 @ O.weight_values(np64(q), np64(s)).T
    assert (np.abs(np64(B.linear_f8(x, q, s)) - want) <= bound(xq, ex, np64(q), np64(s), dtype, want)).all()
