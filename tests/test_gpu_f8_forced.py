"""Repeated runs of every kernel of the 8-bit products with outputs that it makes: the same bits."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_f8_forced import PAIRS
from test_gpu_f8 import BF16, DEV, F16, F32, acts, rng, weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,y", PAIRS)
def test_many_runs_give_the_same_bits(kernel, y):
    dtype = {0: F16, 1: F32, 2: BF16}[y]
    g = rng(21)
    q, s = weight(g, 1000, 2100, "f32", experts=3)
    x = acts(g, 400, 2100, BF16) * 0.01
    off = torch.tensor([0, 130, 131, 390], dtype=torch.int32, device=DEV)
    try:
        for k in (kernel, kernel + 3 * 1024) if kernel > 64 else (kernel,):
            B.set_option(B.OPT_F8_KERNEL, k)
            calls = (lambda: B.linear_f8(x, q[0], s[0], out_dtype=dtype), lambda: B.grouped_linear_f8(x, q, s, off, out_dtype=dtype))
            first = [f() for f in calls]
            for _ in range(30):
                assert all(torch.equal(f(), a) for f, a in zip(calls, first))
    finally:
        B.set_option(B.OPT_F8_KERNEL, 0)
