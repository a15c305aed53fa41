"""What the quantiser makes of gated rows against g / (1 + exp(-g)) u in 64 bits: a value in 8 bits has to be one that the exact value, off by no more
than the gate's bound, is rounded to."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, F16, F32, np64, rng

pytestmark = pytest.mark.gpu
# In units of 2^-24: exp2 2 (1 ulp), its argument's correction 1, their product 1; the sum with 1 one more; reciprocal 2 (1 ulp); products with g and u 1 each
EPS = 9 * 2.0**-24


def exact(x):
    g, u = np.split(np64(x), 2, axis=1)
    return g / (1 + np.exp(-g)), u


def check(x):
    """x [rows, 2 * 128 n]"""
    r = B.quantise_f8(x, gated=True)
    n, kb = x.shape[0], x.shape[1] // 256
    byte = r.scales.transpose(0, 1).reshape(n, -1)[:, :kb].cpu().numpy().astype(int)
    q = np64(r.q).reshape(n, kb, 128)
    silu, u = exact(x)
    v, slack = (silu * u).reshape(n, kb, 128), (2.0**-149 * np.abs(u) + 2.0**-150).reshape(n, kb, 128)   # g / (1 + exp(-g)) may be a denormal: a whole step; and the product, half a step
    low, high = np.maximum(np.abs(v) * (1 - EPS) - slack, 0), np.abs(v) * (1 + EPS) + slack
    assert (byte - 127 >= O.exponent(low.max(axis=2))).all() and (byte - 127 <= O.exponent(high.max(axis=2))).all()
    s = np.ldexp(1.0, byte - 127)[:, :, None]
    a = np.abs(q)
    bad = (a < O.round_e4m3(np.minimum(low / s, 448))) | (a > O.round_e4m3(np.minimum(high / s, 448))) | ((q != 0) & (np.sign(q) != np.sign(v)))
    assert not bad.any(), f"{bad.sum()} of {bad.size}, at gates {np.split(np64(x), 2, axis=1)[0].reshape(v.shape)[bad][:8]}"


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("lo,hi", [(-100, -80), (-80, -40), (-40, -20), (-20, -8), (-8, -4), (-4, 4), (4, 100)])
def test_gates(dtype, lo, hi):
    """a block's gates lie within a half of each other, so that its values are of a size, and u brings them to one that 8 bits hold"""
    g = rng(lo)
    rows, width = 1500, 1024
    first = torch.rand((rows, width // 128, 1), generator=g, device=DEV, dtype=torch.float64) * (hi - lo - 0.5) + lo
    gate = (first + 0.5 * torch.rand((rows, width // 128, 128), generator=g, device=DEV, dtype=torch.float64)).reshape(rows, width)
    u = torch.randn((rows, width), generator=g, device=DEV, dtype=torch.float64) * (1 if dtype is F16 else 1e20 if lo <= -80 else 1e3)
    check(torch.cat([gate, u], dim=1).to(dtype))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_gates_at_the_ends(dtype):
    big = float(torch.finfo(dtype).max)
    rows = [(-87.5, 1.0), (-88.5, 1.0), (-90.0, 1e30), (-100.0, 1e30), (-103.5, 1e38), (-150.0, 1e38), (-1e5, 1e38), (-big, 1.0), (0.0, 1.0), (-0.0, 3.0), (1e-38, 1.0), (-1e-38, 1e5),
            (big, 1.0), (big, 1e-30), (200.0, 1e30), (110.0, -2.0), (90.0, 0.0), (64.0, 1.0), (-64.0, 1.0), (-64.5, 1.0), (104.5, 1.0)]
    gate, u = (torch.tensor([r[i] for r in rows], device=DEV, dtype=torch.float64)[:, None].expand(len(rows), 128) for i in (0, 1))
    check(torch.cat([gate, u], dim=1).to(dtype))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", [7, 128 + 7])
def test_a_gate_or_value_that_is_no_number(bad, where):
    x = torch.ones((2, 256), device=DEV)
    x[1, where] = bad
    v = B.quantise_f8(x, gated=True).values()
    assert v[1].isnan().all() and v[0].isfinite().all()
