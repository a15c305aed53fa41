"""Offsets past 32 bits: weights of many experts, rows close to what 31-bit offsets reach, long tables of rows."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, F16, F32, np64, rng, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 40, 200])
def test_experts_past_4_gib(rows):
    """24 experts of 14336 x 16384, 5.6 GB: the rows of the last one and of one inside the first 4 GiB"""
    e, out, inn = 24, 14336, 16384
    g = rng(11)
    q = torch.zeros((e, out, inn), dtype=torch.float8_e4m3fn, device=DEV)
    s = torch.full((e, out // 128, inn // 128), 120, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    for k in (2, e - 1):
        q[k] = (torch.randn((out, inn), generator=g, device=DEV, dtype=F16) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    off = [0] * 3 + [rows] * (e - 3) + [2 * rows]
    x = torch.randn((2 * rows, inn), generator=g, device=DEV).to(BF16)
    y = B.grouped_linear_f8(x, q, s, torch.tensor(off, dtype=torch.int32, device=DEV))
    x8, _ = O.quantise_rows(np64(x))
    take = torch.arange(0, out, 1021, device=DEV)
    for k, at in ((2, slice(0, rows)), (e - 1, slice(rows, 2 * rows))):
        w = np64(q[k].view(torch.uint8)[take].view(torch.float8_e4m3fn)) * 2.0**-7
        want = x8[at] @ w.T
        assert (np.abs(np64(y[at][:, take]) - want) <= tolerance(x8[at], w, BF16, want)).all()


def test_rows_up_to_2_gib():
    """the most rows of 8192 columns that a call takes, and one more"""
    n, out, inn = (2**31 - 1) // 8192, 128, 8192
    g = rng(12)
    q = (torch.randn((out, inn), generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    s = torch.full((1, inn // 128), 120, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    x = torch.zeros((n + 1, inn), dtype=F16, device=DEV)
    take = torch.tensor([0, 1, n // 2, n - 129, n - 2, n - 1], device=DEV)
    x[take] = torch.randn((len(take), inn), generator=g, device=DEV).to(F16)
    y = B.linear_f8(x[:n], q, s)
    x8, _ = O.quantise_rows(np64(x[take]))
    w = np64(q) * 2.0**-7
    want = x8 @ w.T
    assert (np.abs(np64(y[take]) - want) <= tolerance(x8, w, F16, want)).all()
    y[take] = 0
    assert not y.any()
    with pytest.raises(B.BitStackError):
        B.linear_f8(x, q, s)


def test_outputs_past_4_gib():
    """y of 4.3 GB, one block of columns"""
    n, out = 17 * 1024, 131072
    g = rng(13)
    q = (torch.randn((out, 16), generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    s = torch.full((out // 128, 1), 120, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    x = torch.randn((n, 16), generator=g, device=DEV).to(F16)
    y = B.linear_f8(x, q, s)
    rows, cols = torch.tensor([0, 1000, n - 1], device=DEV), torch.arange(0, out, 997, device=DEV)
    x8, _ = O.quantise_rows(np64(x[rows]))
    w = np64(q.view(torch.uint8)[cols].view(torch.float8_e4m3fn)) * 2.0**-7
    want = x8 @ w.T
    assert (np.abs(np64(y[rows][:, cols]) - want) <= tolerance(x8, w, F16, want)).all()


def test_combine_of_a_long_table():
    n, width = 700_000, 4096   # 5.7 GB
    h = torch.zeros((n, width), dtype=F16, device=DEV)
    slots = torch.tensor([[0, n - 1], [n // 2, n], [n - 2, -1]], dtype=torch.int32, device=DEV)
    weights = torch.tensor([[0.5, 2.0], [1.0, 7.0], [0.25, 3.0]], device=DEV)
    for i, r in enumerate((0, n - 1, n // 2, n - 2)):
        h[r] = i + 1
    y = B.combine(h, slots, weights)
    assert torch.equal(y.float(), torch.tensor([4.5, 3.0, 1.0], device=DEV)[:, None].expand(3, width))


def test_quantise_past_4_gib():
    """rows of x 16 GiB apart in all"""
    x = torch.zeros((2**20 + 3, 4096), dtype=F32, device=DEV)[:, :512]
    x[-1], x[-2, 5] = 3.0, -448.0
    r = B.quantise_f8(x)
    v = r.q.view(torch.uint8)
    assert not v[:-2].any() and torch.equal(B.F8Rows(r.q[-2:], r.scales[:, -2:].contiguous(), 512).values(), x[-2:])


def test_combine_of_many_tokens():
    """more tokens than a launch has workgroups"""
    n, width = 20_000_001, 3
    h = torch.arange(12, device=DEV).view(4, width).to(F16)
    slots = (torch.arange(n, device=DEV) % 5 - 1).to(torch.int32).view(n, 1)   # -1: nothing
    y = B.combine(h, slots, torch.full((n, 1), 2.0, device=DEV))
    want = torch.cat([torch.zeros((1, width), dtype=F16, device=DEV), 2 * h])
    assert torch.equal(y[: n // 5 * 5].view(-1, 5, width), want.expand(n // 5, 5, width)) and torch.equal(y[n // 5 * 5 :], want[: n % 5])
