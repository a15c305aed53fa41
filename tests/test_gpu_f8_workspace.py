"""One workspace for calls of any number of rows up to the one that it was made for."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_experts import check_grouped
from test_gpu_f8 import BF16, DEV, F32, acts, np64, rng, tolerance, weight

pytestmark = pytest.mark.gpu


def need(rows, out, inn, dtype, grouped, x_dtype=0):
    import ctypes as C
    from paper_2410_23918_amd import f8
    x, w = f8._Rows(256, 256, inn, x_dtype, rows, 0), f8._Weight(256, inn, 256, 1, out, inn, 1)
    return f8._f8_lib().bitstack_f8_call_workspace_bytes(C.byref(x), C.byref(w), rows, 1 if dtype is F32 else 2, grouped)


@pytest.mark.parametrize("out,inn,most", [(14336, 4096, 4096), (8192, 8192, 4096), (1024, 4096, 1500), (640, 2048, 700)])
def test_fewer_rows_in_a_workspace_for_many(out, inn, most):
    """all rows that are tried; those whose partial sums would need more among them"""
    g = rng(out)
    q, s = weight(g, out, inn, "f32")
    x = acts(g, most, inn, BF16)
    x8, _ = O.quantise_rows(np64(x[:700]))
    take = torch.arange(0, out, max(1, out // 64), device=DEV)
    w = O.weight_values(np64(q), np64(s))[take.cpu().numpy()]
    ws = torch.empty(B.f8_workspace_bytes(most, inn, most, out), dtype=torch.uint8, device=DEV)
    smaller = 0
    for rows in (1, 16, 17, 33, 64, 100, 128, 200, 257, 300, 512, 513, 700, 1024, 2048, most):
        if rows > most:
            continue
        for dtype in (BF16, F32):
            smaller += need(rows, out, inn, dtype, 0) > ws.numel() or need(rows, out, inn, dtype, 1) > ws.numel()
            y = B.linear_f8(x[:rows], q, s, out_dtype=dtype, workspace=ws)
            z = B.grouped_linear_f8(x[:rows], q[None], s[None], torch.tensor([0, rows], dtype=torch.int32, device=DEV), out_dtype=dtype, workspace=ws)
            n = min(rows, 700)
            want = x8[:n] @ w.T
            for got in (y, z):
                assert (np.abs(np64(got[:n][:, take]) - want) <= tolerance(x8[:n], w, dtype, want)).all(), (rows, dtype)
    assert smaller or most < 4096


@pytest.mark.parametrize("experts", [8, 64])
def test_fewer_rows_through_experts(experts):
    g = rng(experts)
    out, inn, most = 256, 1100, 3000
    q, s = weight(g, out, inn, "e8m0", experts=experts)
    x = acts(g, most, inn, F32) * 0.1
    ws = torch.empty(B.f8_workspace_bytes(most, inn, most, out, experts), dtype=torch.uint8, device=DEV)
    for rows in (1, 15, 40, 200, 900, most):
        off = np.sort(np.concatenate([[0, rows], np.random.default_rng(rows).integers(0, rows + 1, experts - 1)])).astype(np.int32)
        y = B.grouped_linear_f8(x[:rows], q, s, torch.from_numpy(off).to(DEV), workspace=ws)
        check_grouped(y, x[:rows], q, s, off, None, F32)


def test_without_room_for_slices():
    """rows that are in 8 bits already need a workspace for partial sums alone; a byte less than the least that any call needs is refused"""
    g = rng(3)
    rows, out, inn = 128, 640, 8192
    q, s = weight(g, out, inn, "f32")
    x = acts(g, rows, inn, BF16)
    x8, _ = O.quantise_rows(np64(x))
    w = O.weight_values(np64(q), np64(s))
    want = x8 @ w.T
    assert need(rows, out, inn, F32, 0, 3) > 0
    for size in (256, 1 << 20, 1 << 24):
        y = B.linear_f8(B.quantise_f8(x), q, s, out_dtype=F32, workspace=torch.empty(size, dtype=torch.uint8, device=DEV))
        assert (np.abs(np64(y) - want) <= tolerance(x8, w, F32, want)).all()
    least = rows * (8192 + 64)
    B.linear_f8(x, q, s, workspace=torch.empty(least, dtype=torch.uint8, device=DEV))
    with pytest.raises(B.BitStackError) as e:
        B.linear_f8(x, q, s, workspace=torch.empty(least - 1, dtype=torch.uint8, device=DEV))
    assert e.value.code == -6
