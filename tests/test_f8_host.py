"""CPU-only checks of include/bitstack_f8.h: sizes, and refusals, which come before anything is enqueued (the device pointers here are never
followed).  The oracle of the 8-bit values against PyTorch's conversion."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O

NULL, RANGE, SHAPE, ALIGN, SIZE, ARG = -1, -3, -2, -4, -6, -8
P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def L():
    B.linear_f8   # loads f8.py
    from paper_2410_23918_amd import f8
    return f8._f8_lib()


def test_sizes(L):
    for inn, row, scales in ((1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (513, 640, 8), (4096, 4096, 32)):
        assert (L.bitstack_f8_row_bytes(inn), L.bitstack_f8_row_scales(inn)) == (row, scales)
    assert L.bitstack_f8_row_bytes(0) == L.bitstack_f8_row_bytes((1 << 20) + 1) == 0
    assert L.bitstack_f8_workspace_bytes(10, 300, 10, 64, 1) >= 10 * (384 + 4)
    for bad in ((-1, 300, 1, 64, 1), (1, 0, 1, 64, 1), (1, 300, -1, 64, 1), (1, 300, 1, 0, 1), (1, 300, 1, 64, 0), (1, 300, 1, 64, 1025), (1 << 20, 4096, 1, 64, 1)):
        assert L.bitstack_f8_workspace_bytes(*bad) == 0
    from paper_2410_23918_amd.f8 import _Rows, _Weight
    for tokens, grouped, dtype in ((1, 0, 0), (1, 1, 0), (40, 0, 2), (300, 1, 0), (5, 0, 3)):   # a call's own needs are no more than what is said ahead
        n = L.bitstack_f8_call_workspace_bytes(C.byref(_Rows(P, P, 4096, dtype, tokens, 0)), C.byref(_Weight(P, 4096, P, 0, 512, 4096, 3 if grouped else 1)), tokens, 0, grouped)
        assert n <= L.bitstack_f8_workspace_bytes(tokens, 4096, tokens, 512, 3 if grouped else 1)
        assert (n == 0) == (not grouped and tokens <= 16)
    assert L.bitstack_f8_call_workspace_bytes(None, None, 1, 0, 0) == 0
    for bad in ((-1, 8, 2), (1, 0, 1), (1, 8, 0), (1, 8, 9), (1, 1025, 1), (1, 64, 33)):
        assert L.bitstack_route_workspace_bytes(*bad) == 0
    with pytest.raises(B.BitStackError):
        B.f8_workspace_bytes(1, 0, 1, 1)


def refused(L, code, x=None, w=None, **change):
    from paper_2410_23918_amd.f8 import _Rows, _Weight
    weight = dict(q=P, ld=256, scales=P, scale_type=0, out=64, inn=256, experts=1) | (w or {})
    rows = dict(x=P, scales=P, ld=256, dtype=0, rows=40, gated=0) | (x or {})
    a = dict(y=P, y_dtype=0, ld_y=64, ws=P, ws_bytes=1 << 20) | change
    args = (C.byref(_Rows(**rows)), C.byref(_Weight(**weight)))
    end = (a["y"], a["y_dtype"], a["ld_y"], a["ws"], a["ws_bytes"], None)
    assert L.bitstack_f8_linear(*args, *end) == code
    if "experts" not in (w or {}):
        assert L.bitstack_f8_grouped_linear(*args, P, P, rows["rows"], *end) == code


def test_refusals_of_the_products(L):
    assert L.bitstack_f8_linear(None, None, P, 0, 64, P, 1 << 20, None) == NULL
    for code, x, w in (
        (NULL, dict(x=None), None), (NULL, None, dict(q=None)), (NULL, None, dict(scales=None)), (NULL, dict(dtype=3, scales=None), None),
        (SHAPE, None, dict(inn=0)), (SHAPE, None, dict(out=0)), (SHAPE, None, dict(experts=0)), (SHAPE, None, dict(experts=2)), (SHAPE, None, dict(ld=240)),
        (SHAPE, None, dict(ld=(1 << 22) + 16)), (SHAPE, dict(ld=255), None), (SHAPE, dict(ld=511, gated=1), None),
        (ALIGN, None, dict(q=P + 8)), (ALIGN, None, dict(ld=264)), (ALIGN, None, dict(scales=P + 2, scale_type=1)), (ALIGN, dict(x=P + 1), None), (ALIGN, dict(x=P + 8, dtype=3), None),
        (ARG, None, dict(scale_type=2)), (ARG, dict(dtype=4), None), (ARG, dict(gated=2), None), (RANGE, dict(rows=-1), None), (RANGE, dict(rows=1 << 24), None),
    ):
        refused(L, code, x, w)
    refused(L, ARG, y_dtype=3)
    refused(L, ALIGN, y=P + 1)
    refused(L, SHAPE, ld_y=63)
    refused(L, NULL, y=None)
    refused(L, NULL, ws=None)
    refused(L, ALIGN, ws=P + 16)
    refused(L, SIZE, ws_bytes=100)
    from paper_2410_23918_amd.f8 import _Rows, _Weight
    args = (C.byref(_Rows(P, P, 256, 0, 40, 0)), C.byref(_Weight(P, 256, P, 0, 64, 256, 3)))
    grouped = lambda off, index, n: L.bitstack_f8_grouped_linear(*args, off, index, n, P, 0, 64, P, 1 << 20, None)
    assert grouped(None, None, 40) == NULL
    assert grouped(P, None, 41) == RANGE   # rows of y that x does not have
    assert grouped(P, None, -1) == RANGE
    assert grouped(P + 2, None, 40) == ALIGN and grouped(P, P + 2, 40) == ALIGN


def test_refusals_of_the_others(L):
    q = lambda **k: L.bitstack_f8_quantise(*(dict(x=P, dtype=0, ld=256, rows=4, inn=256, gated=0, q=P, s=P) | k).values(), None)
    assert [q(x=None), q(dtype=3), q(dtype=9), q(ld=200), q(rows=-1), q(inn=0), q(gated=5), q(q=None), q(s=None), q(q=P + 8), q(x=P + 1)] == \
        [NULL, ARG, ARG, SHAPE, RANGE, SHAPE, ARG, NULL, NULL, ALIGN, ALIGN]
    assert q(rows=0) == 0
    w = lambda **k: L.bitstack_f8_quantise_weight(*(dict(w=P, dtype=0, ld=256, out=64, inn=256, q=P, ld_q=256, s=P) | k).values(), None)
    assert [w(w=None), w(dtype=3), w(ld=255), w(out=0), w(inn=0), w(q=P + 1), w(ld_q=248), w(ld_q=240), w(s=None)] == \
        [NULL, ARG, SHAPE, SHAPE, SHAPE, ALIGN, ALIGN, SHAPE, NULL]
    r = lambda **k: L.bitstack_route(*(dict(l=P, dtype=0, ld=8, tokens=4, experts=8, top_k=2, renormalise=1, c=P, w=P, s=P, i=P, o=P, ws=P, n=1 << 20) | k).values(), None)
    assert [r(l=None), r(dtype=3), r(ld=7), r(tokens=-1), r(experts=0), r(top_k=9), r(top_k=0), r(renormalise=2), r(o=None), r(ws=None), r(ws=P + 8), r(n=16), r(i=P + 2)] == \
        [NULL, ARG, SHAPE, RANGE, SHAPE, SHAPE, SHAPE, ARG, NULL, NULL, ALIGN, SIZE, ALIGN]
    c = lambda **k: L.bitstack_combine(*(dict(h=P, dtype=0, ld=64, rows=8, width=64, s=P, w=P, tokens=4, k=2, y=P, ld_y=64) | k).values(), None)
    assert [c(h=None), c(dtype=3), c(ld=63), c(rows=-1), c(width=0), c(s=None), c(w=None), c(tokens=-1), c(k=0), c(k=33), c(y=None), c(y=P + 1), c(ld_y=3)] == \
        [NULL, ARG, SHAPE, RANGE, SHAPE, NULL, NULL, RANGE, SHAPE, SHAPE, NULL, ALIGN, SHAPE]
    assert c(tokens=0) == 0


def test_without_a_gpu_tensor():
    q = torch.zeros((64, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.zeros((1, 1), dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for call in (lambda: B.linear_f8(torch.zeros((1, 128), dtype=torch.float16), q, s), lambda: B.quantise_f8(torch.zeros((1, 128))),
                 lambda: B.route(torch.zeros((1, 8)), 2), lambda: B.combine(torch.zeros((1, 8)), torch.zeros((1, 1), dtype=torch.int32), torch.zeros((1, 1)))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AttributeError):
        B.no_such_name


def test_oracle_rounds_as_e4m3_does():
    rng = np.random.default_rng(3)
    v = np.concatenate([rng.standard_normal(20000) * np.exp(rng.uniform(-8, 5, 20000)), np.arange(-448, 449, 0.5), np.arange(-64, 65) * 2.0**-10]).clip(-448, 448).astype(np.float32)
    assert np.array_equal(O.round_e4m3(v.astype(np.float64)), torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy())
    assert O.exponent(448.0) == 0 and O.exponent(np.nextafter(np.float32(448), np.float32(500))) == 1 and O.exponent(0.0) == -126
    amax = np.abs(rng.standard_normal(1000)).astype(np.float32)
    e = O.exponent(amax)
    assert (amax <= 448 * 2.0**e).all() and (amax > 448 * 2.0 ** (e - 1)).all()
