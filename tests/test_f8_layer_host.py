"""CPU-only checks of the layer of experts for a few tokens: sizes, and refusals, which come before anything is enqueued (the device pointers here are never
followed)."""
import ctypes as C

import pytest
import torch

import paper_2410_23918_amd as B

OK, NULL, SHAPE, RANGE, ALIGN, SIZE, ARG = 0, -1, -2, -3, -4, -6, -8
P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def L():
    B.linear_f8   # loads f8.py
    from paper_2410_23918_amd import f8
    return f8._f8_lib()


def call(L, w1=None, w2=None, **change):
    from paper_2410_23918_amd.f8 import _Weight
    first = dict(q=P, ld=256, scales=P, scale_type=0, out=2 * 96, inn=256, experts=8) | (w1 or {})
    second = dict(q=P, ld=96, scales=P, scale_type=0, out=256, inn=96, experts=8) | (w2 or {})
    a = dict(x=P, dtype=0, ld_x=256, logits=P, logits_dtype=1, ld_logits=8, tokens=4, top_k=2, renormalise=1) | {k: v for k, v in change.items() if k in
        ("x", "dtype", "ld_x", "logits", "logits_dtype", "ld_logits", "tokens", "top_k", "renormalise")}
    b = dict(residual=None, ld_r=256, y=P, ld_y=256, ws=P, n=1 << 40) | {k: v for k, v in change.items() if k in ("residual", "ld_r", "y", "ld_y", "ws", "n")}
    return L.bitstack_f8_expert_layer(*a.values(), C.byref(_Weight(**first)), C.byref(_Weight(**second)), *b.values(), None)


def test_sizes(L):
    size = L.bitstack_f8_expert_layer_workspace_bytes
    assert size(0, 256, 96, 8, 2) >= 256
    assert size(64, 256, 96, 8, 2) >= size(1, 256, 96, 8, 2) >= 2 * 96 * 2 * 3
    for bad in ((-1, 256, 96, 8, 2), (65, 256, 96, 8, 2), (1, 7, 96, 8, 2), (1, 256, 0, 8, 2), (1, 256, 96, 0, 1), (1, 256, 96, 1025, 2), (1, 256, 96, 8, 9), (1, 256, 96, 64, 33),
                (1, 256, 96, 8, 0), (1, (1 << 20) + 1, 96, 8, 2), (1, 256, (1 << 20) + 1, 8, 2)):
        assert size(*bad) == 0
        with pytest.raises(B.BitStackError):
            B.expert_layer_workspace_bytes(*bad)


def test_refusals(L):
    assert L.bitstack_f8_expert_layer(P, 0, 256, P, 1, 8, 1, 2, 1, None, None, None, 0, P, 256, P, 1 << 40, None) == NULL
    assert call(L, tokens=0) == OK
    for code, change in (
        (RANGE, dict(tokens=-1)), (RANGE, dict(tokens=65)), (SHAPE, dict(top_k=0)), (SHAPE, dict(top_k=9)), (ARG, dict(dtype=3)), (ARG, dict(dtype=-1)), (ARG, dict(logits_dtype=3)),
        (ARG, dict(renormalise=2)), (NULL, dict(x=None)), (NULL, dict(logits=None)), (NULL, dict(y=None)), (NULL, dict(ws=None)), (ALIGN, dict(x=P + 1)), (ALIGN, dict(y=P + 1)),
        (ALIGN, dict(residual=P + 1)), (ALIGN, dict(logits=P + 2)), (ALIGN, dict(ws=P + 16)), (SHAPE, dict(ld_x=255)), (SHAPE, dict(ld_y=255)), (SHAPE, dict(residual=P, ld_r=255)),
        (SHAPE, dict(ld_logits=7)), (SIZE, dict(n=256)),
    ):
        assert call(L, **change) == code, change
    for code, w1, w2 in (
        (SHAPE, dict(out=2 * 95), None), (SHAPE, dict(out=96), None), (SHAPE, None, dict(out=255)), (SHAPE, None, dict(experts=7)), (SHAPE, dict(experts=1025), dict(experts=1025)),
        (SHAPE, dict(inn=7), dict(out=7)), (SHAPE, dict(ld=240), None), (SHAPE, None, dict(ld=80)), (SHAPE, dict(ld=(1 << 22) + 16), None), (ALIGN, dict(ld=264), None),
        (ALIGN, dict(q=P + 8), None), (ALIGN, None, dict(q=P + 8)), (ALIGN, dict(scales=P + 2, scale_type=1), None), (ARG, dict(scale_type=2), None), (ARG, None, dict(scale_type=-1)),
        (NULL, dict(q=None), None), (NULL, None, dict(scales=None)),
        (RANGE, dict(ld=1 << 22, out=2048), dict(ld=1024, inn=1024)),   # 8 GiB of an expert's w1
    ):
        assert call(L, w1, w2) == code, (w1, w2)
    wide = dict(out=2 << 20, ld=16, inn=16), dict(out=16, ld=1 << 20, inn=1 << 20)
    assert call(L, *wide, tokens=64, top_k=8) == RANGE   # 3 GiB of h


def test_without_a_gpu_tensor():
    q = lambda *shape: torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = lambda *shape: torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    w1, w2 = (q(8, 192, 256), s(8, 2, 2)), (q(8, 256, 96), s(8, 2, 1))
    x, logits = torch.zeros((4, 256)), torch.zeros((4, 8))
    for change in ({}, dict(x=x[:, :255]), dict(logits=logits[:, :7]), dict(logits=logits[:3]), dict(w1=(q(8, 190, 256), s(8, 2, 2))), dict(w2=(q(7, 256, 96), s(7, 2, 1))),
                   dict(x=x.T.contiguous().T), dict(x=x.double()), dict(logits=logits.to(torch.int32)), dict(w1=(q(8, 192, 256), s(8, 2, 1))), dict(residual=x[:3]),
                   dict(residual=x.half()), dict(y=x[:, :255])):
        with pytest.raises(ValueError):
            a = dict(x=x, logits=logits, w1=w1, w2=w2, top_k=2) | change
            B.expert_layer_f8(**a)
