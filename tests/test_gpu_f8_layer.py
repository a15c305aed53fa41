"""A layer of experts for a few tokens in one call, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, EPS, F16, F32, rng

pytestmark = pytest.mark.gpu


def weights(g, experts, out, inn, scales):
    """e4m3 values of any size with scales far apart, whose products with numbers around 1 are around 1; NaN behind the rows"""
    ld = -(-inn // 16) * 16
    q = (torch.randn((experts, out, ld), generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    q.view(torch.uint8)[:, :, inn:] = 0x7F
    shape = (experts, -(-out // 128), -(-inn // 128))
    e = torch.randint(-2, 2, shape, generator=g, device=DEV) - int(np.log2(60 * inn**0.5))
    if scales == "e8m0":
        s = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    else:
        s = torch.exp2(e.float()) * (1 + torch.rand(shape, generator=g, device=DEV))
    return q[:, :, :inn], s


def values(w, e):
    """an expert's weight in 64 bits"""
    q, s = w[0][e].double(), w[1][e].double()
    return q * s.repeat_interleave(128, 0)[: q.shape[0]].repeat_interleave(128, 1)[:, : q.shape[1]]


def inputs(tokens, experts, hidden, dtype, g, masked):
    x = torch.randn((tokens, hidden), generator=g, device=DEV)
    x[:, :: max(1, hidden // 5)] *= 10
    logits = torch.randn((tokens, experts), generator=g, device=DEV) * 2
    if masked:
        drop = torch.rand((tokens, experts), generator=g, device=DEV) < 0.4
        logits[drop] = -torch.inf
        logits[::5] = -torch.inf
        logits[1::7, 0] = torch.nan
        logits[2::7, experts - 1] = torch.inf
    return x.to(dtype), logits


def reference(x, logits, w1, w2, top_k, renormalise, residual):
    """y and how far it may be off, in 64 bits"""
    tokens, hidden = x.shape
    width, experts = w2[0].shape[2], w1[0].shape[0]
    chosen, p, *_ = O.route(logits.float().cpu().numpy(), top_k, renormalise)
    unit, parts = 2.0**-23, 3 if x.dtype is F32 else 1
    # sums: a rounding (2^-23, in case the matrix cores cut off) for each of the 128 terms of a block, for each part of an operand, for each block, the eight partial sums
    # and the parts of the columns, relative to the sum of magnitudes
    up_steps, down_steps = 128 * parts + -(-hidden // 128) + 8, 128 * 3 + -(-width // 128) + 8 + 16 + top_k
    split = 2.0**-23 if x.dtype is F32 else 2.0**-17   # of h: 24 or 16 bits
    xd = x.double()
    y, off = torch.zeros((tokens, hidden), dtype=torch.float64, device=DEV), torch.zeros((tokens, hidden), dtype=torch.float64, device=DEV)
    finite = np.where(np.isfinite(logits.float().cpu().numpy()), logits.float().cpu().numpy(), 0)
    p_off = (np.abs(finite).max() * 2 + experts + 8) * unit   # of a softmax: the differences' rounding, the exponentials, their sum
    for e in range(experts):
        t, j = np.nonzero(chosen == e)
        if len(t) == 0:
            continue
        pt = torch.from_numpy(p[t, j]).to(DEV)[:, None]
        t = torch.from_numpy(t).to(DEV)
        a, b = values(w1, e), values(w2, e)
        s, size = xd[t] @ a.T, xd[t].abs() @ a.abs().T
        sg, su = (up_steps * unit * v for v in size.chunk(2, 1))
        gate, u = s.chunk(2, 1)
        silu = gate * torch.sigmoid(gate)
        h = silu * u
        h_off = 1.1 * sg * u.abs() + silu.abs() * su + 1.1 * sg * su + (2.0**-21 + split) * h.abs()   # |d silu / dg| <= 1.1; the gate 8 * 2^-24
        y[t] += pt * (h @ b.T)
        off[t] += pt * (h_off @ b.abs().T + (down_steps * unit + p_off) * (h.abs() @ b.abs().T))
    if residual is not None:
        y += residual.double()
        off += 2.0**-24 * y.abs()
    return y, off + EPS[x.dtype] * y.abs() + (2.0**-25 if x.dtype is F16 else 0)


def check(y, want, off):
    d = (y.double() - want).abs()
    assert (d <= off).all(), f"{(d / off).max().item():.2f} times what it may be"


SHAPES = [  # tokens, experts, top_k, hidden, width
    (1, 1, 1, 8, 1), (1, 8, 2, 512, 768), (2, 4, 2, 130, 100), (3, 5, 3, 300, 33), (4, 2, 1, 127, 129), (7, 4, 2, 512, 768), (15, 16, 4, 257, 130), (16, 8, 2, 2001, 1056),
    (17, 8, 8, 640, 256), (31, 60, 6, 384, 200), (33, 64, 6, 1024, 131), (48, 3, 3, 200, 1001), (57, 64, 6, 1024, 384), (64, 2, 2, 1300, 512), (64, 128, 8, 256, 64),
    (5, 300, 4, 128, 16), (64, 1024, 32, 64, 16), (1, 1024, 32, 64, 20),
]


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,experts,top_k,hidden,width", SHAPES)
def test_layer(tokens, experts, top_k, hidden, width, dtype, scales):
    g = rng(tokens + 7 * hidden + width)
    w1, w2 = weights(g, experts, 2 * width, hidden, scales), weights(g, experts, hidden, width, scales)
    for masked in (False, True):
        x, logits = inputs(tokens, experts, hidden, dtype, g, masked)
        residual = torch.randn((tokens, hidden), generator=g, device=DEV).to(dtype) if masked else None
        y = B.expert_layer_f8(x, logits, w1, w2, top_k, renormalise=not masked, residual=residual)
        assert y.dtype is dtype and y.shape == x.shape
        check(y, *reference(x, logits, w1, w2, top_k, not masked, residual))


LONG = [  # more columns, more units of work than workgroups, experts with more tokens than a unit takes
    (9, 8, 2, 2300, 1056), (20, 4, 2, 2300, 260), (40, 3, 2, 4096, 640), (12, 6, 2, 5001, 520), (40, 3, 2, 5001, 520), (10, 4, 2, 8200, 264), (64, 2, 2, 8200, 264), (64, 4, 4, 1500, 640),
    (50, 5, 2, 2300, 131), (64, 2, 1, 2300, 1001), (64, 64, 8, 2304, 1024), (1, 16, 8, 4096, 1536), (5, 4, 3, 6144, 2048),
]


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,experts,top_k,hidden,width", LONG)
def test_longer(tokens, experts, top_k, hidden, width, dtype, scales):
    g = rng(tokens + 7 * hidden + width)
    w1, w2 = weights(g, experts, 2 * width, hidden, scales), weights(g, experts, hidden, width, scales)
    x, logits = inputs(tokens, experts, hidden, dtype, g, tokens % 2 == 0)
    residual = torch.randn((tokens, hidden), generator=g, device=DEV).to(dtype)
    check(B.expert_layer_f8(x, logits, w1, w2, top_k, residual=residual), *reference(x, logits, w1, w2, top_k, True, residual))
