"""The products grouped by expert, the routing and the weighted sums against the oracle in 64 bits, through the public entry points."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, EPS, F16, F32, acts, np64, rng, tolerance, weight

pytestmark = pytest.mark.gpu


def check_grouped(y, x, q, s, offsets, rows, dtype, gated=False):
    x = O.gated(np64(x)) if gated else np64(x)
    x8, _ = O.quantise_rows(x)
    got = np64(y)
    end = 0
    for e in range(q.shape[0]):
        a, b = offsets[e], offsets[e + 1]
        end = b
        if a == b:
            continue
        xe = x8[a:b] if rows is None else np.stack([x8[r] if 0 <= r < len(x8) else np.zeros(x8.shape[1]) for r in rows[a:b]])
        w = O.weight_values(np64(q[e]), np64(s[e]))
        want = xe @ w.T
        assert (np.abs(got[a:b] - want) <= tolerance(xe, w, dtype, want)).all(), e
    assert not got[end:].any()


CASES = [  # experts, the rows of each, out, in
    ([1], 64, 128), ([0, 1], 100, 200), ([2, 0, 0, 3], 130, 300), ([16, 15, 17, 1, 0, 33], 96, 513), ([0, 0, 0], 64, 256), ([70, 0, 5, 129], 257, 384),
    ([1] * 40, 48, 256), ([0] * 20 + [300] + [0] * 3, 200, 640), ([64, 64, 128, 256], 128, 512), ([513, 2, 259], 300, 1000), ([3] * 65 + [0] * 70 + [1], 33, 140),
]


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("counts,out,inn", CASES, ids=[f"{len(c[0])}x{max(c[0])}_{c[1]}x{c[2]}" for c in CASES])
def test_grouped(counts, out, inn, dtype, scales):
    g = rng(len(counts) + out)
    q, s = weight(g, out, inn, scales, experts=len(counts))
    s = s if s.dtype is not F32 else s * 0.1
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n = int(off[-1]) + 5   # rows past the last group
    offsets = torch.from_numpy(off).to(DEV)
    x = acts(g, n, inn, dtype) * 0.1
    y = B.grouped_linear_f8(x, q, s, offsets)
    check_grouped(y, x, q, s, off, None, dtype)
    # gathered, some from nowhere
    tokens = 11
    rows = torch.randint(0, tokens, (n,), generator=g, device=DEV, dtype=torch.int32)
    rows[::9] = -1
    rows[4::13] = tokens
    y = B.grouped_linear_f8(x[:tokens], q, s, offsets, rows)
    check_grouped(y, x[:tokens], q, s, off, rows.cpu().numpy(), dtype)


def test_grouped_is_the_single_product_of_every_expert():
    g = rng(77)
    counts, out, inn = [40, 1, 0, 200, 7], 384, 1100
    q, s = weight(g, out, inn, "e8m0", experts=5)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    x = acts(g, int(off[-1]), inn, BF16)
    y = B.grouped_linear_f8(x, q, s, torch.from_numpy(off).to(DEV), out_dtype=F32)
    for e in range(5):
        a, b = off[e], off[e + 1]
        if a < b:   # the same blocks in another order of sums at most
            one = B.linear_f8(x[a:b], q[e], s[e], out_dtype=F32)
            x8, _ = O.quantise_rows(np64(x[a:b]))
            w = O.weight_values(np64(q[e]), np64(s[e]))
            assert (np.abs(np64(one) - np64(y[a:b])) <= 2 * tolerance(x8, w, F32, np64(one))).all()


def test_offsets_that_break_the_rules_stay_inside():
    """an entry below an earlier one counts as that one, an entry past the end as the end"""
    g = rng(6)
    q, s = weight(g, 70, 256, "e8m0", experts=5)
    x = acts(g, 50, 256, BF16)
    y = B.grouped_linear_f8(x, q, s, torch.tensor([3, 20, 10, 1000, -7, 60], dtype=torch.int32, device=DEV), out_dtype=F32)
    check_grouped(y, x, q, s, [0, 20, 20, 50, 50, 50], None, F32)


def test_grouped_gated():
    g = rng(8)
    counts, out, inn = [20, 0, 130, 3], 200, 700
    q, s = weight(g, out, inn, "f32", experts=4)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    offsets = torch.from_numpy(off).to(DEV)
    x = acts(g, int(off[-1]), 2 * inn, F16)
    rows8 = B.quantise_f8(x, gated=True)
    y = B.grouped_linear_f8(x, q, s, offsets, gated=True, out_dtype=F32)
    assert torch.equal(y, B.grouped_linear_f8(rows8, q, s, offsets, out_dtype=F32))
    x8 = np64(rows8.values())
    for e in range(4):
        a, b = off[e], off[e + 1]
        w = O.weight_values(np64(q[e]), np64(s[e]))
        want = x8[a:b] @ w.T
        assert (np.abs(np64(y[a:b]) - want) <= tolerance(x8[a:b], w, F32, want)).all()


@pytest.mark.parametrize("dtype", [F16, F32], ids=["f16", "f32"])
def test_grouped_few_rows(dtype):
    """one to a few tokens decoded: the products bring the rows to 8 bits themselves, gathered ones and ones from nowhere among them"""
    g = rng(31)
    q, s = weight(g, 200, 512, "e8m0", experts=9)
    off = np.array([0, 0, 2, 2, 3, 3, 3, 9, 9, 9], np.int32)
    offsets = torch.from_numpy(off).to(DEV)
    x = acts(g, 4, 512, dtype) * 0.1
    rows = torch.tensor([0, 3, 1, 2, -1, 4, 0, 1, 3, 2, 2], dtype=torch.int32, device=DEV)
    y = B.grouped_linear_f8(x, q, s, offsets, rows)
    check_grouped(y, x, q, s, off, rows.cpu().numpy(), dtype)
    assert torch.equal(y, B.grouped_linear_f8(B.quantise_f8(x), q, s, offsets, rows, out_dtype=dtype))


def test_grouped_without_rows():
    g = rng(10)
    q, s = weight(g, 64, 128, "e8m0", experts=3)
    zero = torch.zeros(4, dtype=torch.int32, device=DEV)
    assert tuple(B.grouped_linear_f8(torch.empty((0, 128), dtype=F16, device=DEV), q, s, zero).shape) == (0, 64)
    y = B.grouped_linear_f8(torch.empty((0, 128), dtype=F16, device=DEV), q, s, torch.tensor([0, 1, 2, 3], dtype=torch.int32, device=DEV),
                            torch.zeros(5, dtype=torch.int32, device=DEV))
    assert tuple(y.shape) == (5, 64) and not y.any()


ROUTES = [(0, 8, 2), (1, 1, 1), (1, 8, 2), (3, 5, 5), (57, 8, 2), (64, 64, 8), (65, 60, 3), (130, 128, 8), (1000, 100, 6), (4096, 16, 4), (700, 256, 8), (200, 1000, 32), (20000, 130, 2)]


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,experts,top_k", ROUTES)
def test_route(tokens, experts, top_k, dtype, renormalise):
    """Whole numbers bit for bit.  Weights: fp32 exponentials of differences up to ~20 (2^-24 * 20 of the argument, 2^-22 of the function), their sum of up
    to 1000 and a quotient, relative 2^-17 at most."""
    g = rng(tokens + experts)
    l = (torch.randn((tokens, experts), generator=g, device=DEV) * 2).to(dtype)
    l = torch.where(torch.rand(l.shape, generator=g, device=DEV) < 0.2, l.round(), l)   # ties
    if tokens > 2:
        l[torch.rand(l.shape, generator=g, device=DEV) < 0.3] = float("-inf")
        l[torch.rand(l.shape, generator=g, device=DEV) < 0.02] = float("nan")
        l[1] = float("-inf")
        l[2] = torch.finfo(dtype).min   # a mask of the lowest value is a number: such experts can be taken
        l[0, 0], l[0, experts - 1] = 0.0, -0.0
    r = B.route(l, top_k, renormalise=renormalise)
    experts_, weights, slots, rows, offsets = O.route(np64(l), top_k, renormalise)
    for got, want in ((r.experts, experts_), (r.slots, slots), (r.rows, rows), (r.offsets, offsets)):
        assert np.array_equal(got.cpu().numpy(), want)
    assert (np.abs(np64(r.weights) - weights) <= 2.0**-17 * weights + 1e-38).all()


def test_route_infinite_logits():
    inf = float("inf")
    l = torch.tensor([[1.0, inf, 2.0, inf], [inf, -inf, 0.0, 1.0], [float("nan")] * 4], device=DEV)
    r = B.route(l, 3)
    assert r.experts.tolist() == [[1, 3, 2], [0, 3, 2], [-1, -1, -1]]
    assert r.weights.tolist() == [[0.5, 0.5, 0.0], [1.0, 0.0, 0.0], [0.0, 0.0, 0.0]]


def test_route_strided_logits():
    l = torch.randn((70, 40), device=DEV)
    a, b = B.route(l[:, 3:13], 2), B.route(l[:, 3:13].contiguous(), 2)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens,width,top_k", [(1, 1, 1), (1, 4096, 2), (57, 4096, 2), (9, 1001, 6), (300, 520, 8), (2, 7, 32)])
def test_combine(tokens, width, top_k, dtype):
    """one rounding of a product-sum per row in fp32, then the output's"""
    g = rng(tokens + width)
    h = torch.randn((tokens * top_k, width), generator=g, device=DEV).to(dtype)
    slots = torch.randperm(tokens * top_k, generator=g, device=DEV).view(tokens, top_k).to(torch.int32)
    weights = torch.rand((tokens, top_k), generator=g, device=DEV)
    slots[::3, 0] = -1
    slots[1::3, top_k - 1] = tokens * top_k   # no row either
    weights[::3, 0] = float("nan")
    y = B.combine(h, slots, weights)
    sl, wt, hh = slots.cpu().numpy(), np64(weights), np64(h)
    want, size = np.zeros((tokens, width)), np.zeros((tokens, width))
    for t in range(tokens):
        for j in range(top_k):
            if 0 <= sl[t, j] < len(hh):
                want[t] += wt[t, j] * hh[sl[t, j]]
                size[t] += abs(wt[t, j] * hh[sl[t, j]])
    assert (np.abs(np64(y) - want) <= top_k * 2.0**-24 * size + EPS[dtype] * np.abs(want) + 1e-7 * (dtype is F16)).all()
    # rows apart, at odd places
    wide = torch.zeros((tokens * top_k, width + 3), dtype=dtype, device=DEV)
    wide[:, 1 : 1 + width] = h
    out = torch.full((tokens, width + 5), 7.0, dtype=dtype, device=DEV)
    B.combine(wide[:, 1 : 1 + width], slots, weights, y=out[:, 2 : 2 + width])
    assert torch.equal(out[:, 2 : 2 + width], y) and (out[:, :2] == 7).all() and (out[:, 2 + width :] == 7).all()


def test_a_layer_of_experts_in_a_graph():
    """the routing, both products and the sums as a decoder calls them, captured once and replayed on other inputs"""
    g = rng(12)
    experts, top_k, hidden, width, tokens = 6, 2, 512, 384, 33
    w1, s1 = B.quantise_weight_f8(torch.randn((experts, 2 * width, hidden), generator=g, device=DEV) * 0.05)
    w2, s2 = B.quantise_weight_f8(torch.randn((experts, hidden, width), generator=g, device=DEV) * 0.05)
    x = torch.randn((tokens, hidden), generator=g, device=DEV).to(BF16)
    logits = torch.randn((tokens, experts), generator=g, device=DEV)

    def layer():
        r = B.route(logits, top_k)
        h = B.grouped_linear_f8(x, w1, s1, r.offsets, r.rows)
        return B.combine(B.grouped_linear_f8(h, w2, s2, r.offsets, gated=True), r.slots, r.weights)

    layer()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer()
    for i in range(4):
        x.copy_(torch.randn((tokens, hidden), generator=rng(i), device=DEV))
        logits.copy_(torch.randn((tokens, experts), generator=rng(i + 10), device=DEV))
        if i == 2:
            logits[5:9] = float("-inf")
        graph.replay()
        torch.cuda.synchronize()
        want = layer()
        assert torch.equal(y, want)
        if i == 2:
            assert not y[5:9].any()


def test_refusals():
    g = rng(5)
    q, s = weight(g, 64, 256, "e8m0", experts=3)
    x = acts(g, 6, 256, F16)
    off = torch.tensor([0, 2, 4, 6], dtype=torch.int32, device=DEV)
    for call in (
        lambda: B.grouped_linear_f8(x, q, s, off.long()),
        lambda: B.grouped_linear_f8(x, q, s, off[:3]),
        lambda: B.grouped_linear_f8(x, q[:2], s, off),
        lambda: B.grouped_linear_f8(x, q, s, off, torch.zeros(6, device=DEV)),
        lambda: B.grouped_linear_f8(x, q[:, :40], s, off),
        lambda: B.combine(x, torch.zeros((2, 2), device=DEV), torch.zeros((2, 2), device=DEV)),
        lambda: B.combine(x, torch.zeros((2, 2), dtype=torch.int32, device=DEV), torch.zeros((2, 3), device=DEV)),
        lambda: B.route(x.double(), 2),
    ):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.route(x[:, :4], 5), lambda: B.route(x[:, :4], 0), lambda: B.route(torch.zeros((2, 1025), device=DEV), 1)):
        with pytest.raises(B.BitStackError) as e:
            call()
        assert e.value.code == -2
