"""The layer of experts for a few tokens as it is called: ties, strides, in place, other streams, captured graphs, shared workspaces, values that are no
numbers, large offsets, and together with the products around it."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_gpu_f8 import BF16, DEV, F16, F32, rng
from test_gpu_f8_layer import check, inputs, reference, values, weights

pytestmark = pytest.mark.gpu


def make(tokens=19, experts=8, top_k=2, hidden=300, width=200, dtype=BF16, scales="e8m0", seed=0, masked=False):
    g = rng(seed)
    w1, w2 = weights(g, experts, 2 * width, hidden, scales), weights(g, experts, hidden, width, scales)
    return (*inputs(tokens, experts, hidden, dtype, g, masked), w1, w2, top_k)


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("experts,top_k", [(3, 3), (16, 5), (17, 4), (64, 16), (64, 17), (128, 8), (256, 6), (257, 6)])
def test_equal_logits(experts, top_k, renormalise):
    """few different logits: of equal ones the lower index is taken"""
    x, _, w1, w2, _ = make(tokens=40, experts=experts, hidden=64, width=40, dtype=F32)
    logits = torch.randint(-1, 2, (40, experts), generator=rng(experts), device=DEV).float()
    logits[0] = 0
    logits[1] = -0.0
    logits[1, ::2] = 0.0
    logits[2] = torch.inf
    check(B.expert_layer_f8(x, logits, w1, w2, top_k, renormalise=renormalise), *reference(x, logits, w1, w2, top_k, renormalise, None))


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("hidden,width", [(300, 200), (129, 33), (1040, 131)])
def test_strides(dtype, hidden, width):
    """rows further apart than they are long and at odd elements, with numbers that are none between them"""
    x, logits, w1, w2, k = make(hidden=hidden, width=width, dtype=dtype)
    n = x.shape[0]
    residual = torch.randn((n, hidden), generator=rng(5), device=DEV).to(dtype)

    def apart(t, fill=torch.nan):
        big = torch.full((n, t.shape[1] + 7), fill, device=DEV, dtype=t.dtype)
        big[:, 3 : 3 + t.shape[1]] = t
        return big, big[:, 3 : 3 + t.shape[1]]
    want = B.expert_layer_f8(x, logits, w1, w2, k, residual=residual)
    check(want, *reference(x, logits, w1, w2, k, True, residual))
    big, y = apart(torch.zeros_like(x), 7.0)
    assert B.expert_layer_f8(apart(x)[1], apart(logits)[1], w1, w2, k, residual=apart(residual)[1], y=y) is y
    assert torch.equal(y, want)
    assert (big[:, :3] == 7).all() and (big[:, 3 + hidden :] == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_logits_of_16_bits(dtype):
    x, logits, w1, w2, k = make()
    logits = logits.to(dtype)
    assert torch.equal(B.expert_layer_f8(x, logits, w1, w2, k), B.expert_layer_f8(x, logits.float(), w1, w2, k))


@pytest.mark.parametrize("tokens", [1, 5, 20, 64])
def test_in_place_and_the_same_bits_every_time(tokens):
    x, logits, w1, w2, k = make(tokens=tokens, experts=6, top_k=3, hidden=640, width=384)
    residual = torch.randn_like(x)
    want = B.expert_layer_f8(x, logits, w1, w2, k, residual=residual)
    for _ in range(20):
        y = residual.clone()
        B.expert_layer_f8(x, logits, w1, w2, k, residual=y, y=y)
        assert torch.equal(y, want)


def test_workspace_for_more_tokens_with_anything_in_it():
    x, logits, w1, w2, k = make(tokens=64, experts=6, top_k=3, hidden=640, width=384)
    n = B.expert_layer_workspace_bytes(64, 640, 384, 6, 3)
    for tokens in (64, 33, 17, 16, 9, 8, 5, 1):
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
        assert torch.equal(B.expert_layer_f8(x[:tokens], logits[:tokens], w1, w2, k, workspace=ws), B.expert_layer_f8(x[:tokens], logits[:tokens], w1, w2, k))
    with pytest.raises(B.BitStackError) as e:
        B.expert_layer_f8(x, logits, w1, w2, k, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.code == -6
    assert B.expert_layer_f8(x[:0], logits[:0], w1, w2, k).shape == (0, 640)
    with pytest.raises(B.BitStackError) as e:
        B.expert_layer_f8(torch.cat([x, x]), torch.cat([logits, logits]), w1, w2, k)
    assert e.value.code == -3


@pytest.mark.parametrize("dtype", [F16, F32], ids=["f16", "f32"])
@pytest.mark.parametrize("tokens", [5, 40])
def test_values_that_are_no_numbers_stay_with_their_tokens(tokens, dtype):
    x, logits, w1, w2, k = make(tokens=tokens, hidden=300, width=200, dtype=dtype)
    want = B.expert_layer_f8(x, logits, w1, w2, k)
    bad = x.clone()
    bad[1, 7] = torch.nan
    bad[3, 299] = torch.inf
    y = B.expert_layer_f8(bad, logits, w1, w2, k)
    others = [t for t in range(tokens) if t not in (1, 3)]
    assert torch.equal(y[others], want[others])
    assert not y[[1, 3]].isfinite().any()   # every weight is finite and hardly any is 0: infinite gates and values, whose sums over width have no value
    # a token without an expert whose x is no number: nothing of it arrives
    masked = logits.clone()
    masked[[1, 3]] = -torch.inf
    y = B.expert_layer_f8(bad, masked, w1, w2, k)
    assert torch.equal(y[others], B.expert_layer_f8(x, masked, w1, w2, k)[others]) and not y[[1, 3]].any()
    # no token has one
    residual = torch.randn_like(x)
    none = torch.full_like(logits, -torch.inf)
    assert torch.equal(B.expert_layer_f8(bad, none, w1, w2, k, residual=residual), residual)
    assert not B.expert_layer_f8(bad, torch.full_like(logits, torch.nan), w1, w2, k).any()


def test_weights_that_are_not_wanted_are_not_looked_at():
    """an expert without tokens may hold anything, and so may what lies between the rows"""
    x, logits, w1, w2, k = make(scales="f32")
    want = B.expert_layer_f8(x, logits, w1, w2, k)
    logits = logits.clone()
    logits[:, 2] = -torch.inf
    want = B.expert_layer_f8(x, logits, w1, w2, k)
    for q, s in (w1, w2):
        q[2].view(torch.uint8)[:] = 0x7F
        s[2] = torch.nan
    assert torch.equal(B.expert_layer_f8(x, logits, w1, w2, k), want)


def test_on_another_stream():
    x, logits, w1, w2, k = make(tokens=30, hidden=640, width=384)
    want = B.expert_layer_f8(x, logits, w1, w2, k, residual=x)
    side, busy = torch.cuda.Stream(), torch.randn((2048, 2048), device=DEV)
    for _ in range(3):
        a, b = x.clone(), logits.clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                busy = busy @ busy * 1e-3
        y = B.expert_layer_f8(a, b, w1, w2, k, residual=a, stream=side)
        sizes = [t.numel() * t.element_size() for t in (a, b)]
        del a, b
        over = [torch.full((n,), 0xEE, dtype=torch.uint8, device=DEV) for n in sizes]   # on the current stream, while the call waits its turn
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y, want)
        torch.cuda.synchronize()
        del over, y


def test_two_graphs_with_one_workspace():
    """captured calls of several sizes, replayed in turn with eager work between; the inputs change between replays"""
    x, logits, w1, w2, k = make(tokens=64, experts=6, top_k=3, hidden=640, width=384)
    ws = torch.empty(B.expert_layer_workspace_bytes(64, 640, 384, 6, 3), dtype=torch.uint8, device=DEV)
    graphs = []
    side = torch.cuda.Stream()
    for tokens in (64, 3):
        a, b, y = x[:tokens].clone(), logits[:tokens].clone(), torch.empty_like(x[:tokens])
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            B.expert_layer_f8(a, b, w1, w2, k, y=y, workspace=ws)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                B.expert_layer_f8(a, b, w1, w2, k, residual=a, y=y, workspace=ws)
        graphs.append((g, a, b, y))
    torch.cuda.synchronize()
    for i in range(4):
        for g, a, b, y in graphs:
            a.copy_(x[: len(a)].roll(i, 1))
            b.copy_(logits[: len(b)].roll(i, 1))
            g.replay()
            want = B.expert_layer_f8(a, b, w1, w2, k, residual=a)
            assert torch.equal(y, want)
            torch.cuda.synchronize()


def test_offsets_past_31_bits():
    """an expert's w1 of 2.3 GB"""
    hidden, width, ld = 256, 280, 1 << 22
    g = rng(3)
    q1 = torch.empty((1, 2 * width * ld), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).as_strided((1, 2 * width, hidden), (2 * width * ld, ld, 1))
    w1, w2 = weights(g, 1, 2 * width, hidden, "f32"), weights(g, 1, hidden, width, "f32")
    q1.view(torch.uint8).copy_(w1[0].view(torch.uint8))
    x, logits = inputs(5, 1, hidden, BF16, g, False)
    y = B.expert_layer_f8(x, logits, (q1, w1[1]), w2, 1)
    assert torch.equal(y, B.expert_layer_f8(x, logits, w1, w2, 1))
    check(y, *reference(x, logits, w1, w2, 1, True, None))


@pytest.mark.parametrize("tokens", [1, 33])
def test_a_decoder_layers_feed_forward(tokens):
    """A dense product with gates, one onto the residual stream, then a layer of experts onto it, against the same in 64 bits from what the first call
    gives: each call reads what the one before wrote."""
    g = rng(tokens)
    hidden, width = 512, 384
    (q1, s1), (q2, s2) = ((t[0][0], t[1][0]) for t in (weights(g, 1, 2 * width, hidden, "e8m0"), weights(g, 1, hidden, width, "e8m0")))
    _, logits, w1, w2, k = make(tokens=tokens, hidden=hidden, width=width)
    x = torch.randn((tokens, hidden), generator=g, device=DEV).to(BF16)
    h = B.linear_f8(x, q1, s1, activation="silu_gated")
    stream = x.clone()
    B.linear_f8(h, q2, s2, residual=stream, y=stream)
    out = B.expert_layer_f8(stream, logits, w1, w2, k, residual=stream, y=torch.empty_like(stream))
    check(out, *reference(stream, logits, w1, w2, k, True, stream))
    # activations in 8 bits: half a step is 2^-4 of a value, which independent roundings bring to some 2 % of a sum of as many; twice, and the gate's slope
    a = x.double() @ values((q1[None], s1[None]), 0).T
    gate, u = a.chunk(2, 1)
    want = x.double() + (gate * torch.sigmoid(gate) * u) @ values((q2[None], s2[None]), 0).T
    assert ((stream.double() - want).norm() / want.norm()).item() < 0.1
