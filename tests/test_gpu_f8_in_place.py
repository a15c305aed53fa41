"""Products whose y lies over their x."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_gpu_f8 import BF16, DEV, F16, F32, acts, rng, weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16, F32], ids=["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 5, 16, 17, 40, 300])
@pytest.mark.parametrize("out", [16, 1000, 4096])
def test_y_over_x(out, tokens, dtype):
    """the same bits as with y elsewhere: each of many workgroups has all of x"""
    g = rng(tokens + out)
    inn = 4096
    q, s = weight(g, out, inn, "e8m0")
    x = acts(g, tokens, inn, dtype) * 0.003
    bias = torch.randn(out, generator=g, device=DEV)
    for e in ({}, dict(activation="gelu", bias=bias), dict(residual=x[:, :out])):
        want = B.linear_f8(x, q, s, **e)
        for ws in (None, torch.empty(B.f8_epilogue_workspace_bytes(tokens, inn, out, e.get("activation")), dtype=torch.uint8, device=DEV)):
            for _ in range(3):
                a = x.clone()
                y = a[:, :out]
                B.linear_f8(a, q, s, **(e | (dict(residual=y) if "residual" in e else {})), y=y, workspace=ws)
                assert torch.equal(y, want) and torch.equal(a[:, out:], x[:, out:])


@pytest.mark.parametrize("tokens", [1, 7, 16])
def test_y_between_the_rows_of_x(tokens):
    """x and y side by side in the rows of one matrix share nothing: no workspace is needed"""
    g = rng(tokens)
    q, s = weight(g, 512, 1024, "e8m0")
    both = torch.zeros((tokens, 1536), dtype=F16, device=DEV)
    x, y = both[:, :1024], both[:, 1024:]
    x.copy_(acts(g, tokens, 1024, F16) * 0.003)
    want = B.linear_f8(x.clone(), q, s)
    assert B.linear_f8(x, q, s, y=y, workspace=torch.empty(0, dtype=torch.uint8, device=DEV)) is y
    assert torch.equal(y, want)


def test_captured():
    g = rng(1)
    q, s = weight(g, 2048, 2048, "f32")
    x = acts(g, 3, 2048, BF16) * 0.003
    a, side = x.clone(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.linear_f8(a, q, s, residual=a, y=a)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.linear_f8(a, q, s, residual=a, y=a)
    torch.cuda.synchronize()
    for i in range(4):
        a.copy_(x.roll(i, 1))
        want = B.linear_f8(x.roll(i, 1), q, s, residual=x.roll(i, 1))
        graph.replay()
        assert torch.equal(a, want)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F16, F32], ids=["f16", "f32"])
@pytest.mark.parametrize("tokens", [1, 19, 64])
def test_a_layer_of_experts_over_its_x(tokens, dtype):
    """x is read by the first of its two kernels, y written by the second"""
    from test_gpu_f8_layer_use import make
    x, logits, w1, w2, k = make(tokens=tokens, experts=6, top_k=3, hidden=640, width=384, dtype=dtype)
    want = B.expert_layer_f8(x, logits, w1, w2, k)
    for _ in range(3):
        a = x.clone()
        assert torch.equal(B.expert_layer_f8(a, logits, w1, w2, k, y=a), want)
    want = B.expert_layer_f8(x, logits, w1, w2, k, residual=x)
    a = x.clone()
    assert torch.equal(B.expert_layer_f8(a, logits, w1, w2, k, residual=a, y=a), want)
