"""The example's layer of experts at sizes that its one call for a few tokens does not take."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_gpu_expert_layer import example  # noqa: F401

pytestmark = pytest.mark.gpu


def weights(experts, out, inn, ld, g):
    q, s = B.quantise_weight_f8(torch.randn((experts, out, inn), generator=g, device="cuda") * inn**-0.5)
    room = torch.empty((experts * out * ld,), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).as_strided(q.shape, (out * ld, ld, 1))
    room.view(torch.uint8).copy_(q.view(torch.uint8))
    return room, s


@pytest.mark.parametrize("hidden,width,experts,ld", [(4, 16, 3, 16), (7, 130, 3, 16), (256, 1024, 1, 1 << 22)])
@pytest.mark.parametrize("tokens", [1, 64])
def test_few_tokens(example, hidden, width, experts, ld, tokens):   # noqa: F811
    """hidden sizes below 8; an expert's w1 of 8 GiB.  Bringing x and the gated values to 8 bits: half a step is 2^-4 of a value, and of a sum of two as much at most for each side;
    twice, times the gate's slope of 1.1, and twice for gate and value: 0.3 of the norm, where a wrong row or expert is off by all of it."""
    g = torch.Generator(device="cuda")
    g.manual_seed(hidden + tokens)
    router = torch.randn((experts, hidden), generator=g, device="cuda")
    layer = example.ExpertLayer(router, weights(experts, 2 * width, hidden, ld, g), weights(experts, hidden, width, -(-width // 16) * 16, g), min(2, experts))
    x = torch.randn((tokens, hidden), generator=g, device="cuda").to(torch.bfloat16)
    y, want = layer(x), example.plain(layer, x)
    assert y.shape == x.shape and ((y.float() - want).norm() / want.norm()).item() < 0.3
