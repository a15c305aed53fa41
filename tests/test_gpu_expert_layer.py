"""The example's layer of experts, from stacks of blocks to outputs."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(os.path.dirname(HERE), "examples", "expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens", [1, 19, 300])
def test_layer(example, tokens):
    """Bringing x and the gated values to 8 bits costs up to 2^-4 of an element each time, some 3 % of a sum of independent ones; bf16 between the products
    2^-9.  10 % of the norm holds that three times over; a wrong expert, row or weight is off by 100 %."""
    layer = example.make(hidden=256, width=512, experts=5, blocks=2)
    x = torch.randn((tokens, 256), device="cuda").to(torch.bfloat16)
    y = layer(x)
    want = example.plain(layer, x)
    assert y.dtype is torch.bfloat16 and tuple(y.shape) == (tokens, 256)
    assert ((y.float() - want).norm() / want.norm()).item() < 0.1


def test_restored_weight_in_8_bits():
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    ps = B.PackedStack.from_dense(torch.randn((288, 512), generator=g, device="cuda"), np.ones(512), n=2, iterations=4)
    dense = ps.restore_weight(2).double().cpu().numpy()
    want, e = O.quantise_weight(dense)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        q, s = ps.restore_weight_f8(2, stream=stream)
        torch.cuda.synchronize()
        assert np.array_equal(s.view(torch.uint8).cpu().numpy().astype(int) - 127, e)
        assert np.array_equal(O.weight_values(q.double().cpu().numpy(), np.ldexp(1.0, e)), want)
    scratch = torch.empty((288, 512), dtype=torch.float16, device="cuda")
    q2, s2 = ps.restore_weight_f8(2, w_dense=scratch)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scratch.double().cpu(), torch.from_numpy(dense))
