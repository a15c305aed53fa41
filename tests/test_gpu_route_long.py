"""Routing of as many tokens as 31-bit places reach."""
import pytest
import torch

import paper_2410_23918_amd as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n", [2**31 - 64, 2**31 - 1])
def test_most_tokens(n):
    """one expert, masked for three tokens (39 GB)"""
    l = torch.zeros((n, 1), dtype=torch.float16, device=DEV)
    masked = [5, 2**30 + 63, n - 2]
    l[masked] = float("-inf")
    r = B.route(l, 1)
    del l
    assert r.offsets.tolist() == [0, n - 3]
    step = 1 << 28
    for a in range(0, n, step):
        b = min(n, a + step)
        token = torch.arange(a, b, dtype=torch.int32, device=DEV)
        out = torch.zeros(b - a, dtype=torch.bool, device=DEV)
        before = torch.zeros_like(token)
        for t in masked:
            out |= token == t
            before += (token > t).to(torch.int32)
        assert torch.equal(r.experts[a:b, 0], torch.where(out, -1, 0).to(torch.int32))
        assert torch.equal(r.weights[a:b, 0], (~out).float())
        assert torch.equal(r.slots[a:b, 0], torch.where(out, -1, token - before))
        assert torch.equal(r.rows[(token - before)[~out].long()], token[~out])
    assert r.rows[n - 3 :].tolist() == [-1] * 3
