"""Every entry point of the 8-bit products on a stream that is not the current one: after what that stream has to do before, with inputs dropped and
their memory asked for again at once."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_gpu_f8 import BF16, DEV, F16, acts, rng, weight

pytestmark = pytest.mark.gpu


def values(r):
    if isinstance(r, B.F8Rows):
        return [r.q.view(torch.uint8), r.scales]
    return [t.view(torch.uint8) if t.element_size() == 1 else t for t in ([r] if isinstance(r, torch.Tensor) else list(r))]


def calls():
    g = rng(41)
    q, s = weight(g, 256, 640, "e8m0", experts=5)
    off = torch.tensor([0, 100, 100, 300, 301, 700], dtype=torch.int32, device=DEV)
    rows = torch.randint(0, 500, (700,), generator=g, device=DEV, dtype=torch.int32)
    slots = torch.randperm(700, generator=g, device=DEV).view(350, 2).to(torch.int32)
    weights = torch.rand((350, 2), generator=g, device=DEV)
    return {
        "quantise": (lambda x, **k: B.quantise_f8(x, **k), lambda: (acts(rng(1), 500, 640, BF16),)),
        "quantise_gated": (lambda x, **k: B.quantise_f8(x, gated=True, **k), lambda: (acts(rng(2), 500, 640, BF16),)),
        "quantise_weight": (lambda w, **k: B.quantise_weight_f8(w, **k), lambda: (acts(rng(3), 600, 640, F16),)),
        "linear": (lambda x, **k: B.linear_f8(x, q[0], s[0], **k), lambda: (acts(rng(4), 500, 640, F16),)),
        "grouped": (lambda x, o, r, **k: B.grouped_linear_f8(x, q, s, o, r, **k), lambda: (acts(rng(5), 500, 640, F16) * 0.1, off.clone(), rows.clone())),
        "grouped_rows_in_8_bits": (lambda x, o, **k: B.grouped_linear_f8(x, q, s, o, **k), lambda: (B.quantise_f8(acts(rng(6), 700, 640, F16) * 0.1), off.clone())),
        "route": (lambda l, **k: B.route(l, 3, **k), lambda: (torch.randn((900, 50), generator=rng(7), device=DEV),)),
        "combine": (lambda h, p, w, **k: B.combine(h, p, w, **k), lambda: (acts(rng(8), 700, 512, F16), slots.clone(), weights.clone())),
    }


NAMES = ["quantise", "quantise_gated", "quantise_weight", "linear", "grouped", "grouped_rows_in_8_bits", "route", "combine"]


@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream(name):
    call, make = calls()[name]
    want = values(call(*make()))
    side = torch.cuda.Stream()
    busy = torch.randn((2048, 2048), device=DEV)
    for _ in range(3):
        inputs = make()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):   # some work in front of the call
            for _ in range(20):
                busy = busy @ busy * 1e-3
        out = call(*inputs, stream=side)
        sizes = [t.numel() * t.element_size() for t in inputs if isinstance(t, torch.Tensor)]
        del inputs
        over = [torch.full((n,), 0xEE, dtype=torch.uint8, device=DEV) for n in sizes]   # on the current stream, while the call waits its turn
        torch.cuda.current_stream().wait_stream(side)
        got = values(out)
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
        del over, out, got


def test_given_output_and_workspace_on_another_stream():
    g = rng(9)
    q, s = weight(g, 256, 640, "f32", experts=3)
    off = torch.tensor([0, 70, 70, 200], dtype=torch.int32, device=DEV)
    x = acts(g, 200, 640, F16) * 0.1
    want = B.grouped_linear_f8(x, q, s, off)
    side = torch.cuda.Stream()
    y = torch.zeros_like(want)
    ws = torch.empty(B.f8_workspace_bytes(200, 640, 200, 256, 3), dtype=torch.uint8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    assert B.grouped_linear_f8(x, q, s, off, y=y, workspace=ws, stream=side) is y
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    slots = torch.arange(200, device=DEV).view(100, 2).to(torch.int32)
    weights = torch.rand((100, 2), generator=g, device=DEV)
    out = torch.zeros((100, 256), dtype=F16, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    assert B.combine(y, slots, weights, y=out, stream=side) is out
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, B.combine(y, slots, weights))
