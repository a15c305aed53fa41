"""8-bit weights written where the caller wants them: an expert among the others of a layer."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_gpu_f8 import BF16, DEV, F16, acts, rng

pytestmark = pytest.mark.gpu
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def pair(*shape, ld=None):
    *e, out, inn = shape
    ld = ld or -(-inn // 128) * 128
    q = torch.full((*e, out, ld), 0x55, dtype=torch.uint8, device=DEV).view(F8)[..., :inn]
    return q, torch.full((*e, -(-out // 128), -(-inn // 128)), 0x55, dtype=torch.uint8, device=DEV).view(E8)


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("out,inn", [(1, 100), (1, 128), (40, 100), (130, 256), (257, 1000)])
@pytest.mark.parametrize("extra", [0, 16, 256])
def test_into_a_given_pair(out, inn, extra):
    g = rng(out)
    w = acts(g, 3 * out, inn, BF16).view(3, out, inn)
    want = B.quantise_weight_f8(w)
    all_ = pair(3, out, inn, ld=-(-inn // 16) * 16 + extra)
    assert B.quantise_weight_f8(w, out=all_) is all_ and same(all_, want)
    all_ = pair(3, out, inn)
    for e in (2, 0):
        B.quantise_weight_f8(w[e], out=(all_[0][e], all_[1][e]))
        assert same((all_[0][e], all_[1][e]), (want[0][e], want[1][e]))
    assert (all_[0][1].view(torch.uint8) == 0x55).all() and (all_[1][1].view(torch.uint8) == 0x55).all()


def test_restored_into_a_given_pair():
    g = rng(7)
    ps = B.PackedStack.from_dense(torch.randn((96, 256), generator=g, device=DEV), torch.ones(256).numpy(), n=2, iterations=4)
    want = ps.restore_weight_f8(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        given = pair(96, 256)
        side.wait_stream(torch.cuda.current_stream())
        assert ps.restore_weight_f8(2, out=given, stream=stream) is given
        torch.cuda.synchronize()
        assert same(given, want)


def test_refusals():
    w = torch.zeros((40, 100), dtype=F16, device=DEV)
    q, s = pair(40, 100)
    bare = torch.zeros((39 * 112 + 100,), dtype=torch.uint8, device=DEV).as_strided((40, 100), (112, 1)).view(F8)   # nothing behind the last row
    for out in ((q[:39], s), (q, s.view(torch.uint8)), (q.view(torch.uint8), s), (q, s[:, :0]), (q[None], s[None]), (q.cpu(), s), (q.t().contiguous().t(), s), (bare, s)):
        with pytest.raises(ValueError):
            B.quantise_weight_f8(w, out=out)
    odd = torch.zeros((40, 104), dtype=torch.uint8, device=DEV).view(F8)[:, :100]
    with pytest.raises(B.BitStackError) as e:
        B.quantise_weight_f8(w, out=(odd, s))
    assert e.value.code == -4


@pytest.mark.parametrize("tokens", [5, 64, 65, 3000])
def test_routing_keeps_its_tables_alone(tokens):
    experts, top_k = 512, 2
    logits = torch.randn((tokens, experts), device=DEV)
    B.route(logits, top_k)
    r = B.route(logits, top_k)
    held = r.offsets.untyped_storage().nbytes()
    assert all(t.untyped_storage().data_ptr() == r.offsets.untyped_storage().data_ptr() for t in r)
    assert held <= 4 * (4 * tokens * top_k + experts + 1) + 512
