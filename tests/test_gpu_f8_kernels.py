"""Every kernel of the 8-bit products, forced, at sizes where its tiles, its ring or its last block end early, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_experts import check_grouped
from test_gpu_f8 import BF16, DEV, F16, F32, acts, np64, rng, tolerance, weight

pytestmark = pytest.mark.gpu
KERNELS = [16, 17, 32, 64, 65, 128, 129, 256, 65 + 2 * 1024, 128 + 3 * 1024, 256 + 2 * 1024]   # + 1024 x column slices, joined afterwards


@pytest.fixture
def forced():
    yield lambda k: B.set_option(B.OPT_F8_KERNEL, k)
    B.set_option(B.OPT_F8_KERNEL, 0)


SHAPES = [  # tokens, out, in: one to many blocks of columns, odd and even, ends at, before and after a 16-byte piece
    (1, 1, 1), (1, 300, 128), (3, 256, 256), (17, 33, 384), (64, 257, 112), (65, 128, 513), (129, 300, 640), (130, 255, 777), (256, 512, 1000), (257, 513, 1293), (600, 700, 896), (5, 1056, 9000),
]


@pytest.mark.parametrize("dtype,scales", [(F16, "e8m0"), (BF16, "f32"), (F32, "e8m0"), (F32, "f32")], ids=["f16-e8m0", "bf16-f32", "f32-e8m0", "f32-f32"])
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("tokens,out,inn", SHAPES)
def test_linear(forced, tokens, out, inn, kernel, dtype, scales):
    g = rng(tokens + out * 3 + inn)
    q, s = weight(g, out, inn, scales)
    x = acts(g, tokens, inn, dtype) * 0.05
    forced(kernel)
    y = np64(B.linear_f8(x, q, s))
    x8, _ = O.quantise_rows(np64(x))
    w = O.weight_values(np64(q), np64(s))
    want = x8 @ w.T
    assert (np.abs(y - want) <= tolerance(x8, w, dtype, want)).all()


@pytest.mark.parametrize("dtype,scales", [(F16, "e8m0"), (BF16, "f32"), (F32, "e8m0")], ids=["f16-e8m0", "bf16-f32", "f32-e8m0"])
@pytest.mark.parametrize("kernel", KERNELS)
def test_grouped(forced, kernel, dtype, scales):
    g = rng(kernel)
    counts, out, inn = [3, 0, 257, 16, 128, 0, 300, 1], 400, 900
    q, s = weight(g, out, inn, scales, experts=len(counts))
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n = int(off[-1]) + 70
    offsets = torch.from_numpy(off).to(DEV)
    x = acts(g, n, inn, dtype) * 0.05
    forced(kernel)
    check_grouped(B.grouped_linear_f8(x, q, s, offsets), x, q, s, off, None, dtype)
    rows = torch.randint(-1, 38, (n,), generator=g, device=DEV, dtype=torch.int32)
    check_grouped(B.grouped_linear_f8(x[:37], q, s, offsets, rows), x[:37], q, s, off, rows.cpu().numpy(), dtype)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("out", [512, 509])
def test_whole_numbers_and_outputs_inside_a_larger_matrix(forced, kernel, out):
    """exact in any order; also into rows apart, at odd places"""
    g = rng(out)
    tokens, inn = 300, 1100
    q = torch.randint(-1, 2, (out, 1104), generator=g, device=DEV).float().to(torch.float8_e4m3fn)[:, :inn]
    x = torch.randint(-1, 2, (tokens, inn), generator=g, device=DEV).to(F16)
    want = torch.from_numpy(np64(x) @ np64(q).T)
    s = torch.full((-(-out // 128), 9), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    forced(kernel)
    for scales in (s, s.float()):
        for dtype in (F16, F32):
            assert torch.equal(B.linear_f8(x, q, scales, out_dtype=dtype).double().cpu(), want)
    wide = torch.full((tokens, out + 9), 7, dtype=F16, device=DEV)
    B.linear_f8(x, q, s, y=wide[:, 3 : 3 + out])
    assert torch.equal(wide[:, 3 : 3 + out].double().cpu(), want) and (wide[:, :3] == 7).all() and (wide[:, 3 + out :] == 7).all()


@pytest.mark.parametrize("kernel", KERNELS)
def test_many_runs_give_the_same_bits(forced, kernel):
    g = rng(21)
    q, s = weight(g, 1000, 2100, "e8m0")
    x = acts(g, 400, 2100, BF16)
    forced(kernel)
    first = B.linear_f8(x, q, s)
    for _ in range(50):
        assert torch.equal(B.linear_f8(x, q, s), first)
