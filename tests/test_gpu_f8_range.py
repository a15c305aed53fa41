"""Products whose scales lie far apart: rows near the ends of fp32's range and weights whose scales bring y back into it, in every kernel."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, F32, np64, rng, tolerance

pytestmark = pytest.mark.gpu
KERNELS = {BF16: [16, 17, 32, 65, 128, 129, 256, 65 + 2 * 1024], F32: [16, 17, 32, 64, 65, 128, 128 + 2 * 1024]}   # those that make such outputs


@pytest.fixture
def forced():
    yield lambda k: B.set_option(B.OPT_F8_KERNEL, k)
    B.set_option(B.OPT_F8_KERNEL, 0)


def operands(tokens, out, inn, dtype, scales, x_size, w_scale, experts=None):
    """all of one sign, so that a block's sum is as large as it can be; w_scale is rounded to a power of two where the scales are"""
    g = rng(tokens + out + inn)
    e = experts or 1
    x = ((torch.rand((tokens, inn), generator=g, device=DEV) + 1) * x_size).to(dtype)
    q = (torch.rand((e, out, -(-inn // 16) * 16), generator=g, device=DEV) * 300 + 148).to(torch.float8_e4m3fn)[:, :, :inn]
    shape = (e, -(-out // 128), -(-inn // 128))
    if scales == "e8m0":
        s = torch.full(shape, int(np.rint(np.log2(w_scale))) + 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    else:
        s = (torch.rand(shape, generator=g, device=DEV, dtype=torch.float64) + 0.5).mul(w_scale).float()
    return x, (q, s) if experts else (q[0], s[0])


# (size of x, the weight's scale): the activations' scale on a block's sum, or the weight's, or both, would pass fp32's range or leave it below
SIZES = [(2e36, 1e-4), (8e37, 1e-12), (2e36, 1e-36), (1e-36, 1e4), (1e-36, 1e30), (1e-38, 1e36)]


@pytest.mark.parametrize("x_size,w_scale", SIZES)
@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype,kernel", [(d, k) for d in KERNELS for k in KERNELS[d]], ids=lambda v: str(v).replace("torch.", ""))
def test_scales_far_apart(forced, dtype, kernel, scales, x_size, w_scale):
    forced(kernel)
    for tokens, out, inn in ((5, 96, 528), (150, 260, 1100)):
        if kernel >= 1024 and inn < 1024:
            continue
        x, (q, s) = operands(tokens, out, inn, dtype, scales, x_size, w_scale)
        x8, _ = O.quantise_rows(np64(x))
        w = O.weight_values(np64(q), np64(s))
        want = x8 @ w.T
        assert np.isfinite(want).all() and (np.abs(want) < 3e38).all() and (np.abs(want) > 1e-37).all()
        assert (np.abs(np64(B.linear_f8(x, q, s)) - want) <= tolerance(x8, w, dtype, want)).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_scales_far_apart_grouped(dtype):
    x, (q, s) = operands(90, 200, 600, dtype, "f32", 2e36, 1e-4, experts=3)
    y = np64(B.grouped_linear_f8(x, q, s, torch.tensor([0, 40, 41, 90], dtype=torch.int32, device=DEV)))
    x8, _ = O.quantise_rows(np64(x))
    for e, (a, b) in enumerate(((0, 40), (40, 41), (41, 90))):
        w = O.weight_values(np64(q[e]), np64(s[e]))
        want = x8[a:b] @ w.T
        assert (np.abs(y[a:b] - want) <= tolerance(x8[a:b], w, dtype, want)).all()


@pytest.mark.parametrize("tokens", [3, 40, 300])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_scales_that_are_zero_denormal_or_no_numbers(dtype, tokens):
    """one row block of the weight each: 0, the least denormal, the least normal and the largest number, infinity, NaN; and 2^-127 and NaN as powers of two"""
    scales = [0.0, 2.0**-149, 2.0**-126, float(np.finfo(np.float32).max), float("inf"), float("nan"), 3.0]
    x = torch.full((tokens, 128), 2.0**-60, device=DEV).to(dtype)
    q = torch.ones((128 * len(scales), 128), device=DEV).to(torch.float8_e4m3fn)
    want = np.repeat(np.array(scales), 128) * 2.0**-53
    got = np64(B.linear_f8(x * 2.0**60 if dtype is F32 else x, q, torch.tensor(scales, device=DEV)[:, None]))
    want = want * 2.0**60 if dtype is F32 else want
    for i, s in enumerate(scales):
        mine, ref = got[:, 128 * i : 128 * (i + 1)], want[128 * i]
        if np.isnan(s):
            assert np.isnan(mine).all()
        elif np.isinf(s) or abs(ref) > 3.4e38:
            assert (mine == np.inf).all()
        elif ref < 2.0**-126:
            assert (np.abs(mine - ref) <= 2.0**-126).all()   # a denormal may be zero
        else:
            assert (mine == float(torch.tensor(ref).to(dtype))).all()
    bytes_ = torch.tensor([0, 255, 130], dtype=torch.uint8, device=DEV)[:, None].view(torch.float8_e8m0fnu)
    x = torch.full((tokens, 128), 2.0**60, device=DEV).to(dtype)
    got = np64(B.linear_f8(x, q[:384], bytes_))
    assert (got[:, :128] == 2.0**-60).all() and np.isnan(got[:, 128:256]).all() and (got[:, 256:] == 2.0**70).all()
