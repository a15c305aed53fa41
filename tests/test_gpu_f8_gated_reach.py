"""Gates and values further apart than 31-bit offsets reach, against the definition in 64 bits."""
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, F16, F32, acts, np64, rng, weight
from test_gpu_f8_epilogue import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,scales", [(F16, "f32"), (BF16, "e8m0"), (F32, "f32")], ids=["f16", "bf16", "f32"])
def test_two_gigabytes_apart(dtype, scales):
    """whole blocks of 128 gates, as a weight's columns inside wide rows: (256 + 256) 2^22 is past 2^31 - 1, (128 + 256) 2^22 is not; a workspace that the caller gives, too"""
    ld, inn = 1 << 22, 300
    room = torch.empty((512 * ld,), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    for out in (256, 512):
        g = rng(out)
        near, s = weight(g, out, inn, scales)
        q = room.as_strided((out, inn), (ld, 1))
        q.view(torch.uint8).copy_(near.view(torch.uint8))
        w = O.weight_values(np64(near), np64(s))
        for tokens in (1, 40, 300):
            x = acts(g, tokens, inn, dtype) * 0.003
            bias, residual = torch.randn(out, generator=g, device=DEV), torch.randn((tokens, out // 2), generator=g, device=DEV).to(dtype)
            e = dict(bias=bias, activation="silu_gated", residual=residual)
            y = B.linear_f8(x, q, s, **e)
            check(y, O.quantise_rows(np64(x))[0], w, dtype, bias, "silu_gated", residual)
            ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
            assert torch.equal(B.linear_f8(x, q, s, **e, workspace=ws), y)
