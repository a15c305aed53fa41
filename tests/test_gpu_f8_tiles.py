"""A product whose tiles, with the kernel that would be fastest, are more than a launch has workgroups."""
import numpy as np
import pytest
import torch

import paper_2410_23918_amd as B
from oracle import f8_oracle as O
from test_gpu_f8 import BF16, DEV, np64, rng, tolerance

pytestmark = pytest.mark.gpu


def test_most_outputs_through_many_experts():
    """100 experts of 2^24 x 16 (27 GB), 200 rows of 2^24 outputs (6.7 GB)"""
    experts, out, inn, rows = 100, 1 << 24, 16, 200
    g = rng(5)
    one = (torch.randn((out, inn), generator=g, device=DEV, dtype=torch.float16) * 60).clamp(-448, 448).to(torch.float8_e4m3fn)
    q = one.view(torch.uint8)[None].repeat(experts, 1, 1).view(torch.float8_e4m3fn)
    s = (torch.arange(experts, device=DEV) % 7 + 117).to(torch.uint8)[:, None, None].repeat(1, out // 128, 1).view(torch.float8_e8m0fnu)
    x = torch.randn((rows, inn), generator=g, device=DEV).to(BF16)
    y = B.grouped_linear_f8(x, q, s, torch.arange(0, 2 * experts + 1, 2, dtype=torch.int32, device=DEV))
    take = torch.cat([torch.tensor([0, 1, out - 2, out - 1], device=DEV), torch.arange(77, out, 65537, device=DEV)])
    x8, _ = O.quantise_rows(np64(x))
    w = np64(one.view(torch.uint8)[take].view(torch.float8_e4m3fn))
    scale = np.repeat(2.0 ** (np.arange(experts) % 7 - 10), 2)[:, None]
    want = x8 @ w.T * scale
    assert (np.abs(np64(y[:, take]) - want) <= tolerance(x8, w, BF16, want / scale) * scale).all()
