"""Forms of arguments that the entry points of the 8-bit products take."""
import pytest
import torch

import paper_2410_23918_amd as B
from test_gpu_experts import check_grouped
from test_gpu_f8 import BF16, DEV, F32, acts, rng

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inn", [100, 128, 300])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_experts_of_one_row(dtype, inn):
    """as quantise_weight_f8 lays them out"""
    g = rng(inn)
    q, s = B.quantise_weight_f8(torch.randn((4, 1, inn), generator=g, device=DEV))
    x = acts(g, 21, inn, dtype)
    off = [0, 5, 5, 6, 21]
    y = B.grouped_linear_f8(x, q, s, torch.tensor(off, dtype=torch.int32, device=DEV))
    check_grouped(y, x, q, s, off, None, dtype)
