"""Where the rows of a layer of experts lie, taken from the tensor's strides (no GPU: only the argument block is filled)."""
import pytest
import torch

import paper_2410_23918_amd as B


def fill(e, out, inn, ld):
    B.linear_f8   # loads f8.py
    from paper_2410_23918_amd import f8
    q = torch.zeros((e, out, ld), dtype=torch.uint8).view(torch.float8_e4m3fn)[:, :, :inn]
    s = torch.zeros((e, -(-out // 128), -(-inn // 128)))
    assert f8._fill_weight(q, s, True) == (out, inn, e)
    return f8._args.w.ld


@pytest.mark.parametrize("e,out,inn,ld", [(4, 1, 100, 128), (4, 1, 100, 112), (3, 1, 256, 512), (1, 1, 100, 128), (4, 2, 100, 128), (1, 5, 48, 64)])
def test_rows_of_the_experts(e, out, inn, ld):
    """also those of one row each, which have no distance of their own: it is the one between the experts"""
    got = fill(e, out, inn, ld)
    assert got == ld or (e == out == 1 and got >= inn and got % 16 == 0)


def test_experts_apart_are_refused():
    B.linear_f8
    from paper_2410_23918_amd import f8
    q = torch.zeros((4, 6, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)[::2, :2]
    with pytest.raises(ValueError):
        f8._fill_weight(q, torch.zeros((2, 1, 1)), True)
