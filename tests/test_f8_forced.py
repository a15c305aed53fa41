"""The hook that forces a kernel of the 8-bit products: what it refuses, and that a call's plan is the forced kernel's (no GPU: plans come from sizes)."""
import ctypes as C

import pytest

import paper_2410_23918_amd as B

TOKENS = {16: 16, 17: 16, 32: 32, 64: 64, 65: 64, 128: 128, 129: 128, 256: 256}   # of a kernel's tile
PAIRS = [(k, y) for k in TOKENS for y in (0, 1, 2) if (y != 1 if k in (129, 256) else y == 1 if k == 64 else True)]   # y: 0 fp16, 1 fp32, 2 bf16


@pytest.fixture
def forced():
    yield lambda k: B.set_option(B.OPT_F8_KERNEL, k)
    B.set_option(B.OPT_F8_KERNEL, 0)


def list_bytes(rows, out, inn, y):
    """workspace of a grouped call whose rows are in 8 bits already: the work list, 16 bytes for each tile of rows, and partial sums"""
    B.linear_f8   # loads f8.py
    from paper_2410_23918_amd.f8 import _f8_lib, _Rows, _Weight
    return _f8_lib().bitstack_f8_call_workspace_bytes(C.byref(_Rows(256, 256, 0, 3, rows, 0)), C.byref(_Weight(256, inn, 256, 0, out, inn, 1)), rows, y, 1)


@pytest.mark.parametrize("kernel,y", PAIRS)
def test_the_plan_is_the_forced_kernel(forced, kernel, y):
    forced(kernel)
    rows = 8192
    assert list_bytes(rows, 300, 640, y) == -(-(rows // TOKENS[kernel] + 2) * 16 // 256) * 256
    if kernel > 64:   # two slices of the columns, fp32 sums of whole tiles
        forced(kernel + 2048)
        t = TOKENS[kernel]
        tile_rows = 256 if kernel > 128 else 128
        tiles = (rows // t + 2) * -(-300 // tile_rows)
        assert list_bytes(rows, 300, 640, y) == -(-(rows // t + 2) * 16 // 256) * 256 + 2 * tiles * tile_rows * t * 4


@pytest.mark.parametrize("kernel,y", [(64, 0), (64, 2), (129, 1), (256, 1)])
def test_a_kernel_that_does_not_make_such_outputs(forced, kernel, y):
    own = list_bytes(700, 300, 640, y)
    forced(kernel)
    assert list_bytes(700, 300, 640, y) == own


@pytest.mark.parametrize("value", [1, 15, 63, 127, 255, 257, 16 + 1024, 64 + 2048, 1024, 66 + 1024])
def test_no_such_kernel(forced, value):
    with pytest.raises(B.BitStackError) as e:
        forced(value)
    assert e.value.code == -8
