"""Products of more tiles than a launch has workgroups are refused before anything is enqueued (the device pointers are never followed)."""
import ctypes as C

import pytest

import paper_2410_23918_amd as B

RANGE, P = -3, 1 << 20


@pytest.mark.parametrize("y_dtype,rows,out,experts", [(0, 2**31 - 1, 1, 1), (2, 2**31 - 1, 1, 1024), (1, 2**30 + 128, 1, 1), (0, 2**20, 2**24, 1), (1, 2**23, 2**20, 64)])
def test_more_tiles_than_workgroups(y_dtype, rows, out, experts):
    B.linear_f8   # loads f8.py
    from paper_2410_23918_amd.f8 import _f8_lib, _Rows, _Weight
    x, w = _Rows(P, P, 16, 0, 3, 0), _Weight(P, 16, P, 0, out, 16, experts)
    assert _f8_lib().bitstack_f8_grouped_linear(C.byref(x), C.byref(w), P, P, rows, P, y_dtype, out, P, 1 << 50, None) == RANGE
