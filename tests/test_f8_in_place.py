"""A product whose y lies over its x: what it needs and what is refused (no GPU: nothing is enqueued, the pointers are never followed)."""
import ctypes as C

import pytest

from test_f8_epilogue_host import L, NULL, SIZE, structs  # noqa: F401

P = 1 << 30   # an aligned address


def product(L, epilogue, y, ws, n, rows=5, inn=1024, out=1024, ld=1024, ld_y=1024):   # noqa: F811
    x, w, e = structs(dict(x=P, rows=rows, ld=ld), dict(q=1 << 40, scales=1 << 41, out=out, inn=inn, ld=inn), dict(activation=1, ld_residual=ld_y, residual=y))
    if epilogue:
        return L.bitstack_f8_linear_epilogue(C.byref(x), C.byref(w), C.byref(e), y, 0, ld_y, ws, n, None)
    return L.bitstack_f8_linear(C.byref(x), C.byref(w), y, 0, ld_y, ws, n, None)


@pytest.mark.parametrize("epilogue", [False, True])
@pytest.mark.parametrize("rows", [1, 5, 16])
def test_without_a_workspace(L, rows, epilogue):   # noqa: F811
    """few rows, which every workgroup reads for itself while others write: over x they go through a workspace"""
    x, w, e = structs(dict(x=P, rows=rows, ld=1024), dict(out=1024, inn=1024, ld=1024))
    assert L.bitstack_f8_call_workspace_bytes(C.byref(x), C.byref(w), rows, 0, 0) == 0   # for outputs elsewhere
    for y in (P, P + 2, P + 2046, P + (rows - 1) * 2048 + 2046, P - (rows - 1) * 2048 - 2046):
        assert product(L, epilogue, y, None, 0, rows) == NULL, y - P
        assert product(L, epilogue, y, P << 4, 256, rows) == SIZE
    if rows > 1:   # both in the rows of one matrix: x its first 1024 columns of 2047, y its last 1024, and one that is x's
        assert product(L, epilogue, P + 1023 * 2, None, 0, rows, ld=2047 + 1, ld_y=2047 + 1) == NULL
    assert L.bitstack_f8_workspace_bytes(rows, 1024, rows, 1024, 1) >= rows * 1024
