"""The hook that forces a kernel, for gates and values that share a block of 128 (no GPU: plans come from sizes)."""
import ctypes as C

import pytest

import paper_2410_23918_amd as B
from test_f8_epilogue_host import L, structs  # noqa: F401
from test_f8_forced import PAIRS, TOKENS, forced  # noqa: F401


def sums(L, rows, out, inn, y):   # noqa: F811
    """bytes of the partial sums, all that such a call with rows in 8 bits needs"""
    s = structs(dict(dtype=3, rows=rows), dict(out=out, inn=inn, ld=-(-inn // 16) * 16), dict(activation=5, ld_residual=out))
    return L.bitstack_f8_epilogue_call_workspace_bytes(*(C.byref(v) for v in s), y)


@pytest.mark.parametrize("kernel,y", PAIRS)
def test_the_plan_is_the_forced_kernel(L, forced, kernel, y):   # noqa: F811
    rows, out, inn = 700, 1202, 1803
    own = sums(L, rows, out, inn, y)
    for slices in (1, 3):
        forced(kernel + (1024 * slices if kernel > 64 else 0))
        tile = (256 if kernel > 128 else 128, TOKENS[kernel])
        padded = -(-out // tile[0]) * tile[0] * -(-rows // tile[1]) * tile[1]
        assert sums(L, rows, out, inn, y) == (slices * padded * 4 if kernel > 64 else own)
