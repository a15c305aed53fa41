"""Gates and values further apart than 31-bit offsets reach: the plan of such a call (no GPU: it comes from sizes, and refusals before anything is enqueued)."""
import ctypes as C

import pytest

from test_f8_epilogue_host import L, RANGE, SHAPE, SIZE, call, structs  # noqa: F401

GATED = dict(activation=5, ld_residual=1024)


@pytest.mark.parametrize("out,ld,inside", [(512, 1 << 22, False), (512, (1 << 22) - 16, True), (256, 1 << 22, True), (1536, 1 << 21, False), (1024, 1 << 22, False), (500, 1 << 22, False)])
def test_they_meet_inside_the_product_or_in_memory(L, out, ld, inside):   # noqa: F811
    """inside: (out / 2 + 256) ld < 2^31, and then no more workspace than without gates; else the fp32 sums of all rows"""
    assert inside == (out // 2 % 128 == 0 and (out // 2 + 256) * ld < 1 << 31)
    s = structs(None, dict(out=out, ld=ld), GATED)
    need = L.bitstack_f8_epilogue_call_workspace_bytes(*(C.byref(v) for v in s), 0)
    plain = L.bitstack_f8_call_workspace_bytes(C.byref(s[0]), C.byref(s[1]), 40, 0, 0)
    assert need == plain if inside else need >= plain + 40 * out * 4
    assert need and call(L, w=dict(out=out, ld=ld), e=GATED, ld_y=1024, ws_bytes=need - 1) == SIZE


def test_what_is_refused(L):   # noqa: F811
    wide = dict(ld_y=1 << 20, ws_bytes=256)
    e = dict(activation=5, ld_residual=1 << 20)
    assert call(L, w=dict(out=2048, ld=1 << 22), e=e, **wide) == RANGE   # 4 GiB
    assert call(L, w=dict(out=2048, ld=(1 << 22) - 16), e=e, **wide) == SIZE
    assert call(L, w=dict(out=2050, ld=1 << 22), e=e, **wide) == SIZE    # they share a block
    assert call(L, w=dict(out=2048, ld=(1 << 22) + 16), e=e, **wide) == SHAPE
    assert call(L, w=dict(out=2048, ld=1 << 60), e=e, **wide) == SHAPE


def test_sizes_for_up_to_so_many_rows(L):   # noqa: F811
    """of a weight whose rows lie next to each other: 2^20 columns put 4096 rows 4 GiB apart"""
    size = L.bitstack_f8_epilogue_workspace_bytes
    s = structs(dict(ld=1 << 20), dict(out=4096, inn=1 << 20, ld=1 << 20), dict(activation=5, ld_residual=2048))
    need = L.bitstack_f8_epilogue_call_workspace_bytes(*(C.byref(v) for v in s), 0)
    assert size(40, 1 << 20, 4096, 5) >= need >= 40 * 4096 * 4
