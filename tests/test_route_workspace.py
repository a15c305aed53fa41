"""The routing's workspace: counts for as many chunks as there are (no GPU: sizes only)."""
import pytest

import paper_2410_23918_amd as B


@pytest.mark.parametrize("tokens,experts,top_k,size", [(0, 8, 2, 256), (1, 8, 2, 256), (64, 1024, 8, 256), (65, 128, 8, 1024), (200, 60, 2, 1024), (16384, 128, 8, 131072), (10**6, 128, 8, 131072)])
def test_no_more_than_the_chunks(tokens, experts, top_k, size):
    B.route   # loads f8.py
    from paper_2410_23918_amd import f8
    assert f8._f8_lib().bitstack_route_workspace_bytes(tokens, experts, top_k) == size
