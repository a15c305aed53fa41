"""Which of its two ways the example's layer of experts takes, from sizes alone (no GPU: the weights have no data)."""
import importlib.util
import os

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))


def layer(experts, top_k, hidden, width, ld=None):
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(os.path.dirname(HERE), "examples", "expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    ld = ld or -(-hidden // 128) * 128
    q = torch.empty((1,), dtype=torch.float8_e4m3fn, device="meta").as_strided
    return m.ExpertLayer(None, (q((experts, 2 * width, hidden), (2 * width * ld, ld, 1)), None), None, top_k)


@pytest.mark.parametrize("sizes,tokens,dtype,one", [
    ((64, 6, 4096, 1024), 64, torch.bfloat16, True), ((64, 6, 4096, 1024), 65, torch.bfloat16, False), ((64, 6, 4096, 1024), 5, torch.float32, True),
    ((64, 6, 4096, 1024), 64, torch.float32, False), ((8, 2, 4096, 14336), 1, torch.float16, True), ((8, 2, 4096, 14336), 32, torch.float16, True),
    ((8, 2, 4096, 14336), 33, torch.float16, False), ((8, 2, 4096, 14336), 2, torch.float32, True), ((8, 2, 4096, 14336), 3, torch.float32, False),
    ((384, 8, 7168, 2048), 1, torch.bfloat16, False), ((4, 2, 512, 768), 64, torch.float32, True), ((8, 2, 2001, 1056), 64, torch.bfloat16, True),
    ((8, 2, 2048, 8192), 32, torch.float32, True), ((8, 2, 2048, 8192), 33, torch.float32, False),
    ((4, 2, 7, 16), 3, torch.float16, False), ((4, 2, 8, 16), 3, torch.float16, True), ((1, 1, 256, 512, 1 << 22), 3, torch.float16, False),
    ((1, 1, 256, 511, 1 << 22), 3, torch.float16, True), ((1, 1, 8, 1 << 15), 3, torch.float16, True), ((1, 1, 8, (1 << 15) + 1), 3, torch.float16, False),
])
def test_one_call_or_four(sizes, tokens, dtype, one):
    l = layer(*sizes)
    assert l.in_one_call(torch.empty((tokens, sizes[2]), dtype=dtype, device="meta")) == one
