"""CPU-only checks of the 8-bit product with bias, activation and residual: sizes, and refusals, which come before anything is enqueued (the device pointers here are
never followed); and its kernels' assembly, as that of the products without."""
import ctypes as C
import shutil
import subprocess

import pytest
import torch

import paper_2410_23918_amd as B
from test_asm_distances import CSRC, HIPCC, faults, functions, registers, too_close, wrap

OK, NULL, SHAPE, RANGE, ALIGN, SIZE, ARG = 0, -1, -2, -3, -4, -6, -8
P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def L():
    B.linear_f8   # loads f8.py
    from paper_2410_23918_amd import f8
    return f8._f8_lib()


def structs(x=None, w=None, e=None):
    from paper_2410_23918_amd.f8 import _Epilogue, _Rows, _Weight
    weight = dict(q=P, ld=256, scales=P, scale_type=0, out=64, inn=256, experts=1) | (w or {})
    rows = dict(x=P, scales=P, ld=256, dtype=0, rows=40, gated=0) | (x or {})
    epilogue = dict(bias=P, bias_dtype=0, activation=0, residual=P, ld_residual=64) | (e or {})
    return _Rows(**rows), _Weight(**weight), _Epilogue(**epilogue)


def call(L, x=None, w=None, e=None, **change):
    a = dict(y=P, y_dtype=0, ld_y=64, ws=P, ws_bytes=1 << 24) | change
    return L.bitstack_f8_linear_epilogue(*(C.byref(s) for s in structs(x, w, e)), a["y"], a["y_dtype"], a["ld_y"], a["ws"], a["ws_bytes"], None)


def test_refusals(L):
    assert L.bitstack_f8_linear_epilogue(*(C.byref(s) for s in structs()[:2]), None, P, 0, 64, P, 1 << 24, None) == NULL
    for code, e in ((ARG, dict(activation=-1)), (ARG, dict(activation=6)), (ARG, dict(bias_dtype=3)), (ALIGN, dict(bias=P + 1)), (ALIGN, dict(residual=P + 1)), (SHAPE, dict(ld_residual=63))):
        assert call(L, e=e) == code, e
    assert call(L, dict(rows=0)) == OK
    gated = dict(activation=5, ld_residual=32)
    assert call(L, w=dict(out=63), e=gated) == SHAPE
    assert call(L, w=dict(out=64), e=dict(activation=5, ld_residual=31)) == SHAPE
    assert call(L, w=dict(out=64), e=gated, ld_y=31) == SHAPE
    assert call(L, w=dict(out=64), e=gated, ws_bytes=256) == SIZE
    assert call(L, w=dict(out=2048, ld=1 << 22), e=dict(activation=5, ld_residual=1024), ld_y=1024) == RANGE   # gates and values 4 GiB apart
    # what the product without it refuses
    for code, x, w, change in ((NULL, dict(x=None), None, {}), (SHAPE, None, dict(experts=2), {}), (ALIGN, None, dict(q=P + 8), {}), (SHAPE, dict(ld=255), None, {}), (ARG, None, None, dict(y_dtype=3)),
                               (NULL, None, None, dict(y=None)), (SHAPE, None, None, dict(ld_y=63)), (NULL, None, None, dict(ws=None)), (SIZE, None, None, dict(ws_bytes=100))):
        assert call(L, x, w, **change) == code


def test_sizes(L):
    size, plain = L.bitstack_f8_epilogue_workspace_bytes, L.bitstack_f8_workspace_bytes
    assert size(300, 4096, 1000, 2) == plain(300, 4096, 300, 1000, 1)
    assert size(300, 4096, 1024, 5) == plain(300, 4096, 300, 1024, 1)
    assert size(300, 4096, 1000, 5) >= 300 * 1000 * 4   # half of 1000 is no multiple of 128: the sums of all rows
    for bad in ((300, 4096, 1000, -1), (300, 4096, 1000, 6), (300, 4096, 999, 5), (-1, 4096, 1000, 0), (1, 0, 8, 0), (1, 8, 0, 0)):
        assert size(*bad) == 0
    with pytest.raises(B.BitStackError):
        B.f8_epilogue_workspace_bytes(300, 4096, 999, "silu_gated")
    with pytest.raises(B.BitStackError):
        B.f8_epilogue_workspace_bytes(300, 4096, 999, "tanh")
    need = L.bitstack_f8_epilogue_call_workspace_bytes
    for rows in (1, 5, 40, 300, 2048):
        for out in (1000, 1024):
            for act in range(6):
                for y in (0, 1, 2):
                    s = structs(dict(rows=rows, ld=4096), dict(out=out, inn=4096, ld=4096), dict(activation=act, ld_residual=out))
                    assert need(*(C.byref(v) for v in s), y) <= size(rows, 4096, out, act)
    assert need(None, None, None, 0) == 0


def test_without_a_gpu_tensor():
    q, s = torch.zeros((64, 128), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((1, 1), dtype=torch.uint8).view(torch.float8_e8m0fnu)
    x = torch.zeros((3, 128), dtype=torch.float16)
    for change in (dict(activation="relu"), dict(activation="tanh"), dict(bias=torch.zeros(63)), dict(bias=torch.zeros(128)[::2]), dict(bias=torch.zeros(64, dtype=torch.float64)),
                   dict(residual=x), dict(residual=torch.zeros((3, 64))), dict(activation="silu_gated", residual=torch.zeros((3, 64), dtype=torch.float16)),
                   dict(activation="silu_gated", q=q[:63])):
        with pytest.raises(ValueError):
            B.linear_f8(**(dict(x=x, q=q, scales=s) | change))


# wait states that the compiler leaves in one block between a product and an instruction of another kind that reads its result
BEHIND = {"v_mfma_f32_16x16x32_f16": 8, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_scale_f32_16x16x128_f8f6f4": 12}


def early_readers(assembly):
    """instructions that read a product's result too early, along every path: the compiler has been seen to leave one wait state where a branch lies between"""
    found = []
    for name, code, before in functions(assembly):
        for at, ins in enumerate(code):
            if ins.product or not ins.name.startswith(("v_", "ds_", "buffer_store", "global_store")):
                continue
            operands = [registers(o) for o in ins.text.partition(" ")[2].split(",")]
            reads = set().union(*(operands[1:] if ins.vector and not ins.name.startswith(("v_fmac", "v_dot", "v_mac")) else operands))
            for product, states in BEHIND.items():
                other = too_close(code, before, at, states, lambda o: o.name == product and o.writes & reads)
                if other:
                    found.append(f"{name}: {other.text}   ...   {ins.text}")
    return found


def test_early_readers_are_told_apart():
    product = "\tv_mfma_f32_16x16x32_f16 v[0:3], v[16:19], v[20:23], v[0:3]"
    assert early_readers(wrap(product, "\ts_nop 6", "\tv_fma_f32 v9, v3, v8, v9")) and not early_readers(wrap(product, "\ts_nop 7", "\tv_fma_f32 v9, v3, v8, v9"))
    assert early_readers(wrap(product, "\ts_cbranch_scc1 .LBB0_1", "\ts_nop 15", ".LBB0_1:", "\tds_write_b128 v9, v[0:3]"))
    assert not early_readers(wrap(product, "\tv_fma_f32 v9, v4, v8, v9"))


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no compiler")
@pytest.mark.parametrize("source", ["f8_epilogue.hip", "f8_gated.hip", "expert_layer.hip"])
def test_assembly(source, tmp_path):
    from paper_2410_23918_amd import build
    out = tmp_path / "kernels.asm"
    subprocess.run([HIPCC, *[f for f in build.FLAGS if f != "-shared"], "--cuda-device-only", "-S", str(CSRC / source), "-o", str(out)], check=True, capture_output=True)
    assembly = out.read_text()
    if source != "expert_layer.hip":
        assert len([name for name, code, _ in functions(assembly) if any(i.product for i in code)]) == 32   # as many as without an epilogue
        assert sum(i.in_asm and i.vector for _, code, _ in functions(assembly) for i in code) >= 10
    found = faults(assembly) + early_readers(assembly)
    assert not found, "\n".join(found[:10])
    assert "v_pk_fma_f32" not in assembly and "v_pk_mul_f32" not in assembly and "v_pk_add_f32" not in assembly
    assert "scratch_load" not in assembly   # no sum leaves the registers
