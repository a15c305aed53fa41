"""The distances that test_asm_distances.py keeps between statements written as assembly and matrix-core products, in the kernels of the 8-bit products."""
import shutil
import subprocess

import pytest

from test_asm_distances import CSRC, HIPCC, faults, functions


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no compiler")
def test_statements_keep_their_distance_from_products(tmp_path):
    from paper_2410_23918_amd import build
    out = tmp_path / "kernels.asm"
    subprocess.run([HIPCC, *[f for f in build.FLAGS if f != "-shared"], "--cuda-device-only", "-S", str(CSRC / "f8_product.hip"), "-o", str(out)], check=True,
                   capture_output=True)
    assembly = out.read_text()
    kernels = [name for name, code, _ in functions(assembly) if any(i.product for i in code)]
    # two of k_f8_tile256, three each of 128 x 128 and 128 x 64, two of 256 x 128, 22 of k_f8_slices
    assert len(kernels) == 32
    assert sum(i.in_asm and i.vector for _, code, _ in functions(assembly) for i in code) >= 10   # the weight's scales in every tile kernel
    found = faults(assembly)
    assert not found, "\n".join(found[:10])
    assert "v_pk_fma_f32" not in assembly and "v_pk_mul_f32" not in assembly and "v_pk_add_f32" not in assembly
    assert "scratch_load" not in assembly   # no sum leaves the registers
