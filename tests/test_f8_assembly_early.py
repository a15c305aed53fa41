"""Readers of a product's result in the kernels of the bare 8-bit products, as test_f8_epilogue_host.py looks for them in the others."""
import shutil
import subprocess

import pytest

from test_asm_distances import CSRC, HIPCC
from test_f8_epilogue_host import early_readers


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no compiler")
def test_readers_keep_their_distance_from_products(tmp_path):
    from paper_2410_23918_amd import build
    out = tmp_path / "kernels.asm"
    subprocess.run([HIPCC, *[f for f in build.FLAGS if f != "-shared"], "--cuda-device-only", "-S", str(CSRC / "f8_product.hip"), "-o", str(out)], check=True, capture_output=True)
    assembly = out.read_text()
    assert assembly.count("v_mfma_scale_f32_16x16x128_f8f6f4") > 100 and assembly.count("v_mfma_f32_16x16x32_f16") > 100   # they are there
    found = early_readers(assembly)
    assert not found, "\n".join(found[:10])
