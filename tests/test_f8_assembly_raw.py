"""The kernels that bring rows to 8 bits on the way take them as they come, in no groups: their assembly reads neither a table of rows nor a list of tiles."""
import re
import shutil
import subprocess

import pytest

from test_asm_distances import CSRC, HIPCC


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no compiler")
def test_no_tables_of_rows(tmp_path):
    from paper_2410_23918_amd import build
    out = tmp_path / "kernels.asm"
    subprocess.run([HIPCC, *[f for f in build.FLAGS if f != "-shared"], "--cuda-device-only", "-S", str(CSRC / "f8_product.hip"), "-o", str(out)], check=True,
                   capture_output=True)
    tables = {}
    for name, body in re.findall(r"^(_ZN8bitstack11k_f8_slices\w+):(.*?)^\.Lfunc_end", out.read_text(), re.M | re.S):
        rows = re.search(r"k_f8_slicesILi\d+ELi(\d+)ELi\d+ELi\d+ELi(\d+)E", name)
        tables.setdefault(rows.group(2) == "3", set()).add((int(rows.group(1)), len(re.findall(r"\bglobal_load", body))))
    assert tables[True] == {(1, 1), (2, 2), (4, 4)}   # rows in 8 bits: a row's place for every fragment of them
    assert tables[False] == {(1, 0)}
