"""Builds libbitstack.so (C ABI + gfx950 HIP kernels) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbitstack.so")
SOURCES = ["host.cpp", "manager.cpp", "kernels.hip", "decode.hip", "panel.hip", "restore.hip", "batch.hip", "rows.hip", "token.hip", "dense.hip", "decompose.hip",
           "f8_host.cpp", "f8_rows.hip", "f8_product.hip", "f8_epilogue.hip", "f8_gated.hip", "experts.hip", "expert_layer.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-munsafe-fp-atomics",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        def run(cmd):
            res = subprocess.run(cmd, capture_output=True, text=True)
            if res.returncode != 0:
                raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
            if verbose:
                print(" ".join(cmd))

        def compiled(source):
            to = os.path.join(objects, source + ".o")
            run([hipcc, *[f for f in FLAGS if f != "-shared"], "-c", os.path.join(CSRC, source), "-o", to])
            return to

        run([hipcc, *FLAGS, *pool.map(compiled, SOURCES), "-o", LIB])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
