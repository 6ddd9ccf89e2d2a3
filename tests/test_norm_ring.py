"""The resident norm kernel's blocks and rings (norm_ring() in block_internal.h), without a GPU: tests/norm_ring.cpp, compiled
with the host compiler, checks that all blocks that a launch counts on fit an SM's shared memory together."""
import os
import shutil
import subprocess

import pytest

from paper_1908_11263_gb300 import build as qbuild

HERE = os.path.dirname(os.path.abspath(__file__))


def test_the_blocks_of_an_sm_fit_it_together(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(qbuild.nvcc())))
    exe = str(tmp_path / "norm_ring")
    subprocess.run([cxx, "-std=c++17", "-O1", f"-I{os.path.join(cuda, 'include')}", f"-I{qbuild.INCLUDE}",
                    os.path.join(HERE, "norm_ring.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.rstrip().endswith("fails=0"), out.stdout[-2000:]
