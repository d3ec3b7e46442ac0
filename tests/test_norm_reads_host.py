"""The loads of the norm kernels stay inside their arrays: enumerated on the host from the kernels' own index functions."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("nvcc") is None, reason="nvcc compiles the program (host code only)")
def test_vectors_of_rows_of_odd_width_stay_inside(tmp_path):
    exe = str(tmp_path / "norm_reads")
    subprocess.check_call(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-o", exe, os.path.join(HERE, "support", "norm_reads.cu")])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
