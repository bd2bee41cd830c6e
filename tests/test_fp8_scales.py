"""The addresses of the 8-bit products' scale loads, compiled for the host: no lane
reads past the row it is for, whatever the number of rows and of blocks of K, and
every scale is in its place when its step takes it."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_scale_loads(tmp_path):
    exe = str(tmp_path / "fp8_scales")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2609_33385_amd", "csrc"),
                    os.path.join(HERE, "native", "fp8_scales.cpp"), "-o", exe],
                   check=True, capture_output=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("ALL OK"), r.stdout[-500:]
