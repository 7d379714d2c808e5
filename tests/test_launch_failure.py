"""A launch that fails must not spoil the next call."""
import subprocess
from pathlib import Path

import pytest

from paper_2607_08782_b200 import build

ROOT = Path(__file__).resolve().parent.parent


def test_a_failed_second_launch_of_the_gradient_leaves_the_counters_clean(tmp_path):
    try:
        nvcc = build._nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    exe = tmp_path / "gradient_launch_fails"
    cmd = [nvcc, "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "--expt-relaxed-constexpr", "-cudart", "none",
           f"-I{build.INCLUDE}", f"-I{build.CSRC}", "-o", str(exe), str(ROOT / "tests" / "c_abi" / "gradient_launch_fails.cpp"),
           str(build.CSRC / "director_ffn_grad.cu")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
