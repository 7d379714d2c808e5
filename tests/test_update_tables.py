"""The tables that norm, clipping and AdamW launch their kernels with, walked on the CPU (see c_abi/update_tables.cu)."""
import subprocess
from pathlib import Path

import pytest

from paper_2607_08782_b200 import build

ROOT = Path(__file__).resolve().parent.parent


def test_every_element_belongs_to_one_thread_and_failed_steps_are_not_counted(tmp_path):
    try:
        nvcc = build._nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    exe = tmp_path / "update_tables"
    cmd = [nvcc, "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "--expt-relaxed-constexpr", "-cudart", "none",
           f"-I{build.INCLUDE}", f"-I{build.CSRC}", "-o", str(exe), str(ROOT / "tests" / "c_abi" / "update_tables.cu")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
