"""Masters and moments at any address: AdamW's tables walked on the CPU (see c_abi/update_states.cu), with the alignment bit as it is and
with one that is wrong."""
import subprocess
from pathlib import Path

import pytest

from paper_2607_08782_b200 import build

ROOT = Path(__file__).resolve().parent.parent
PROGRAM = ROOT / "tests" / "c_abi" / "update_states.cu"


def _run(tmp_path, source):
    try:
        nvcc = build._nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    exe = tmp_path / "update_states"
    cmd = [nvcc, "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "--expt-relaxed-constexpr", "-cudart", "none",
           f"-I{build.INCLUDE}", f"-I{build.CSRC}", "-o", str(exe), str(source)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)


def test_whole_accesses_of_masters_and_moments_are_aligned(tmp_path):
    r = _run(tmp_path, PROGRAM)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.parametrize("forgotten", ["pad_of<float>(p[i].exp_avg) == 0 && ", " && pad_of<float>(p[i].exp_avg_sq) == 0",
                                       " && (!wb || pad_of<float>(p[i].master) == 0)"])
def test_the_walk_sees_an_array_that_the_alignment_bit_forgets(tmp_path, forgotten):
    """The mistake is planted in a copy that never runs on a GPU."""
    kernels = (build.CSRC / "director_update.cu").read_text()
    assert kernels.count(forgotten) == 1
    (tmp_path / "planted.cu").write_text(kernels.replace(forgotten, ""))
    include = '#include "../../paper_2607_08782_b200/csrc/director_update.cu"'
    walk = PROGRAM.read_text()
    assert walk.count(include) == 1
    (tmp_path / "walk.cu").write_text(walk.replace(include, f'#include "{tmp_path}/planted.cu"'))
    r = _run(tmp_path, tmp_path / "walk.cu")
    assert r.returncode != 0 and "a whole access is aligned" in r.stdout
