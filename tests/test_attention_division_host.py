"""How the attention kernels divide their work, walked on the host without a GPU: the code that the kernels run, compiled for the host."""
import os
import shutil
import subprocess

import pytest

from paper_2505_22654_b200 import _build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if not _build.have_nvcc():
        pytest.skip("nvcc wanted")
    exe = tmp_path_factory.mktemp("division") / "walk"
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-I", _build.INCLUDE, "-I", _build.CSRC,
                    os.path.join(HERE, "division_walk.cu"), "-o", str(exe)], check=True, capture_output=True)
    return str(exe)


@pytest.mark.parametrize("first,last", [(1, 8), (9, 24), (25, 40), (41, 64)])
def test_every_step_is_met_once_and_every_partial_result_joined_once(walk, first, last):
    """Groups of 1 to 64 heads: whole tokens make tiles of 86 to 128 rows (or twice that), an odd number for groups of 5, 11, 13, 17, ..."""
    done = subprocess.run([walk, str(first), str(last)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
