"""Thread maps and launch sizes of the token kernels, walked on the CPU by tests/token_launch.cpp from the header that
the kernels and their launchers share."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2209_13603_amd", "csrc")


@pytest.fixture(scope="module")
def walker(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not installed")
    exe = str(tmp_path_factory.mktemp("launch") / "token_launch")
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, os.path.join(HERE, "token_launch.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    return exe


@pytest.mark.parametrize("what", ["join", "grid"])
def test_maps(walker, what):
    r = subprocess.run([walker, what], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
