"""The operators' host code against a runtime of host memory in which calls fail (tests/ops_host.cpp; CPU only)."""
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parents[1]
CSRC = ROOT / "paper_2609_13544_gb300" / "csrc"


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2609_13544_gb300 import buildlib
    cuda = Path(buildlib.nvcc()).resolve().parents[1] / "include"
    exe = tmp_path_factory.mktemp("ops_host") / "ops_host"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", f"-I{ROOT / 'include'}", f"-I{CSRC}", f"-isystem{cuda}",
                    str(ROOT / "tests" / "ops_host.cpp"), str(CSRC / "ops_api.cpp"), "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("name", ["words_after_a_failed_launch", "words_after_a_failed_clear", "growing_sizes",
                                  "lists_allocate_once", "one_row_is_aligned", "host_memory"])
def test_host(program, name):
    r = subprocess.run([str(program), name], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
