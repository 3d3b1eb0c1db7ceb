"""More of the host code of the 4-bit products and of the norm on a runtime of host memory (tests/ops4_host_edges.cpp; CPU
only)."""
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parents[1]
CSRC = ROOT / "paper_2609_13544_gb300" / "csrc"
CHECKS = ["no_k_no_scales", "norm_of_nothing", "mxfp4_has_no_scales", "workspace"]


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2609_13544_gb300 import buildlib
    cuda = Path(buildlib.nvcc()).resolve().parents[1] / "include"
    exe = tmp_path_factory.mktemp("ops4_host_edges") / "ops4_host_edges"
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{ROOT / 'include'}", f"-I{CSRC}", f"-isystem{cuda}",
                    str(ROOT / "tests" / "ops4_host_edges.cpp"), str(CSRC / "ops4_api.cpp"), "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("name", CHECKS)
def test_host(program, name):
    r = subprocess.run([str(program), name], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
