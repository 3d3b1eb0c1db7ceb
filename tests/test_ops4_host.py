"""The host code of the 4-bit products and of the norm against a runtime of host memory (tests/ops4_host.cpp), and what
needs no GPU of the binding (CPU only)."""
import ctypes
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parents[1]
CSRC = ROOT / "paper_2609_13544_gb300" / "csrc"


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2609_13544_gb300 import buildlib
    cuda = Path(buildlib.nvcc()).resolve().parents[1] / "include"
    exe = tmp_path_factory.mktemp("ops4_host") / "ops4_host"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", f"-I{ROOT / 'include'}", f"-I{CSRC}", f"-isystem{cuda}",
                    str(ROOT / "tests" / "ops4_host.cpp"), str(CSRC / "ops4_api.cpp"), "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("name", ["quantize_refusals", "product_refusals", "operands", "captures", "norm_refusals"])
def test_host(program, name):
    r = subprocess.run([str(program), name], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_layout_and_sizes():
    import paper_2609_13544_gb300 as peat
    from paper_2609_13544_gb300 import ops
    assert ctypes.sizeof(ops.OperandF4) == 56
    for rows, blocks, tiles in ((0, 5, 0), (1, 1, 1), (128, 4, 1), (129, 5, 4), (300, 9, 9)):
        assert peat.f4_scale_bytes(rows, blocks) == 512 * tiles


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "peat_ops.h"\nint main(void) { return sizeof(peat_operand_f4_t) == 56 && PEAT_NVFP4 == 1 && '
                   'peat_f4_scale_bytes(129, 5) == 2048 ? 0 : 1; }\n')
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{ROOT / 'include'}", str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_calls_without_a_handle_are_refused():
    import paper_2609_13544_gb300 as peat
    L = peat.load()
    assert L.peat_quantize_f4(None, None, 0, 0, 0, 0, 0, 0, None, 0, None, None, None, 0, None) == 1
    assert L.peat_matmul_f4(None, 0, None, 0, None, None, None, 0, None, None, None, 0, 0, 0, None, 0, 0, None) == 1
    assert L.peat_product_f4(None, 0, None, None, None, None, 0, 0, None) == 1
    assert L.peat_rmsnorm_backward(None, None, 0, None, 0, None, 0, None, 0, None, 0, 0, 0, None, 0, None, None) == 1


def test_binding_refuses_without_a_gpu():
    import torch
    import paper_2609_13544_gb300 as peat
    q, s = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for call in (lambda: peat.Float4("mxfp4", q, s), lambda: peat.Float4("fp4", q, s), lambda: peat.Linear4(None, q, "int4")):
        with pytest.raises(ValueError):
            call()
