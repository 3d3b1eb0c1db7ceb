"""The playback operators' header, library and binding agree (CPU only)."""
import ctypes
import re
from pathlib import Path

ROOT = Path(__file__).resolve().parents[1]


def declared():
    text = (ROOT / "include" / "peat_ops.h").read_text()
    return sorted(set(re.findall(r"^peat_status_t\s+(peat_\w+)\s*\(", text, re.M)))


def test_header_library_and_binding_agree():
    import paper_2609_13544_gb300 as peat
    from paper_2609_13544_gb300 import buildlib
    L = ctypes.CDLL(str(buildlib.build()))
    assert declared() == sorted(peat.OPS_EXPORTS)
    for name in declared():
        assert hasattr(L, name) and hasattr(peat, name) and hasattr(peat, name + "_raw")


def test_records_have_the_headers_layout():
    import paper_2609_13544_gb300 as peat
    from paper_2609_13544_gb300 import ops
    assert ctypes.sizeof(ops.GradEntry) == 32
    assert peat.GRADNORM_BYTES == 16


def test_header_compiles_as_c(tmp_path):
    import subprocess
    src = tmp_path / "t.c"
    src.write_text('#include "peat_ops.h"\nint main(void) { return sizeof(peat_grad_t) == 32 && '
                   'sizeof(peat_gradnorm_t) == 16 ? 0 : 1; }\n')
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{ROOT / 'include'}", str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_calls_without_a_handle_are_refused():
    import paper_2609_13544_gb300 as peat
    L = peat.load()
    assert L.peat_quantize_i8(None, None, 0, 0, 0, 0, 0, None, 0, None, None, 0, None) == 1
    assert L.peat_matmul_i8(None, None, 0, None, None, 0, None, None, 0, 0, 0, None, 0, 0, None) == 1
    assert L.peat_grad_clip(None, None, 0, 0, 1.0, 1.0, 0.0, 0, None, None, None) == 1
