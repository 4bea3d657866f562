"""The compiler's flags refuse inline assembly that changes a register the compiler keeps for itself."""
import os
import subprocess

import pytest

from paper_2607_08565_amd import build

SOURCE = "#include <hip/hip_runtime.h>\n__global__ void k(int x) { %s }\n"


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
@pytest.mark.parametrize("asm,compiles", [
    ('asm volatile("s_mov_b32 m0, %0" : : "s"(x) : "m0");', False),
    ('int y; asm volatile("s_mov_b32 %0, m0\\n\\ts_mov_b32 m0, %1\\n\\ts_mov_b32 m0, %0" : "=&s"(y) : "s"(x));', True)])
def test_reserved_registers(tmp_path, asm, compiles):
    src = tmp_path / "k.hip"
    src.write_text(SOURCE % asm)
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-c", str(src), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert (r.returncode == 0) == compiles, r.stderr
    if not compiles:
        assert "inline-asm" in r.stderr
