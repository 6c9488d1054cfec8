"""The gfx950 code built here holds no 64-bit shift whose amount lies in the last register of its waves.

Such a shift gives wrong bits now and then: its amount's register is read as if a second one followed
it. The build disassembles every code object and rejects one that holds such a shift; these tests check
that a kernel which does is rejected, and one with the amount a register lower is not (both are
only compiled, never run).
"""
import subprocess

import pytest

from paper_2608_00358_amd import _build

KERNEL = r"""
#include <hip/hip_runtime.h>
__global__ void shift(int* out) {{
    asm volatile("{op}" ::: "v2", "v3", "v6", "v7");
    out[threadIdx.x] = 0;
}}
"""


@pytest.mark.parametrize("op,refused", [
    ("v_lshlrev_b64 v[2:3], v7, v[2:3]", True), ("v_lshrrev_b64 v[2:3], v7, v[2:3]", True), ("v_ashrrev_i64 v[2:3], v7, v[2:3]", True),
    ("v_lshl_add_u64 v[2:3], v[2:3], v7, 0", True),
    ("v_lshlrev_b64 v[2:3], v6, v[2:3]", False), ("v_lshrrev_b64 v[2:3], 7, v[2:3]", False), ("v_lshrrev_b32 v2, v7, v3", False),
])
def test_check_rejects_shifts_by_the_last_register(tmp_path, op, refused):
    try:
        hipcc = _build._hipcc()
    except RuntimeError:
        pytest.skip("hipcc is not available")
    src, obj = tmp_path / "shift.hip", tmp_path / "shift.o"
    src.write_text(KERNEL.format(op=op))
    res = subprocess.run([hipcc, *_build.HIPCC_FLAGS, "-x", "hip", "-c", str(src), "-o", str(obj)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    if refused:
        with pytest.raises(RuntimeError, match="last register in the device code: .*shift"):
            _build.check_device_code(str(obj))
    else:
        _build.check_device_code(str(obj))
