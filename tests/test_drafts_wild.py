"""The launch of the pass over wild queries (csrc/tree_plan.h, plain C++) at the most rows that calls may have."""
import ctypes
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_08097_amd", "csrc")


def test_a_launch_holds_the_threads_of_any_call(tmp_path):
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    (tmp_path / "s.cpp").write_text('#include "tree_plan.h"\nextern "C" unsigned groups(long long rows) {'
                                    ' return oasis::tree_wild_groups(rows); }\nextern "C" int rows = oasis::kTreeWildRows;\n')
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "s.cpp"), "-o", str(tmp_path / "s.so")],
                   check=True)
    shim = ctypes.CDLL(str(tmp_path / "s.so"))
    shim.groups.argtypes, shim.groups.restype = [ctypes.c_longlong], ctypes.c_uint
    each = ctypes.c_int.in_dll(shim, "rows").value
    most = 65535 * 4096  # num_reqs * num_kv_heads and G * num_q_tokens
    for rows in (1, 7, 8, 9, 1000, 1 << 17, (1 << 17) + 1, 1 << 27, most):
        n = shim.groups(rows)
        assert 1 <= n <= -(-rows // each) and n * each * 32 < 1 << 32, rows
        # rows are counted in 31 bits, one turn past the last one too
        assert rows + n * each < 1 << 31, rows
