"""How far tree attention's row references lie above the scores (csrc/tree_plan.h, plain C++)."""
import ctypes
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_08097_amd", "csrc")


def test_the_sums_of_all_tokens_stay_below_a_half(tmp_path):
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    (tmp_path / "s.cpp").write_text('#include "tree_plan.h"\nextern "C" int lift(int units) { return oasis::tree_lift(units); }\n')
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "s.cpp"), "-o", str(tmp_path / "s.so")],
                   check=True)
    lift = ctypes.CDLL(str(tmp_path / "s.so")).lift
    for units in (0, 1, 2, 3, 62, 63, 64, 65, 4094, 4095, 65536, 1 << 26):
        n = lift(units)
        assert 4 * (units + 2) * 2.0 ** (8 - n) <= 0.5 < 8 * (units + 2) * 2.0 ** (8 - n), units
