"""Launch plans of attention over the 4-bit cache (csrc/q4_plan.h, plain C++), and the registers and LDS that the kernels
of the 4-bit cache take."""
import ctypes
import os
import re
import subprocess

import pytest

from tests.test_kernel_resources import LDS, kernels, waves_per_simd  # noqa: F401  (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_08097_amd", "csrc")

SRC = """
#include "q4_plan.h"
extern "C" void plan(long long pairs, int G, int T, int units, long long* out) {
  const oasis::TreePlan p = oasis::q4_plan(pairs, G, T, units);
  out[0] = p.rows; out[1] = p.tiles; out[2] = p.groups; out[3] = p.nsplit; out[4] = p.part_o_floats; out[5] = p.bytes;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("q4_plan")
    (at / "p.cpp").write_text(SRC)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(at / "p.cpp"), "-o",
                    str(at / "p.so")], check=True)
    f = ctypes.CDLL(str(at / "p.so")).plan
    f.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_longlong)]

    def call(*a):
        out = (ctypes.c_longlong * 6)()
        f(*a, out)
        return dict(zip(("rows", "tiles", "groups", "nsplit", "part_o", "bytes"), out))
    return call


def test_plans_cover_the_rows_and_fit_the_workspace(plan):
    for pairs in (0, 1, 2, 7, 16, 64, 100, 256, 500, 512, 1000, 4096, 65535):
        for G, T in ((1, 1), (1, 64), (3, 5), (4, 5), (8, 4), (8, 5), (5, 7), (8, 33), (16, 64), (64, 64), (4096, 1)):
            for units in (0, 1, 2, 5, 33, 65, 1000, 2048, 32768, 1 << 25):
                p = plan(pairs, G, T, units)
                at = (pairs, G, T, units, p)
                assert p["rows"] == G * T, at
                assert 1 <= p["tiles"] <= 8 and p["tiles"] * 16 * p["groups"] >= p["rows"], at
                assert p["tiles"] * 16 * (p["groups"] - 1) < p["rows"], at
                assert 1 <= p["nsplit"] <= 256 and (p["nsplit"] == 1 or 4 * (p["nsplit"] - 1) < units), at
                assert p["nsplit"] == 1 or pairs * p["groups"] * p["nsplit"] <= 1024, at
                n = pairs * p["nsplit"] * p["rows"] if p["nsplit"] > 1 else 0
                assert p["part_o"] == n * 128 and p["bytes"] == n * 130 * 4, at


def test_few_pairs_are_split_and_many_are_not(plan):
    assert plan(1, 8, 1, 2048)["nsplit"] >= 64
    assert plan(64, 4, 5, 2048)["nsplit"] == 8
    assert plan(64, 4, 5, 33)["nsplit"] == 4
    assert plan(512, 4, 7, 33)["nsplit"] == 1
    assert plan(64, 4, 5, 1)["nsplit"] == 1


def test_the_kernels_keep_their_values_in_registers(kernels):  # noqa: F811
    """No vector register spilled and no scratch; two workgroups share a CU of the forms that count on it."""
    seen = {}
    for n, k in kernels.items():
        if not (m := re.match(r"q4_\w+|rotate_kernel", n)):
            continue
        seen.setdefault(m[0], []).append(n)
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
        lds, waves = k[".group_segment_fixed_size"], waves_per_simd(k)
        if m[0] == "q4_attn_kernel":  # four waves, one a SIMD
            assert waves >= 2 and 2 * lds <= LDS, (n, k[".vgpr_count"], lds)
        elif m[0] == "q4_attn_rows_kernel":  # eight waves; two workgroups with one row tile a wave
            two = n.startswith("q4_attn_rows_kernel<1")
            assert waves >= (4 if two else 2) and (2 if two else 1) * lds <= LDS, (n, k[".vgpr_count"], lds)
    assert {n: len(v) for n, v in seen.items()} == {
        "q4_attn_kernel": 16, "q4_attn_rows_kernel": 12, "q4_append_kernel": 2, "q4_summaries_kernel": 2, "rotate_kernel": 2}, seen
