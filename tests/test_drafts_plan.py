"""The speculative step's launch plans (csrc/tree_plan.h, plain C++) over the shapes the entry points take, and the
registers and LDS that they count on."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from tests.test_kernel_resources import LDS, kernels, waves_per_simd  # noqa: F401  (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "tree_plan.h"
extern "C" void plan(long long pairs, int G, int T, int units, int ragged, long long* o) {
  const oasis::TreePlan p = oasis::tree_plan(pairs, G, T, units, ragged);
  o[0] = p.rows; o[1] = p.tiles; o[2] = p.groups; o[3] = p.nsplit; o[4] = p.part_o_floats; o[5] = p.bytes;
}
extern "C" long long wrong_quotients(unsigned d) {
  const oasis::FastDiv f = oasis::fast_div(d);
  long long bad = 0;
  const auto at = [&](unsigned long long n) { bad += n < 1ull << 31 && f((unsigned)n) != n / d; };
  for (unsigned long long n = 0; n < 70000; ++n) at(n);
  for (unsigned long long q = 1; q * d < 1ull << 31; q += 1 + q / 1000)  // around multiples
    for (int e = -1; e <= 1; ++e) at(q * d + e);
  for (unsigned long long e = 1; e < 1000; ++e) at((1ull << 31) - e);
  return bad;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2608_08097_amd", "csrc"), str(d / "shim.cpp"), "-o", str(d / "shim.so")],
                   check=True)
    shim = ctypes.CDLL(str(d / "shim.so"))
    f, shim.wrong_quotients.restype = shim.plan, ctypes.c_longlong

    def call(pairs, G, T, units, ragged):
        o = (ctypes.c_longlong * 6)()
        f(ctypes.c_longlong(pairs), G, T, units, ragged, o)
        return dict(zip(("rows", "tiles", "groups", "nsplit", "part_o", "bytes"), o))

    call.wrong_quotients = shim.wrong_quotients
    return call


def test_quotients_by_multiplication(plan):
    for d in [*range(1, 300), 511, 512, 513, 1000, 4095, 4096, 4097, 65535, 65536, 1000003, 2 ** 30, 2 ** 31 - 1]:
        assert plan.wrong_quotients(d) == 0, d


def test_plans_cover_the_rows_and_fit_the_workspace(plan):
    for pairs in (1, 2, 7, 16, 64, 100, 256, 500, 512, 1000, 4096, 1 << 19, 1 << 24):
        for G, T in ((1, 1), (1, 64), (3, 5), (4, 5), (8, 4), (8, 5), (5, 7), (8, 33), (16, 64), (64, 64), (4096, 1)):
            for units in (0, 1, 2, 5, 33, 65, 1000, 4096, 65536, 1 << 26):
                for ragged in (0, 1):
                    p = plan(pairs, G, T, units, ragged)
                    at = (pairs, G, T, units, ragged, p)
                    assert p["rows"] == G * T, at
                    # the last group has rows, and no tile is left without a group
                    assert 1 <= p["tiles"] <= 8 and p["tiles"] * 16 * p["groups"] >= p["rows"], at
                    assert p["tiles"] * 16 * (p["groups"] - 1) < p["rows"], at
                    assert 1 <= p["nsplit"] <= 256 and (p["nsplit"] == 1 or 4 * (p["nsplit"] - 1) < units), at
                    # a grid of workgroups that a launch can hold wherever it is split
                    assert p["nsplit"] == 1 or pairs * p["groups"] * p["nsplit"] <= 2048, at
                    n = pairs * p["nsplit"] * p["rows"] if p["nsplit"] > 1 else 0
                    assert p["part_o"] == n * 128 and p["bytes"] == n * 130 * 4, at


def test_few_pairs_are_split_and_many_are_not(plan):
    assert plan(1, 8, 1, 4096, 1)["nsplit"] >= 64
    assert plan(64, 4, 5, 4096, 1)["nsplit"] >= 4
    for ragged in (0, 1):
        assert plan(4096, 4, 5, 4096, ragged)["nsplit"] == 1
        assert plan(512, 4, 7, 65, ragged)["nsplit"] == 1
        assert plan(64, 4, 5, 1, ragged)["nsplit"] == 1


def test_the_kernels_keep_their_values_in_registers(kernels):  # noqa: F811
    """No vector register spilled and no scratch; two workgroups of the form for up to two row tiles share a CU, one of
    the form for more takes one alone, and the verification's sixteen waves fit one."""
    seen = {}
    for n, k in kernels.items():
        if not (m := re.match(r"(tree|verify|append)_\w+|append_kernel", n)):
            continue
        seen.setdefault(m[0], []).append(n)
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
        lds = k[".group_segment_fixed_size"]
        if m[0] == "tree_attn_kernel":  # four waves, one a SIMD
            assert waves_per_simd(k) >= 2 and 2 * lds <= LDS, (n, k[".vgpr_count"], lds)
        elif m[0] == "tree_attn_rows_kernel":  # eight waves
            assert waves_per_simd(k) >= 2 and LDS // 2 < lds <= LDS, (n, k[".vgpr_count"], lds)
        elif m[0].startswith("verify"):  # sixteen waves
            assert waves_per_simd(k) >= 4, (n, k[".vgpr_count"])
    assert {n: len(v) for n, v in seen.items()} == {
        "tree_attn_kernel": 16, "tree_attn_rows_kernel": 12, "tree_merge_kernel": 1, "verify_kernel": 2,
        "verify_blocks_kernel": 2, "verify_pick_kernel": 2, "append_kernel": 1}, seen
