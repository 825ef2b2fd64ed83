"""How far the row references of attention over the 4-bit cache lie above the scores (csrc/q4_plan.h, plain C++): as far as
every attended token needs, a block as often as a selection lists it; and what does not follow from that."""
import ctypes
import os
import subprocess

import paper_2608_08097_amd as P

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_08097_amd", "csrc")
SRC = """
#include "q4_plan.h"
extern "C" void plan(long long pairs, int G, int T, int units, int attended, long long* out) {
  const oasis::TreePlan p = oasis::q4_plan(pairs, G, T, units, attended), one = oasis::q4_plan(pairs, G, T, units);
  out[0] = oasis::tree_lift(p.units); out[1] = oasis::tree_lift(one.units);
  out[2] = p.tiles == one.tiles && p.groups == one.groups && p.nsplit == one.nsplit && p.bytes == one.bytes;
}
"""


def test_the_sums_of_all_attended_tokens_stay_below_a_half(tmp_path):
    (tmp_path / "p.cpp").write_text(SRC)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "p.cpp"), "-o",
                    str(tmp_path / "p.so")], check=True)
    plan = ctypes.CDLL(str(tmp_path / "p.so")).plan
    plan.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_longlong)]
    for units in (1, 2, 5, 64, 1000):
        for attended in (units, 2 * units, 16385, 32769):
            if attended < units:
                continue
            for G, T in ((4, 5), (8, 16)):
                out = (ctypes.c_longlong * 3)()
                plan(16, G, T, units, attended, out)
                # four lanes, each with eight probabilities of at most 2^(8 - lift) of 32 tokens, and 64 rows of the tree
                assert 4 * (2 * attended + 2) * 2.0 ** (8 - out[0]) <= 0.5, (units, attended)
                assert out[2] and out[1] <= out[0]


def test_repeated_blocks_take_no_more_workspace():
    for NB in (1, 4, 64, 500):
        d = P.dims(2, 8, 2, 128, 16, NB)
        assert len({P.oasis_tree_attn_q4_workspace_bytes(d, 5, k) for k in (max(1, NB - 1), NB, NB + 1, 4096, 65536)}) == 1
