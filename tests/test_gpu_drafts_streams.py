"""Tree attention over caches and working sets of more than 96 MiB, whose loads go past the caches: every such form of the
kernels, against the float64 oracle. Few of the tokens are attended."""
import re

import pytest

from tests.test_drafts_plan import plan  # noqa: F401  (a fixture)
from tests.test_gpu_drafts import _paged, _sparse
from tests.test_kernel_resources import kernels  # noqa: F401  (a fixture)

STREAM_BYTES = 96 << 20
# paged, G, T, B, blocks of the table or slots: one, two, three and four row tiles
CASES = [(True, 4, 3, 16, 3200), (True, 4, 3, 32, 1600), (True, 4, 7, 16, 3200), (True, 4, 7, 32, 1600),
         (True, 4, 11, 16, 3200), (True, 4, 11, 32, 1600), (True, 8, 8, 32, 1600),
         (False, 4, 3, 16, 1700), (False, 4, 3, 32, 850), (False, 4, 7, 16, 1700), (False, 4, 7, 32, 850),
         (False, 4, 11, 16, 1700), (False, 4, 11, 32, 850), (False, 8, 8, 16, 1700)]
R, HKV = 2, {True: 2, False: 4}


def _pairs_blocks(paged, blocks):
    return R * HKV[paged], blocks if paged else blocks + 1


@pytest.mark.gpu
@pytest.mark.parametrize("paged,G,T,B,blocks", CASES)
def test_loads_past_the_caches(paged, G, T, B, blocks):
    pairs, held = _pairs_blocks(paged, blocks)
    assert pairs * held * B * 512 >= STREAM_BYTES
    lens = [T, (T + 1) // 2]
    if paged:
        _paged(3000 + G * T + B, R, G * 2, 2, T, B, [777, 40], "random", lens, spare=blocks)
    else:  # contexts as long as the working set, which is hardly used
        _sparse(3100 + G * T + B, R, G * 4, 4, T, B, blocks, [blocks * B + 500, 37], "random", lens, free=0.96)


def test_the_cases_launch_every_streaming_form(plan, kernels):  # noqa: F811
    forms = (re.fullmatch(r"tree_attn(_rows)?_kernel<(\d), (\d+), (true|false), true>", n) for n in kernels)
    want = {(bool(m[1]), int(m[2]), int(m[3]), m[4] == "true") for m in forms if m}
    assert len(want) == 12
    got = set()
    for paged, G, T, B, blocks in CASES:
        pairs, held = _pairs_blocks(paged, blocks)
        p = plan(pairs, G, T, -(-held * B // 32), int(paged))
        assert p["tiles"] <= 4  # with more, two tiles a wave, no load goes past the caches
        got.add((p["tiles"] > 2, 1 if p["tiles"] > 2 else p["tiles"], B, paged))
    assert got == want
