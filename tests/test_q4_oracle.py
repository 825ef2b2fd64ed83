"""The 4-bit cache's oracle against values worked out by hand, and its host functions against the oracle (CPU only)."""
import math

import numpy as np
import pytest

import paper_2608_08097_amd as P
from oracle import q4 as Q


def _group(*first):
    return np.array([*first, *[0.0] * (32 - len(first))])


@pytest.mark.parametrize("top,power", [(7.0, 0), (6.0, 0), (4.0, 0), (3.75, 0), (7.03125, 1), (3.5, -1), (3.515625, 0),
                                       (1.0, -2), (0.875, -3), (2.0 ** -126, -126), (2.0 ** -133, -126), (1.5 * 2.0 ** 127, 125),
                                       (2.0 ** 128 * (1 - 2.0 ** -8), 125)])
def test_the_power_is_the_smallest_that_reaches_the_largest_value(top, power):
    codes, byte = Q.quantise(_group(-top, top / 16))
    assert byte == power + 127
    y = top / 2.0 ** power
    assert codes[0] == 8 + int(np.argmin(np.abs(Q.LEVELS - y))) if y < 6 else codes[0] == 15


def test_ties_take_the_even_code():
    edge = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    codes, byte = Q.quantise(_group(6.0, *edge, *-edge))
    assert byte == 127
    assert codes[1:15].tolist() == [0, 2, 2, 4, 4, 6, 6, 8, 10, 10, 12, 12, 14, 14]
    up, _ = Q.quantise(_group(6.0, *np.nextafter(edge, 9)))
    down, _ = Q.quantise(_group(6.0, *np.nextafter(edge, 0)))
    assert up[1:8].tolist() == [1, 2, 3, 4, 5, 6, 7] and down[1:8].tolist() == [0, 1, 2, 3, 4, 5, 6]


def test_zero_and_not_finite_groups():
    codes, byte = Q.quantise(_group())
    assert byte == 1 and not codes.any()
    for x in (np.nan, np.inf, -np.inf):
        codes, byte = Q.quantise(_group(1.0, x))
        assert byte == 255 and not codes.any()
        assert np.isnan(Q.values(codes, byte)).all()


def test_a_page_holds_what_its_layout_says():
    rng = np.random.default_rng(0)
    H, B = 3, 32
    x = rng.normal(size=(1, H, B, 128))
    page = Q.make_pages(x)[0]
    assert len(page) == P.oasis_q4_page_bytes(P.dims(1, 6, H, 128, B, 4)) == H * B * 68
    codes, powers = Q.quantise(x[0].reshape(H, B, 4, 32))
    codes = codes.reshape(H, B, 128)
    seen = page[H * B * 64:].reshape(H, B // 16, 4, 4, 4)
    for h, t, d in ((0, 0, 0), (1, 17, 33), (2, 31, 127), (2, 6, 64)):
        assert page[(h * B + t) * 64 + d // 2] >> (4 * (d % 2)) & 15 == codes[h, t, d]
        assert seen[h, t // 16, t % 4, d // 32, t % 16 // 4] == powers[h, t, d // 32]
    assert np.array_equal(Q.read_page(page, H, B), Q.values(codes.reshape(H, B, 4, 32), powers).reshape(H, B, 128))
    one = np.zeros_like(page)
    for h in range(H):
        for t in range(B):
            Q.write_token(one, H, B, h, t, x[0, h, t])
    assert np.array_equal(one, page)


def test_rotation_by_hand():
    x = np.zeros((1, 1, 8))
    x[0, 0, :4] = 3, 5, 7, 11
    quarter = np.array([0.25, 0.5])
    assert np.allclose(Q.rotate(x, [1], quarter)[0, 0], [-7, -5, 3, -11, 0, 0, 0, 0], atol=1e-14)
    assert np.allclose(Q.rotate(x, [1], quarter, True)[0, 0], [-5, 3, -7, -11, 0, 0, 0, 0], atol=1e-14)
    assert np.allclose(Q.rotate(x, [-1], quarter, False, 2.0)[0, 0], [14, -10, -6, -22, 0, 0, 0, 0], atol=1e-14)
    y = Q.rotate(x, [7], np.array([0.123, 0.0007]), True, 1.5)
    assert np.allclose(Q.rotate(y, [7], np.array([0.123, 0.0007]), True, 1 / 1.5, True), x, atol=1e-13)


def test_the_adjoint_is_the_inverse_rotation():
    rng = np.random.default_rng(1)
    turns, pos = rng.uniform(0, 0.2, 24), rng.integers(0, 10 ** 6, 5)
    for pairs in (False, True):
        x, g = rng.normal(size=(2, 5, 3, 128))
        left = np.sum(g * Q.rotate(x, pos, turns, pairs, 1.3))
        assert math.isclose(left, np.sum(Q.rotate(g, pos, turns, pairs, 1.3, True) * x), rel_tol=1e-10, abs_tol=1e-9)


SCALINGS = {"plain": P.ROTARY_PLAIN, "linear": P.ROTARY_LINEAR, "stretched": P.ROTARY_STRETCHED,
            "by_turns": P.ROTARY_BY_TURNS, "by_index": P.ROTARY_BY_INDEX}


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("dim,base", [(2, 10000.0), (32, 10000.0), (64, 500000.0), (100, 1e6), (128, 10000.0)])
def test_turns_match_the_oracle(scaling, dim, base):
    for factor, first, low, high in ((4.0, 4096.0, 1.0, 32.0), (8.0, 8192.0, 1.0, 4.0), (0.5, 2048.0, 2.0, 64.0)):
        got, amplitude = P.oasis_rotary_turns(dim, base, SCALINGS[scaling], factor, first, low, high)
        want, amp = Q.frequencies(dim, base, scaling, factor, first, low, high)
        assert np.allclose(got, want, rtol=1e-13, atol=0) and math.isclose(amplitude, amp, rel_tol=1e-15)


def test_turns_at_known_places():
    got, _ = P.oasis_rotary_turns(4, 10000.0)
    assert np.allclose(np.array(got) * 2 * math.pi, [1.0, 0.01], rtol=1e-14)
    # many turns: as it is; few: a factor slower; in the middle of 1 and 3 turns: in the middle
    got, _ = P.oasis_rotary_turns(2, 10000.0, P.ROTARY_BY_TURNS, 8.0, 2 * 2 * math.pi, 1.0, 3.0)
    assert math.isclose(got[0] * 2 * math.pi, 0.5 + 0.5 / 8, rel_tol=1e-13)
    _, amplitude = P.oasis_rotary_turns(64, 10000.0, P.ROTARY_BY_INDEX, 32.0, 4096.0)
    assert math.isclose(amplitude, 0.1 * math.log(32.0) + 1)


def test_turns_refusals():
    for args in ((0,), (3,), (130,), (64, 0.0), (64, math.inf), (64, math.nan), (64, 1e4, 5), (64, 1e4, -1),
                 (64, 1e4, P.ROTARY_LINEAR, 0.0), (64, 1e4, P.ROTARY_STRETCHED, math.inf),
                 (64, 1e4, P.ROTARY_BY_TURNS, 2.0, 0.0), (64, 1e4, P.ROTARY_BY_TURNS, 2.0, 4096.0, 4.0, 4.0),
                 (64, 1e4, P.ROTARY_BY_INDEX, 2.0, 4096.0, -1.0, 4.0), (64, 1.0, P.ROTARY_BY_INDEX, 2.0, 4096.0, 1.0, 4.0)):
        with pytest.raises(P.OasisError, match="OASIS_ERR_INVALID_ARG"):
            P.oasis_rotary_turns(*args)
