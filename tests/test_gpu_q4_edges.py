"""The 4-bit cache in the corners of its contract: wild queries where nothing is attended, selections that repeat blocks,
powers that no append writes; attention in every form of the kernel."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from oracle import q4 as Q
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import INF, NAN, _check
from tests.test_gpu_q4 import dev_u8
from workloads import random_bf16

pytestmark = pytest.mark.gpu

H = 2
# G, T, B, blocks of the table past the context: one and two row tiles a wave for itself, one and two of the form that
# shares a unit, each in one split and in several
FORMS = [(4, 3, 16, 0), (4, 3, 32, 3000), (4, 6, 16, 3000), (4, 6, 32, 0), (4, 13, 16, 0), (4, 13, 32, 3000), (8, 12, 16, 6000),
         (8, 16, 32, 6000)]


def _call(form, q, kp, vp, table, ctx, sel=None, cnt=None, scale=None, lse=True):
    G, T, B, _ = form
    R, NB, k = len(table), table.shape[1], 0 if sel is None else sel.shape[2]
    d = P.dims(R, G * H, H, 128, B, NB)
    note(f"4-bit corners G={G} T={T} B={B} NB={NB} k={k} ctx={list(ctx)[:4]}")
    ws = torch.full((P.oasis_tree_attn_q4_workspace_bytes(d, T, k),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, device="cuda") if lse else None
    P.oasis_tree_attn_q4(d, dev_bf16(q), T, dev_u8(kp), dev_u8(vp), dev_i32(table), dev_i32(ctx),
                         None if sel is None else dev_i32(sel), None if cnt is None else dev_i32(cnt), k, None, None, None, None,
                         scale, out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("selected", [False, True])
def test_wild_queries_that_attend_nothing_under_a_scale_of_0(form, selected):
    """Request 0 has pages, request 1 none for its whole context, request 2 only one that the selection of its head 1
    names (every block: the one of its last token). A row without an attended token is 0 and -infinity whatever its query
    holds; one with a token is NaN."""
    G, T, B, spare = form
    L, n = 5 * B - 3, 4
    rng = np.random.default_rng(T)
    kp, vp = (Q.make_pages(rng.normal(size=(6, H, B, 128))) for _ in range(2))
    table = np.full((3, 5 + spare), -1, np.int32)
    table[0, :5] = [3, 1, 0, 2, 4]
    table[1, :5] = [6, -7, 2 ** 31 - 1, -2 ** 31, -1]
    table[2, 2 if selected else 4] = 5
    sel = cnt = None
    if selected:
        sel = np.full((3, H, 3), -1, np.int32)
        sel[:, 0], sel[:, 1] = [1, 3, -1], [n, 0, 2]  # (n is the local block's id: no candidate)
        cnt = np.array([[2, 3], [2, 3], [3, 99]], np.int32)
    q = random_bf16(40 + T, (3, T, G * H, 128))
    q[:, 0, :, 3], q[:, T - 1, :, 120] = NAN, INF
    some = np.zeros((3, H), bool)
    some[0] = True
    some[2] = [False, True] if selected else True
    for lse in (True, False):
        out, got_lse = _call(form, q, kp, vp, table, [L] * 3, sel, cnt, 0.0, lse)
        out = out.cpu().view(3, T, H, G, 128)
        for r in range(3):
            for h in range(H):
                at = out[r, :, h]
                if not some[r, h]:
                    assert not at.view(torch.int16).any(), (r, h)
                else:
                    assert torch.isnan(at[[0, T - 1]]).all() and torch.isfinite(at[1:T - 1]).all(), (r, h)
                if lse:
                    x = got_lse.cpu().view(3, T, H, G)[r, :, h]
                    if not some[r, h]:
                        assert torch.all(x == -torch.inf), (r, h)
                    else:
                        assert torch.isnan(x[[0, T - 1]]).all() and torch.isfinite(x[1:T - 1]).all(), (r, h)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("last", [31, 32, 33, 63, 64, 70])
def test_wild_queries_whose_only_page_is_far_along(form, last):
    """Block `last` of the context, or entry `last` of the selection, is the only one with a page; with none at all the rows
    are 0."""
    G, T, B, spare = form
    L, NB = 80 * B, 80
    rng = np.random.default_rng(last)
    kp, vp = (Q.make_pages(rng.normal(size=(2, H, B, 128))) for _ in range(2))
    q = random_bf16(60 + T, (1, T, G * H, 128))
    q[:, :, :, 9] = NAN
    sel = np.broadcast_to(rng.permutation(NB - 1)[:75], (1, H, 75)).astype(np.int32).copy()
    for some in (True, False):
        for ids in (None, sel):
            table = np.full((1, NB + spare), -1, np.int32)
            if some:
                table[0, last if ids is None else sel[0, 0, last]] = 1
            out, lse = _call(form, q, kp, vp, table, [L], ids, None if ids is None else np.full((1, H), 75, np.int32), 0.0)
            if some:
                assert torch.isnan(out).all() and torch.isnan(lse).all()
            else:
                assert not out.view(torch.int16).any() and torch.all(lse == -torch.inf)


@pytest.mark.parametrize("tree", [False, True])
def test_wild_queries_among_more_rows_than_one_launch_takes_at_once(tree):
    R, T, G, B = 20, 64, 64, 16  # 163,840 rows
    rng = np.random.default_rng(3)
    d = P.dims(R, G * H, H, 128, B, 1)
    note(f"4-bit wild queries of many rows tree={tree}")
    q = torch.zeros((R, T, G * H, 128), dtype=torch.bfloat16, device="cuda")
    wild = rng.choice(R * T * G * H, 50, replace=False)
    wild[:4] = [0, R * T * G * H - 1, 1 << 17, (1 << 17) - 1]
    q.view(-1, 128)[torch.from_numpy(wild).cuda(), torch.from_numpy(rng.integers(0, 128, 50)).cuda()] = float("nan")
    pages = [dev_u8(Q.make_pages(rng.normal(size=(1, H, B, 128)))) for _ in range(2)]
    rows = torch.ones((R, T, H, 128), dtype=torch.bfloat16, device="cuda") if tree else None
    out, lse = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), torch.full(q.shape[:3], 7.0, device="cuda")
    ws = torch.zeros(P.oasis_tree_attn_q4_workspace_bytes(d, T, 0), dtype=torch.uint8, device="cuda")
    P.oasis_tree_attn_q4(d, q, T, *pages, dev_i32(np.zeros((R, 1))), dev_i32(np.full(R, 5)), None, None, 0, rows, rows, None, None,
                         0.0, out, lse, ws)
    want = torch.zeros(R * T * G * H, dtype=torch.bool)
    want[wild] = True
    assert torch.equal(torch.isnan(out).all(-1).view(-1).cpu(), want) and torch.equal(torch.isnan(lse).view(-1).cpu(), want)
    assert torch.isfinite(out.view(-1, 128)[(~want).cuda()]).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("times", [40, 2048])
def test_a_selection_that_repeats_its_blocks(form, times):
    """More selected ids than the table has blocks, each attended as often as it is listed: the largest finite values keep
    finite means, and others are those of the oracle."""
    G, T, B, _ = form
    NB, L = 4, 4 * B - 5
    rng = np.random.default_rng(T + times)
    table = rng.permutation(5)[:NB].reshape(1, NB).astype(np.int32)
    sel = np.tile(np.array([[[0, 2]], [[1, 0]]], np.int32).reshape(1, H, 2), (1, 1, times))
    cnt = np.full((1, H), 2 * times, np.int32)
    kp, vp = (Q.make_pages(rng.normal(size=(5, H, B, 128))) for _ in range(2))
    big = Q.make_pages(np.full((5, H, B, 128), 6.0 * 2.0 ** 125))
    for q, values in ((random_bf16(50 + T, (1, T, G * H, 128)), vp), (random_bf16(51 + T, (1, T, G * H, 128)), big),
                      (np.zeros((1, T, G * H, 128), np.uint16), big)):
        out, lse = _call(form, q, kp, values, table, [L], sel, cnt)
        args = (q, Q.read_pages(kp, H, B), Q.read_pages(values, H, B), table, [L], sel, cnt, None, None, None, [T], B)
        ref, ref_lse = Q.attend(*args)
        ref_abs, _ = Q.attend(*args, magnitude=True)
        _check(out, lse, ref, ref_abs, ref_lse, out)


def _with_powers(rng, n, B, powers):
    """Pages of any codes with powers among the given ones."""
    pages = rng.integers(0, 256, (n, Q.page_bytes(H, B))).astype(np.uint8)
    pages[:, H * B * 64:] = rng.choice(powers, (n, H * B * 4))
    return pages


@pytest.mark.parametrize("B", [16, 32])
def test_the_smallest_and_largest_powers_in_compressed_keys(B):
    rng = np.random.default_rng(B)
    for powers in ([0], [0, 1, 2], [252], [0, 252, 255], list(range(253))):
        pages = _with_powers(rng, 6, B, powers)
        table = np.array([[4, 0, 5, 1, 3, 2]], np.int32)
        out = [torch.zeros((1, H, 6, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        want = [np.zeros((1, H, 6, 128)) for _ in range(2)]
        note(f"powers {powers[:3]} in compressed keys B={B}")
        P.oasis_update_summaries_q4(P.dims(1, H, H, 128, B, 6), dev_u8(pages), dev_i32(table), None, dev_i32([6 * B]), 0, *out)
        Q.update_summaries(pages, table, None, [6 * B], B, *want)
        for got, w in zip(out, want):
            assert np.array_equal(O.bf16_to_f64(host_bits(got)), w), powers[:3]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power,size", [(0, 124), (1, 123), (2, 122), (252, -126), (251, -125)])
def test_the_smallest_and_largest_powers_in_attention(form, power, size):
    """Keys and queries at opposite ends of the range, whose products are logits of a few units; values of any power."""
    G, T, B, spare = form
    NB = 5
    rng = np.random.default_rng(power + T)
    q = rng.normal(size=(1, T, G * H, 128)) * 2.0 ** size
    q = (q.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    kp, vp = _with_powers(rng, NB, B, [power]), _with_powers(rng, NB, B, [0, 1, 100, 127, 129, 252])
    table = np.array([[*rng.permutation(NB), *[-1] * spare]], np.int32)
    L, scale = NB * B - 3, 0.1  # sums of scale |q k| below 16
    out, lse = _call(form, q, kp, vp, table, [L], scale=scale)
    args = (q, Q.read_pages(kp, H, B), Q.read_pages(vp, H, B), table, [L], None, None, None, None, None, [T], B, scale)
    ref, ref_lse = Q.attend(*args)
    ref_abs, _ = Q.attend(*args, magnitude=True)
    _check(out, lse, ref, ref_abs, ref_lse, out)
