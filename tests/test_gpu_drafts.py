"""The speculative step on the GPU against the float64 oracle: tree attention over the paged cache and the working set,
draft verification, append, and the four together."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note, pool_v_from_htd
from workloads import random_bf16

pytestmark = pytest.mark.gpu

NAN = 0x7FC0
INF = 0x7F80
# Probabilities are rounded to bf16 for the second product and the output once: half a step is 2^-8 of a value, so
# the error is at most 2^-8 (|out| + sum p |v|). What float32 logits, exponentials and sums add is below 2^-13 of
# sum p |v|: logits of 128 products of magnitude |q k| / sqrt(128) are off by 129 * 2^-24 of their absolute sum
# (below 16 here), and a probability by as much relatively.
P_STEP, F32_SHARE = 2.0 ** -8, 2.0 ** -13
LSE_ATOL = 2e-4  # the same logit error, 129 * 2^-24 * 16 = 1.2e-4, and a few float32 steps of the result (below 16)


def _parents(rng, R, T, kind):
    if kind == "chain":
        return None
    t = np.arange(T)
    if kind == "beam":
        return np.broadcast_to((t + 1) // 2 - 1, (R, T)).astype(np.int32).copy()
    if kind == "roots":  # nothing but roots, some by a parent that is none
        return rng.choice([-5, -1, T, T + 7], size=(R, T)).astype(np.int32)
    return (t - rng.integers(1, 6, (R, T))).astype(np.int32)  # a negative one is a root


def _unused(rng, shape):
    """What places that must not count hold."""
    return np.where(rng.random(shape) < 0.5, NAN, INF).astype(np.uint16)


def _check(out, lse, ref, ref_abs, ref_lse, before):
    got = O.bf16_to_f64(host_bits(out))
    used = ~np.isnan(ref_lse)
    assert np.array_equal(host_bits(out)[~used], host_bits(before)[~used]), "rows past a tree's end were written"
    tol = P_STEP * (np.abs(ref) + ref_abs) + F32_SHARE * ref_abs + 1e-30
    err = np.abs(got - ref)[used]
    assert not np.isnan(err).any() and np.all(err <= tol[used]), (np.nanmax(err / tol[used]), np.isnan(err).sum())
    if lse is not None:
        e = np.abs(lse.double().cpu().numpy() - ref_lse)[used]
        assert np.all(e <= LSE_ATOL), e.max()


def _magnitude(bits):
    return bits & np.uint16(0x7FFF)


def _inputs(seed, R, Hq, Hkv, T, kind, lens):
    rng = np.random.default_rng(seed)
    q = random_bf16(seed + 1, (R, T, Hq, 128), scale=1.5)
    tk, tv = random_bf16(seed + 2, (R, T, Hkv, 128)), random_bf16(seed + 3, (R, T, Hkv, 128))
    parent = _parents(rng, R, T, kind)
    n = [T] * R if lens is None else lens
    for r in range(R):
        tk[r, n[r]:], tv[r, n[r]:] = NAN, INF
        q[r, n[r]:] = NAN
    return rng, q, tk, tv, parent, n


def _paged(seed, R, Hq, Hkv, T, B, ctx, kind="random", lens=None, bad_pages=False, lse=True, scale=None, pinned=False,
           spare=0):
    rng, q, tk, tv, parent, n = _inputs(seed, R, Hq, Hkv, T, kind, lens)
    ctx = np.array(ctx, np.int32)
    NB = max(1, (max(ctx.max(), 1) + B - 1) // B + int(rng.integers(0, 3)))
    NP = R * NB + 2
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    kp, vp = random_bf16(seed + 4, (NP, Hkv, B, 128)), random_bf16(seed + 5, (NP, Hkv, B, 128))
    held = np.zeros((NP, B), bool)
    for r in range(R):
        for t in range(min(max(int(ctx[r]), 0), NB * B)):
            held[table[r, t // B], t % B] = True
    for x in (kp, vp):
        x.transpose(0, 2, 1, 3)[~held] = _unused(rng, (int((~held).sum()), Hkv, 128))
    if bad_pages:
        table[rng.random((R, NB)) < 0.2] = rng.choice([-1, -2 ** 31, NP, 2 ** 31 - 1])
    if spare:  # a table far longer than the contexts
        table = np.concatenate([table, rng.choice([-1, NP, 2 ** 31 - 1], (R, spare)).astype(np.int32)], 1)
        NB += spare
    d = P.dims(R, Hq, Hkv, 128, B, NB)
    note(f"tree attention paged seed={seed} R={R} Hq={Hq} Hkv={Hkv} T={T} B={B} ctx={ctx.tolist()[:6]} {kind} {n[:6]}")
    before = dev_bf16(random_bf16(seed + 6, (R, T, Hq, 128)))
    out, lse = before.clone(), (torch.full((R, T, Hq), 7.0, device="cuda") if lse else None)
    ws = torch.full((P.oasis_tree_attn_workspace_bytes(d, T),), 255, dtype=torch.uint8, device="cuda")
    pages = [dev_bf16(x) for x in (kp, vp)]
    if pinned:
        pages = [torch.empty(x.shape, dtype=x.dtype, pin_memory=True).copy_(x) for x in pages]
    args = (d, dev_bf16(q), T, *pages, dev_i32(table), dev_i32(ctx), dev_bf16(tk), dev_bf16(tv),
            None if parent is None else dev_i32(parent), None if lens is None else dev_i32(np.array(lens)), scale)
    P.oasis_tree_attn(*args, out, lse, ws)
    torch.cuda.synchronize()
    ref, ref_lse = O.tree_attend(q, kp, vp, table, ctx, tk, tv, parent, n, B, scale)
    ref_abs, _ = O.tree_attend(q, kp, _magnitude(vp), table, ctx, tk, _magnitude(tv), parent, n, B, scale)
    _check(out, lse, ref, ref_abs, ref_lse, before)
    if lse is not None:
        assert torch.all(lse.cpu()[torch.from_numpy(np.isnan(ref_lse))] == 7.0)


@pytest.mark.parametrize("T", [1, 2, 5, 16, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("kind", ["chain", "random"])
def test_paged_tree_sizes(T, kind):
    _paged(100 + T, 2, 8, 2, T, 16, [77, 40], kind, [T, (T + 1) // 2])


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("ctx", [[0], [1], [15, 16, 17], [31, 32, 33], [0, 1000, 64], [-4, 500, 333], [4097]])
def test_paged_lengths(B, ctx):
    _paged(200 + B + len(ctx), len(ctx), 8, 2, 3, B, ctx)


@pytest.mark.parametrize("G", [1, 3, 4, 5, 8, 16])
def test_paged_head_groups(G):
    """Rows from one tile to several groups of tiles."""
    _paged(300 + G, 1, G * 2, 2, 20, 16, [700], "beam")


def test_paged_many_splits_and_roots():
    _paged(400, 1, 4, 1, 7, 16, [9000])
    _paged(401, 3, 4, 1, 9, 32, [9000, 12, 2500], "roots", [9, 4, 0])


def test_paged_wide_rows():
    _paged(402, 1, 32, 2, 64, 32, [1500], "beam", [61])


def test_paged_pages_outside_the_tier():
    _paged(403, 3, 8, 2, 4, 16, [300, 555, 90], bad_pages=True)
    _paged(404, 2, 8, 2, 4, 32, [300, 555], bad_pages=True)


def test_paged_many_pairs():
    _paged(405, 80, 32, 8, 2, 16, list(np.random.default_rng(1).integers(0, 90, 80)))


@pytest.mark.parametrize("R,Hkv,G,T,hi", [(64, 16, 2, 3, 60), (63, 16, 5, 5, 40), (40, 8, 4, 10, 130), (12, 8, 16, 20, 300)])
def test_paged_more_workgroups_than_the_chip_holds(R, Hkv, G, T, hi):
    """The longest requests are taken first: lengths with ties, empty and negative ones, in no order; one, two, three
    and more row tiles and several groups of them."""
    rng = np.random.default_rng(R)
    ctx = rng.integers(0, hi, R)
    ctx[::5], ctx[1::7], ctx[2], ctx[3] = hi // 2, 0, -2 ** 31, -1
    _paged(1200 + R, R, Hkv * G, Hkv, T, 16, list(ctx), lens=list(rng.integers(0, T + 1, R)))


def test_paged_largest_rows_and_most_pairs():
    _paged(1300, 1, 64, 1, 64, 16, [100], "random", [63])
    _paged(1301, 2000, 8, 8, 1, 16, list(np.random.default_rng(3).integers(0, 18, 2000)))


LONG = 6000  # blocks: so many that more than two row tiles take the form that shares its loads


@pytest.mark.parametrize("G,T", [(4, 9), (3, 13), (4, 16), (5, 13), (8, 16), (4, 33), (16, 16), (9, 63), (64, 5)])
def test_paged_shared_loads_rows(G, T):
    """Three, four and more row tiles, in one group and in several, with rows left over."""
    _paged(1400 + G * T, 2, G * 2, 2, T, 16, [777, 40], "random", [T, (T + 1) // 2], spare=LONG)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("ctx", [[0], [1], [15, 16, 17], [31, 32, 33], [0, 1000, 64], [-4, 500, 333], [4097]])
def test_paged_shared_loads_lengths(B, ctx):
    _paged(1500 + B + len(ctx), len(ctx), 24, 2, 5, B, ctx, spare=LONG)
    _paged(1600 + B + len(ctx), len(ctx), 16, 2, 20, B, ctx, "beam", spare=LONG)


def test_paged_shared_loads_masks():
    _paged(1700, 3, 16, 2, 9, 16, [300, 555, 90], bad_pages=True, spare=LONG)
    _paged(1701, 2, 32, 2, 17, 32, [300, 555], "roots", [17, 0], bad_pages=True, spare=LONG)
    _paged(1702, 1, 16, 2, 20, 32, [300], scale=-0.07, spare=LONG)
    _paged(1703, 1, 16, 2, 6, 32, [45], scale=0.0, lse=False, spare=LONG)
    _paged(1704, 2, 16, 2, 7, 16, [300, 20], pinned=True, spare=LONG)


@pytest.mark.parametrize("G,T", [(4, 10), (8, 17)])
@pytest.mark.parametrize("B,ks", [(16, 2600), (32, 1300)])
def test_sparse_shared_loads(G, T, B, ks):
    _sparse(1800 + G * T, 2, G * 2, 2, T, B, ks, [1000, 37], lens=[T, (T + 1) // 2], free=0.9)


def test_paged_scale_and_no_lse():
    _paged(406, 2, 8, 2, 4, 16, [300, 20], lse=False, scale=0.05)
    _paged(407, 1, 8, 2, 4, 16, [300], scale=0.0)
    _paged(409, 1, 8, 2, 4, 16, [300], scale=-0.07)
    _paged(410, 1, 16, 2, 20, 32, [300], scale=-0.07)
    _paged(411, 1, 16, 2, 20, 32, [45], scale=0.0)


def test_paged_pinned_tier():
    _paged(408, 2, 8, 2, 4, 16, [300, 20], pinned=True)


def _sparse(seed, R, Hq, Hkv, T, B, ks, ctx, kind="random", lens=None, free=0.3):
    rng, q, tk, tv, parent, n = _inputs(seed, R, Hq, Hkv, T, kind, lens)
    ctx = np.array(ctx, np.int32)
    pk, pv = random_bf16(seed + 4, (R, ks + 1, Hkv, B, 128)), random_bf16(seed + 5, (R, ks + 1, Hkv, B, 128))
    smap = np.where(rng.random((R, Hkv, ks)) < free, -1, rng.integers(0, 10 ** 6, (R, Hkv, ks))).astype(np.int32)
    NB = max(1, (max(int(ctx.max()), 1) + B - 1) // B)
    for r in range(R):
        local = O.block_counts(min(int(ctx[r]), NB * B), B)[2]
        for x in (pk, pv):
            x[r, ks, :, local:] = _unused(rng, (Hkv, B - local, 128))
            for h in range(Hkv):
                x[r, :ks, h][smap[r, h] < 0] = _unused(rng, (int((smap[r, h] < 0).sum()), B, 128))
    d = P.dims(R, Hq, Hkv, 128, B, NB)
    note(f"tree attention sparse seed={seed} R={R} Hq={Hq} Hkv={Hkv} T={T} B={B} ks={ks} ctx={ctx.tolist()[:6]} {kind}")
    before = dev_bf16(random_bf16(seed + 6, (R, T, Hq, 128)))
    out, lse = before.clone(), torch.full((R, T, Hq), 7.0, device="cuda")
    ws = torch.full((P.oasis_sparse_tree_attn_workspace_bytes(d, T, ks),), 255, dtype=torch.uint8, device="cuda")
    P.oasis_sparse_tree_attn(d, dev_bf16(q), T, dev_bf16(pk), dev_bf16(pool_v_from_htd(pv)),
                             dev_i32(smap) if ks else None, ks, dev_i32(ctx), dev_bf16(tk), dev_bf16(tv),
                             None if parent is None else dev_i32(parent), None if lens is None else dev_i32(np.array(lens)),
                             None, out, lse, ws)
    torch.cuda.synchronize()
    ref, ref_lse = O.sparse_tree_attend(q, pk, pv, smap, ctx, tk, tv, parent, n, B)
    ref_abs, _ = O.sparse_tree_attend(q, pk, _magnitude(pv), smap, ctx, tk, _magnitude(tv), parent, n, B)
    _check(out, lse, ref, ref_abs, ref_lse, before)


@pytest.mark.parametrize("T", [1, 5, 31, 33, 64])
@pytest.mark.parametrize("B", [16, 32])
def test_sparse_tree_sizes(T, B):
    _sparse(500 + T, 2, 8, 2, T, B, 9, [1000, 37], lens=[T, (T + 1) // 2])


@pytest.mark.parametrize("ks", [0, 1, 2, 15, 64, 129])
def test_sparse_slots(ks):
    _sparse(600 + ks, 3, 12, 2, 4, 16, ks, [4000, 16, 0], free=0.5)
    _sparse(700 + ks, 1, 8, 1, 40, 32, ks, [4001], "beam", free=0.9)


def test_sparse_all_free_and_none_free():
    _sparse(800, 2, 8, 2, 6, 16, 128, [0, 0], "chain", free=1.0)  # nothing cached: the tree alone
    _sparse(801, 2, 8, 2, 6, 16, 128, [9000, 2064], "chain", free=0.0)
    _sparse(802, 1, 64, 4, 32, 32, 128, [9000], "beam", free=0.0)


@pytest.mark.parametrize("paged,spare", [(True, 0), (False, 0), (True, LONG), (False, 2000)])
def test_rows_off_the_path_have_no_influence(paged, spare):
    """Infinities and NaN in the keys and values of some rows: rows that attend them take them up, the others are what
    they are with finite values there."""
    R, Hq, Hkv, T, B, L = 1, 8, 2, 40, 16, 100
    rng, q, tk, tv, parent, _ = _inputs(900, R, Hq, Hkv, T, "random", None)
    wild = [7, 20, 33]
    paths = O.tree_paths(parent, [T], T)[0]
    hit = np.array([any(w in p for w in wild) for p in paths])
    assert hit.any() and not hit.all()
    tk2, tv2 = tk.copy(), tv.copy()
    tk2[0, 7, :, 5], tv2[0, 7, :, 3], tv2[0, 20, 1, 100], tv2[0, 33] = NAN, INF, NAN, INF | 0x8000
    NB = (L + B - 1) // B
    kp, vp = random_bf16(901, (NB, Hkv, B, 128)), random_bf16(902, (NB, Hkv, B, 128))
    d = P.dims(R, Hq, Hkv, 128, B, NB + spare)
    junk = np.full((spare, Hkv, B, 128), NAN, np.uint16)  # free slots
    outs = []
    for k, v in ((tk, tv), (tk2, tv2)):
        out, lse = torch.zeros((R, T, Hq, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((R, T, Hq), device="cuda")
        note(f"wild rows paged={paged}")
        tree = (dev_bf16(k), dev_bf16(v), dev_i32(parent), None, None, out, lse)
        if paged:
            ws = torch.zeros(P.oasis_tree_attn_workspace_bytes(d, T), dtype=torch.uint8, device="cuda")
            P.oasis_tree_attn(d, dev_bf16(q), T, dev_bf16(kp), dev_bf16(vp), dev_i32([[*range(NB), *[-1] * spare]]),
                              dev_i32([L]), *tree, ws)
        else:
            ks = NB - 1 + spare
            pools = [np.concatenate([x[:-1], junk, x[-1:]]) for x in (kp, vp)]
            ws = torch.zeros(P.oasis_sparse_tree_attn_workspace_bytes(d, T, ks), dtype=torch.uint8, device="cuda")
            smap = np.broadcast_to(np.array([*range(NB - 1), *[-1] * spare]), (1, Hkv, ks))
            P.oasis_sparse_tree_attn(d, dev_bf16(q), T, dev_bf16(pools[0]), dev_bf16(pool_v_from_htd(pools[1])),
                                     dev_i32(smap), ks, dev_i32([L]), *tree, ws)
        outs.append((out.float().cpu()[0], lse.cpu()[0]))
    (o0, l0), (o1, l1) = outs
    assert torch.equal(o0[~hit], o1[~hit]) and torch.equal(l0[~hit], l1[~hit])
    for t in np.nonzero(hit)[0]:
        p = paths[t]
        for h in range(Hkv):
            o = o1[t, h * 4:(h + 1) * 4]
            if 7 in p:
                assert torch.isnan(o).all()  # a NaN score
                continue
            want = np.full(128, "", object)
            if 20 in p and h == 1:
                want[100] = "nan"
            if 33 in p:
                want[:] = np.where(want == "nan", "nan", "-inf")
            for j in range(128):
                x = o[:, j]
                assert {"": torch.isfinite(x), "nan": torch.isnan(x), "-inf": x == -torch.inf}[want[j]].all(), (t, h, j)


def test_offsets_past_32_bits():
    """Pages and pools of more than 2^32 elements; only the last pages are used."""
    Hkv, B, T, L = 8, 32, 3, 90
    NP = (1 << 32) // (Hkv * B * 128) + 40
    kp, vp = (torch.empty((NP, Hkv, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hk, hv = random_bf16(1001, (3, Hkv, B, 128)), random_bf16(1002, (3, Hkv, B, 128))
    kp[-3:], vp[-3:] = dev_bf16(hk), dev_bf16(hv)
    rng, q, tk, tv, parent, n = _inputs(1003, 1, 16, Hkv, T, "random", None)
    table = np.array([[NP - 1, NP - 3, NP - 2, -1]], np.int32)
    d = P.dims(1, 16, Hkv, 128, B, 4)
    out = torch.zeros((1, T, 16, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(P.oasis_tree_attn_workspace_bytes(d, T), dtype=torch.uint8, device="cuda")
    note("offsets past 32 bits")
    P.oasis_tree_attn(d, dev_bf16(q), T, kp, vp, dev_i32(table), dev_i32([L]), dev_bf16(tk), dev_bf16(tv), dev_i32(parent),
                      None, None, out, None, ws)
    small = np.array([[2, 0, 1, -1]], np.int32)
    ref, ref_lse = O.tree_attend(q, hk, hv, small, [L], tk, tv, parent, n, B)
    ref_abs, _ = O.tree_attend(q, hk, _magnitude(hv), small, [L], tk, _magnitude(tv), parent, n, B)
    _check(out, None, ref, ref_abs, ref_lse, out)
    P.oasis_append_tokens(d, dev_bf16(tk), dev_bf16(tv), T, None, None, kp, vp, dev_i32(table), dev_i32([L]), None)
    O.append_tokens(tk, tv, None, None, hk, hv, small, [L], B)
    assert np.array_equal(host_bits(kp[-3:]), hk) and np.array_equal(host_bits(vp[-3:]), hv)


@pytest.mark.parametrize("G,T", [(4, 3), (20, 2), (20, 4)])
def test_paged_long_contexts_in_one_split(G, T):
    """So many pairs that they are hardly split, or not at all, two of them with thousands of units: lists of units in
    several pieces."""
    R, B, NB = 1024, 32, 2205
    ctx = np.zeros(R, np.int32)
    ctx[[3, 700]] = 1029 * 32 + 5, NB * B - 40
    rng, q, tk, tv, parent, n = _inputs(1100 + G, R, G, 1, T, "random", None)
    NP = 2300
    kp, vp = random_bf16(1101, (NP, 1, B, 128)), random_bf16(1102, (NP, 1, B, 128))
    table = np.broadcast_to(rng.permutation(NP)[:NB], (R, NB)).astype(np.int32)
    table[:, 1025:1031] = -1  # a hole around the end of a piece
    d = P.dims(R, G, 1, 128, B, NB)
    ws = torch.zeros(P.oasis_tree_attn_workspace_bytes(d, T), dtype=torch.uint8, device="cuda")
    note(f"long contexts in one split G={G} T={T}")
    out = torch.zeros((R, T, G, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((R, T, G), device="cuda")
    P.oasis_tree_attn(d, dev_bf16(q), T, dev_bf16(kp), dev_bf16(vp), dev_i32(table), dev_i32(ctx), dev_bf16(tk),
                      dev_bf16(tv), dev_i32(parent), None, None, out, lse, ws)
    some = [0, 3, 512, 700, 1023]
    ref, ref_lse = O.tree_attend(q[some], kp, vp, table[some], ctx[some], tk[some], tv[some], parent[some], [T] * 5, B)
    ref_abs, _ = O.tree_attend(q[some], kp, _magnitude(vp), table[some], ctx[some], tk[some], _magnitude(tv[some]),
                               parent[some], [T] * 5, B)
    _check(out[some], lse[some], ref, ref_abs, ref_lse, out[some])


@pytest.mark.parametrize("T", [2, 4])
def test_sparse_working_set_of_many_slots_in_one_split(T):
    """As above over the working set, in blocks of 16: two slots a unit, many of them free."""
    R, G, B, ks = 1024, 20, 16, 2301
    rng, q, tk, tv, parent, n = _inputs(1110, R, G, 1, T, "random", None)
    ctx = np.zeros(R, np.int32)
    ctx[700] = 5000 * B + 3
    pk, pv = (random_bf16(s, (1, ks + 1, 1, B, 128)) for s in (1111, 1112))
    smap = np.full((R, 1, ks), -1, np.int32)
    smap[700, 0] = np.where(rng.random(ks) < 0.05, -1, 1)
    d = P.dims(R, G, 1, 128, B, 5001)
    ws = torch.zeros(P.oasis_sparse_tree_attn_workspace_bytes(d, T, ks), dtype=torch.uint8, device="cuda")
    dk = torch.empty((R, ks + 1, 1, B, 128), dtype=torch.bfloat16, device="cuda")
    dv = torch.empty((R, ks + 1, 1, 128, B), dtype=torch.bfloat16, device="cuda")
    dk[700], dv[700] = dev_bf16(pk)[0], dev_bf16(pool_v_from_htd(pv))[0]
    note("a working set of many slots in one split")
    out = torch.zeros((R, T, G, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((R, T, G), device="cuda")
    P.oasis_sparse_tree_attn(d, dev_bf16(q), T, dk, dv, dev_i32(smap), ks, dev_i32(ctx), dev_bf16(tk), dev_bf16(tv),
                             dev_i32(parent), None, None, out, lse, ws)
    for one in ([700], [5]):  # the other one: nothing cached
        at = (smap[one], ctx[one])
        rows = (parent[one], [T], B)
        ref, ref_lse = O.sparse_tree_attend(q[one], pk, pv, *at, tk[one], tv[one], *rows)
        ref_abs, _ = O.sparse_tree_attend(q[one], pk, _magnitude(pv), *at, tk[one], _magnitude(tv[one]), *rows)
        _check(out[one], lse[one], ref, ref_abs, ref_lse, out[one])


# -- verification --------------------------------------------------------------------


def _probs(rng, shape, peak):
    x = rng.standard_normal(shape) * peak
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


def _verify_case(seed, R, T, V, kind, certain, peak=3.0, lens=None, pad=0):
    rng = np.random.default_rng(seed)
    parent = _parents(rng, R, T, kind)
    if parent is not None and kind == "random":
        parent = np.maximum(parent, 0)
        parent[:, 0] = -1
    target = _probs(rng, (R, T, V), peak)
    draft = None if certain else _probs(rng, (R, T, V), 0.3) * np.float32(0.5) + target * np.float32(0.5)
    tokens = rng.integers(0, V, (R, T)).astype(np.int32)
    likely = np.argsort(-target, -1)[..., :8]
    for r in range(R):
        for t in range(1, T):
            at = t - 1 if parent is None else min(max(0, parent[r, t]), t - 1)
            if rng.random() < 0.8:
                tokens[r, t] = likely[r, at, rng.integers(0, min(8, V))]
            elif rng.random() < 0.1:
                tokens[r, t] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31])
    return dict(target=target, draft=draft, tokens=tokens, parent=parent, lens=lens, pad=pad,
                ua=rng.random((R, T), dtype=np.float32), us=rng.random(R, dtype=np.float32))


def _run_verify(c):
    R, T, V = c["target"].shape

    def dev(x):
        if x is None:
            return None
        wide = torch.full((R, T, V + c["pad"]), float("nan"), device="cuda")
        wide[..., :V] = torch.from_numpy(np.ascontiguousarray(x)).cuda()
        return wide[..., :V]

    ints = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((R, T), (R,), (R, T))]
    ws = torch.full((P.oasis_verify_workspace_bytes(R, T, V),), 255, dtype=torch.uint8, device="cuda")
    f32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()  # noqa: E731
    P.oasis_verify_drafts(dev(c["target"]), dev(c["draft"]), dev_i32(c["tokens"]),
                          None if c["parent"] is None else dev_i32(c["parent"]),
                          None if c["lens"] is None else dev_i32(np.array(c["lens"])), f32(c["ua"]), f32(c["us"]), *ints, ws)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in ints]


def _assert_verified(c):
    R, T, V = c["target"].shape
    note(f"verify R={R} T={T} V={V} draft={c['draft'] is not None} parent={c['parent'] is not None}")
    got = _run_verify(c)
    ref = O.verify_drafts(c["target"], c["draft"], c["tokens"], c["parent"], [T] * R if c["lens"] is None else c["lens"],
                          c["ua"], c["us"])
    for name, x, y in zip(("path", "path_len", "out_tokens"), got, ref):
        assert np.array_equal(x, y), (name, np.argwhere(x != y)[:4].tolist())
    return ref


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("V", [1, 2, 15, 16, 17, 255, 4095, 4096, 4097, 9001, 50261])
def test_verification_vocabularies(V, certain):
    _assert_verified(_verify_case(1100 + V, 3, 6, V, "random", certain, pad=V % 3))


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("kind", ["chain", "beam", "random", "roots"])
@pytest.mark.parametrize("T", [1, 2, 9, 33, 64])
def test_verification_trees(T, kind, certain):
    lens = [T, 0, T + 9, -3, (T + 1) // 2, 1, T, T]
    _assert_verified(_verify_case(1200 + T, 8, T, 700, kind, certain, lens=lens))


@pytest.mark.parametrize("certain", [False, True])
def test_verification_accepts_whole_paths(certain):
    """Random numbers of 0 accept every drafted token that has any probability: a chain to its end."""
    for kind in ("chain", "random"):
        c = _verify_case(1250, 5, 64, 333, kind, certain)
        c["tokens"] %= 333
        c["ua"][:] = 0
        n = _assert_verified(c)[1]
        assert kind != "chain" or n.tolist() == [64] * 5


def test_verification_of_many_requests():
    _assert_verified(_verify_case(1300, 300, 4, 5000, "beam", False))


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("R,T", [(2, 6), (129, 2)])
def test_verification_long_vocabulary(R, T, certain):
    """Rows past 256 blocks of 1,024 entries, with several workgroups a request and with one."""
    _assert_verified(_verify_case(2500 + R, R, T, 300_001, "random", certain, pad=3))


def test_verification_of_thousands():
    _assert_verified(_verify_case(2600, 3000, 1, 7, "chain", True, lens=[r % 2 for r in range(3000)]))


def test_verification_borders():
    """Probabilities in powers of two and random numbers on the borders between tokens: sums are exact in any order."""
    R, T, V = 40, 3, 8192
    c = _verify_case(1400, R, T, V, "beam", True)
    c["target"] = np.full((R, T, V), 1.0 / V, np.float32)
    c["target"][..., 1::2] = 0
    c["target"][..., 0::2] *= 2
    c["us"] = (np.arange(R) / R * V // 1 / V).astype(np.float32)
    c["us"][:3] = [0.0, 1.0 - 2.0 ** -24, 0.5]
    c["ua"][:] = 0.99
    ref = _assert_verified(c)
    assert np.all(ref[2][:, 0] % 2 == 0)


def test_verification_without_mass():
    """A draft row equal to the target's and rejected children of no probability leave no residual: the target's row
    stands in; a row without any mass emits -1; NaN and negative entries count as 0."""
    R, T, V = 4, 3, 6000
    c = _verify_case(1500, R, T, V, "beam", False)
    c["draft"] = c["target"].copy()
    c["tokens"] %= V
    for r in range(R):
        c["target"][r, 0, c["tokens"][r, 1:]] = c["draft"][r, 0, c["tokens"][r, 1:]] = 0
    c["target"][1, 0] = 0
    c["draft"][1, 0] = 0
    c["target"][2, 0, ::7] = np.nan
    c["draft"][2, 0, ::7] = -1.0
    ref = _assert_verified(c)
    assert ref[1].tolist() == [1] * R and ref[2][1, 0] == -1 and ref[2][0, 0] >= 0


# -- append --------------------------------------------------------------------------


@pytest.mark.parametrize("B,Hkv,T", [(16, 1, 1), (16, 8, 7), (32, 3, 40), (16, 2, 1000)])
@pytest.mark.parametrize("pinned", [False, True])
def test_append(B, Hkv, T, pinned):
    R = 4
    rng = np.random.default_rng(T)
    NB = (T + 100 + B - 1) // B
    NP = R * NB + 1
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    table[2, -1], table[3, 0] = NP, -1
    nk, nv = random_bf16(1600, (R, T, Hkv, 128)), random_bf16(1601, (R, T, Hkv, 128))
    kp, vp = random_bf16(1602, (NP, Hkv, B, 128)), random_bf16(1603, (NP, Hkv, B, 128))
    ctx = np.array([0, 33, NB * B - 1, 3], np.int32)  # the third has room for one token
    path = np.sort(rng.integers(0, T, (R, T)), -1).astype(np.int32)
    path[0, :1] = rng.choice([-1, T])
    for p, n in ((None, None), (None, [T, 0, T + 5, T // 2]), (path, [T, 1, -2, T])):
        pages = [dev_bf16(x) for x in (kp, vp)]
        if pinned:
            pages = [torch.empty(x.shape, dtype=x.dtype, pin_memory=True).copy_(x) for x in pages]
        ends = torch.full((R,), -9, dtype=torch.int32, device="cuda")
        note(f"append B={B} Hkv={Hkv} T={T} pinned={pinned} path={p is not None} n={n}")
        P.oasis_append_tokens(P.dims(R, Hkv, Hkv, 128, B, NB), dev_bf16(nk), dev_bf16(nv), T,
                              None if p is None else dev_i32(p), None if n is None else dev_i32(np.array(n)), *pages,
                              dev_i32(table), dev_i32(ctx), ends)
        torch.cuda.synchronize()
        rk, rv = kp.copy(), vp.copy()
        ref = O.append_tokens(nk, nv, p, n, rk, rv, table, ctx, B)
        assert np.array_equal(ends.cpu().numpy(), ref)
        assert np.array_equal(host_bits(pages[0]), rk) and np.array_equal(host_bits(pages[1]), rv)


# -- together ------------------------------------------------------------------------


class _Loop:
    """Speculative decoding of a few requests over the paged cache: a stand-in model turns attention outputs into the
    target's probabilities; drafted tokens, keys and values come from the seed."""

    R, Hq, Hkv, T, B, V, STEPS = 3, 8, 2, 9, 16, 300, 6

    def __init__(self):
        rng = np.random.default_rng(17)
        R, T, H, NB = self.R, self.T, self.Hkv, 12
        self.NB, self.ctx0 = NB, np.array([20, 15, 33], np.int32)
        self.table = rng.permutation(R * NB).reshape(R, NB).astype(np.int32)
        self.kp, self.vp = random_bf16(1701, (R * NB, H, self.B, 128)), random_bf16(1702, (R * NB, H, self.B, 128))
        self.parent = np.maximum(_parents(rng, R, T, "random"), 0)
        self.parent[:, 0] = -1
        self.steps = [dict(q=random_bf16(1710 + i, (R, T, self.Hq, 128)), k=random_bf16(1730 + i, (R, T, H, 128)),
                           v=random_bf16(1750 + i, (R, T, H, 128)), tokens=rng.integers(0, 4, (R, T)).astype(np.int32),
                           ua=rng.random((R, T), dtype=np.float32), us=rng.random(R, dtype=np.float32))
                      for i in range(self.STEPS)]
        self.head = (rng.standard_normal((self.Hq * 128, self.V)) * 0.3).astype(np.float32)
        self.d = P.dims(R, self.Hq, H, 128, self.B, NB)
        f32 = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        self.dev = [dict(q=dev_bf16(s["q"]), k=dev_bf16(s["k"]), v=dev_bf16(s["v"]), tokens=dev_i32(s["tokens"]),
                         ua=f32(s["ua"]), us=f32(s["us"])) for s in self.steps]
        self.dhead, self.dparent, self.dtable = f32(self.head), dev_i32(self.parent), dev_i32(self.table)
        self.out = torch.zeros((R, T, self.Hq, 128), dtype=torch.bfloat16, device="cuda")
        self.probs = torch.zeros((R, T, self.V), device="cuda")
        self.ints = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((R, T), (R,), (R, T))]
        self.ws = torch.zeros(max(P.oasis_tree_attn_workspace_bytes(self.d, T),
                                  P.oasis_verify_workspace_bytes(R, T, self.V)), dtype=torch.uint8, device="cuda")
        self.reset()

    def reset(self):
        self.dk, self.dv = dev_bf16(self.kp), dev_bf16(self.vp)
        self.ctx = [dev_i32(self.ctx0), dev_i32(self.ctx0)]

    def step(self, i, s):
        """One step: lengths go from self.ctx[i % 2] to the other one."""
        P.oasis_tree_attn(self.d, s["q"], self.T, self.dk, self.dv, self.dtable, self.ctx[i % 2], s["k"], s["v"],
                          self.dparent, None, None, self.out, None, self.ws)
        logits = self.out.view(self.R * self.T, -1).float() @ self.dhead
        logits[:, :4] += 7.0  # a few likely tokens, which the drafts are taken from
        self.probs.copy_(torch.softmax(logits, -1).view(self.R, self.T, self.V))
        P.oasis_verify_drafts(self.probs, None, s["tokens"], self.dparent, None, s["ua"], s["us"], *self.ints, self.ws)
        P.oasis_append_tokens(self.d, s["k"], s["v"], self.T, self.ints[0], self.ints[1], self.dk, self.dv, self.dtable,
                              self.ctx[i % 2], self.ctx[(i + 1) % 2])


def test_the_step_together():
    m = _Loop()
    kp, vp, ctx = m.kp.copy(), m.vp.copy(), m.ctx0.copy()
    grown = 0
    for i, s in enumerate(m.steps):
        note(f"speculative step {i}")
        m.step(i, m.dev[i])
        torch.cuda.synchronize()
        ref, ref_lse = O.tree_attend(s["q"], kp, vp, m.table, ctx, s["k"], s["v"], m.parent, [m.T] * m.R, m.B)
        ref_abs, _ = O.tree_attend(s["q"], kp, _magnitude(vp), m.table, ctx, s["k"], _magnitude(s["v"]), m.parent,
                                   [m.T] * m.R, m.B)
        _check(m.out, None, ref, ref_abs, ref_lse, m.out)
        want = O.verify_drafts(m.probs.cpu().numpy(), None, s["tokens"], m.parent, [m.T] * m.R, s["ua"], s["us"])
        for x, y in zip(m.ints, want):
            assert np.array_equal(x.cpu().numpy(), y)
        ctx = O.append_tokens(s["k"], s["v"], want[0], want[1], kp, vp, m.table, ctx, m.B)
        assert np.array_equal(m.ctx[(i + 1) % 2].cpu().numpy(), ctx)
        assert np.array_equal(host_bits(m.dk), kp) and np.array_equal(host_bits(m.dv), vp)
        grown = max(grown, int(want[1].max()))
    assert grown > 1


def test_the_step_captured_and_replayed():
    """Two steps in a graph, replayed between eager work: the same lengths, tokens and pages as the eager steps."""
    m = _Loop()
    eager = []
    for i in range(m.STEPS):
        m.step(i, m.dev[i])
        torch.cuda.synchronize()
        eager.append([x.clone() for x in (m.out, *m.ints, m.dk, m.dv, m.ctx[(i + 1) % 2])])
    m.reset()
    side = torch.cuda.Stream()
    slot = [{n: t.clone() for n, t in m.dev[i].items()} for i in range(2)]
    keep = [[torch.empty_like(t) for t in eager[0]] for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    note("capture of two speculative steps")
    with torch.cuda.graph(graph, stream=side):
        for i in range(2):
            m.step(i, slot[i])
            for a, b in zip(keep[i], (m.out, *m.ints, m.dk, m.dv, m.ctx[(i + 1) % 2])):
                a.copy_(b)
    for pair in range(m.STEPS // 2):
        for i in range(2):
            for n, t in m.dev[2 * pair + i].items():
                slot[i][n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        torch.ones(1000, device="cuda").cumsum(0)  # eager work in between
        for i in range(2):
            for a, b in zip(keep[i], eager[2 * pair + i]):
                assert torch.equal(a, b), (pair, i)


def test_another_stream_and_two_calls_at_once():
    """Calls on two streams with separate workspaces do not disturb each other."""
    ms = [_Loop(), _Loop()]
    want = []
    for i in range(ms[0].STEPS):
        ms[0].step(i, ms[0].dev[i])
    torch.cuda.synchronize()
    want = [ms[0].dk.clone(), ms[0].dv.clone(), *(x.clone() for x in ms[0].ints)]
    for m in ms:
        m.reset()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(ms[0].STEPS):
        for m, s in zip(ms, streams):
            with torch.cuda.stream(s):
                m.step(i, m.dev[i])
    torch.cuda.synchronize()
    for m in ms:
        for a, b in zip(want, (m.dk, m.dv, *m.ints)):
            assert torch.equal(a, b)


def test_a_stream_given_and_a_row_taken_twice():
    """The stream argument, and an append that names a row twice."""
    m = _Loop()
    s, side = m.dev[0], torch.cuda.Stream()
    for fast in (P._lib._fast, None):
        keep, P._lib._fast = P._lib._fast, fast
        try:
            m.reset()
            torch.cuda.synchronize()
            note("calls on a given stream")
            P.oasis_tree_attn(m.d, s["q"], m.T, m.dk, m.dv, m.dtable, m.ctx[0], s["k"], s["v"], m.dparent, None, None, m.out,
                              None, m.ws, side)
            path = torch.zeros((m.R, m.T), dtype=torch.int32, device="cuda")
            path[:, 0] = 1
            torch.cuda.synchronize()
            n = torch.full((m.R,), 3, dtype=torch.int32, device="cuda")
            torch.cuda.synchronize()
            P.oasis_append_tokens(m.d, s["k"], s["v"], m.T, path, n, m.dk, m.dv, m.dtable, m.ctx[0], m.ctx[1], side)
            side.synchronize()
        finally:
            P._lib._fast = keep
        h = m.steps[0]
        ref, ref_lse = O.tree_attend(h["q"], m.kp, m.vp, m.table, m.ctx0, h["k"], h["v"], m.parent, [m.T] * m.R, m.B)
        ref_abs, _ = O.tree_attend(h["q"], m.kp, _magnitude(m.vp), m.table, m.ctx0, h["k"], _magnitude(h["v"]), m.parent,
                                   [m.T] * m.R, m.B)
        _check(m.out, None, ref, ref_abs, ref_lse, m.out)
        kp, vp = m.kp.copy(), m.vp.copy()
        O.append_tokens(h["k"], h["v"], path.cpu().numpy(), n.cpu().numpy(), kp, vp, m.table, m.ctx0, m.B)
        assert np.array_equal(host_bits(m.dk), kp) and np.array_equal(host_bits(m.dv), vp)


def test_binding_checks_on_the_device():
    m = _Loop()
    s = m.dev[0]
    with pytest.raises(P.OasisError, match="tree_k is not 16-byte aligned"):
        odd = torch.zeros(s["k"].numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(s["k"].shape)
        P.oasis_tree_attn(m.d, s["q"], m.T, m.dk, m.dv, m.dtable, m.ctx[0], odd, s["v"], None, None, None, m.out, None, m.ws)
    with pytest.raises(P.OasisError, match="workspace of 0 bytes"):
        P.oasis_verify_drafts(m.probs, None, s["tokens"], None, None, s["ua"], s["us"], *m.ints, None)
    with pytest.raises(ValueError, match="evenly spaced"):
        P.oasis_verify_drafts(m.probs.transpose(0, 1).contiguous().transpose(0, 1), None, s["tokens"], None, None, s["ua"],
                              s["us"], *m.ints, m.ws)
    with pytest.raises(ValueError, match="draft_probs: shape"):
        P.oasis_verify_drafts(m.probs, m.probs[:, :, :-1], s["tokens"], None, None, s["ua"], s["us"], *m.ints, m.ws)
    with pytest.raises(TypeError, match="target_probs: dtype"):
        P.oasis_verify_drafts(m.probs.double(), None, s["tokens"], None, None, s["ua"], s["us"], *m.ints, m.ws)
    with pytest.raises(ValueError, match="pinned"):
        P.oasis_append_tokens(m.d, s["k"], s["v"], m.T, None, None, m.dk.cpu(), m.dv.cpu(), m.dtable, m.ctx[0], None)
    with pytest.raises(P.OasisError, match="new_ctx_len is ctx_len"):
        P.oasis_append_tokens(m.d, s["k"], s["v"], m.T, None, None, m.dk, m.dv, m.dtable, m.ctx[0], m.ctx[0])


def test_native_marshalling_takes_the_plain_calls_alone():
    """The step's calls go through the native marshalling (status 0), give what the Python binding gives, and hand every
    other form back to it."""
    import ctypes
    L = P._lib
    ms = [_Loop(), _Loop()]
    keep = L._fast
    for m, fast in zip(ms, (keep, None)):
        L._fast = fast
        try:
            for i in range(2):
                m.step(i, m.dev[i])
        finally:
            L._fast = keep
    torch.cuda.synchronize()
    for a, b in zip((ms[0].dk, ms[0].dv, ms[0].out, *ms[0].ints), (ms[1].dk, ms[1].dv, ms[1].out, *ms[1].ints)):
        assert torch.equal(a, b)
    m, s = ms[0], ms[0].dev[0]
    d = ctypes.addressof(m.d)
    smap = torch.full((m.R, m.Hkv, 11), -1, dtype=torch.int32, device="cuda")
    pv = torch.zeros(m.R, 12, m.Hkv, 128, m.B, dtype=torch.bfloat16, device="cuda")
    calls = {
        "tree_attn": [d, s["q"], m.T, m.dk, m.dv, m.dtable, m.ctx[0], s["k"], s["v"], m.dparent, None, None, m.out, None,
                      m.ws, None],
        "sparse_tree_attn": [d, s["q"], m.T, m.dk, pv, smap, 11, m.ctx[0], s["k"], s["v"], m.dparent, None, 0.5, m.out,
                             None, torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), None],
        "verify_drafts": [m.probs, None, s["tokens"], None, None, s["ua"], s["us"], *m.ints, m.ws, None],
        "append_tokens": [d, s["k"], s["v"], m.T, m.ints[0], m.ints[1], m.dk, m.dv, m.dtable, m.ctx[0], m.ctx[1], None],
    }
    wrong = {"tree_attn": {1: s["q"].float(), 2: -1, 3: m.dk[:-1], 5: m.dtable[:1], 6: m.ctx[0].long(), 7: s["k"][:1],
                           9: m.dparent.cpu(), 11: 1, 12: m.out.transpose(0, 1), 14: m.out, 15: "0"},
             "sparse_tree_attn": {3: m.dk[:-1], 6: 12, 5: None, 8: s["v"][:, :1], 14: m.out},
             "verify_drafts": {0: m.probs.double(), 1: m.probs[:, :, :-1], 2: None, 5: s["ua"].double(), 6: s["ua"],
                               7: m.ints[1], 10: m.out},
             "append_tokens": {1: s["k"].float(), 3: 1 << 40, 4: m.ints[1], 6: m.dk[:-1], 8: None, 10: m.ctx[1].long()}}
    for name, args in calls.items():
        note(f"native marshalling of {name}")
        assert getattr(keep, name)(*args) == 0
        assert getattr(keep, name)(*args[:-1]) is None
        for i, x in wrong[name].items():
            bad = list(args)
            bad[i] = x
            assert getattr(keep, name)(*bad) is None, (name, i)
    torch.cuda.synchronize()
