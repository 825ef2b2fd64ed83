"""The 4-bit cache on the GPU against the float64 oracle: rotary positions, the append that quantises, compressed keys,
attention over every block and over the selected ones."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from oracle import q4 as Q
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import INF, NAN, _check, _parents
from workloads import random_bf16

pytestmark = pytest.mark.gpu


def dev_u8(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _turns(dim, scaling="by_turns"):
    return Q.frequencies(dim, 10000.0, scaling, 8.0, 4096.0, 1.0, 4.0)[0]


def _rotary(dim, interleaved, amplitude):
    return P.Rotary.from_turns(torch.from_numpy(_turns(dim)).cuda(), interleaved, amplitude)


# -- rotary positions ------------------------------------------------------------------


def _rotate_case(seed, R, T, Hq, Hkv, dim, interleaved, packed, explicit, inverse=False, amplitude=1.25, which="qk", in_place=False):
    rng = np.random.default_rng(seed)
    note(f"rotate seed={seed} R={R} T={T} Hq={Hq} Hkv={Hkv} dim={dim} next={interleaved} packed={packed} {which}")
    heads = Hq + 2 * Hkv
    bits = random_bf16(seed, (R, T, heads, 128), scale=3.0)
    ctx = rng.integers(-3, 1 << 20, R).astype(np.int32)
    at = rng.integers(-2 ** 31, 2 ** 31, (R, T)).astype(np.int32) if explicit else np.maximum(ctx, 0)[:, None] + np.arange(T)
    joint = dev_bf16(bits)
    q, k = joint[:, :, :Hq], joint[:, :, Hq:Hq + Hkv]
    if not packed:
        q, k = q.contiguous(), k.contiguous()
    outs = [(x if in_place else torch.full(x.shape, 7.0, dtype=torch.bfloat16, device="cuda")) if n in which else None
            for x, n in ((q, "q"), (k, "k"))]
    d = P.dims(R, Hq, Hkv, 128, 16, 1)
    rot = _rotary(dim, interleaved, amplitude)
    P.oasis_rotate(d, rot, T, dev_i32(at) if explicit else None, None if explicit else dev_i32(ctx),
                   q if "q" in which else None, outs[0], k if "k" in which else None, outs[1], inverse)
    torch.cuda.synchronize()
    for x, out in ((bits[:, :, :Hq], outs[0]), (bits[:, :, Hq:Hq + Hkv], outs[1])):
        if out is None:
            continue
        x = O.bf16_to_f64(np.ascontiguousarray(x))
        want = Q.rotate(x, at, _turns(dim), interleaved, amplitude, inverse)
        got = O.bf16_to_f64(host_bits(out))
        assert np.array_equal(got[..., dim:], x[..., dim:])
        a, b = (x[..., 0:dim:2], x[..., 1:dim:2]) if interleaved else (x[..., :dim // 2], x[..., dim // 2:dim])
        both = np.abs(a) + np.abs(b)
        size = np.repeat(both, 2, -1) if interleaved else np.concatenate([both, both], -1)
        # one rounding to bf16; sine, cosine, products and their sum are rounded to 2^-24 of the pair's size, four times
        tol = 2.0 ** -8 * np.abs(want[..., :dim]) + 4 * 2.0 ** -24 * amplitude * size
        err = np.abs(got - want)[..., :dim]
        assert np.all(err <= tol), np.max(err / tol)
    if in_place:
        assert np.array_equal(host_bits(joint[:, :, Hq + Hkv:]), bits[:, :, Hq + Hkv:])  # the values beside them


@pytest.mark.parametrize("dim", [2, 4, 6, 16, 30, 32, 48, 50, 64, 96, 112, 126, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_dims(dim, interleaved):
    _rotate_case(100 + dim, 3, 5, 8, 2, dim, interleaved, dim % 4 == 0, dim % 3 == 0)


@pytest.mark.parametrize("R,T,Hq,Hkv", [(1, 1, 1, 1), (1, 1, 32, 8), (5, 33, 3, 3), (2, 700, 8, 2), (1, 9001, 4, 1), (700, 1, 8, 8)])
def test_rotate_sizes(R, T, Hq, Hkv):
    _rotate_case(200 + T, R, T, Hq, Hkv, 128, False, True, False)
    _rotate_case(300 + T, R, T, Hq, Hkv, 64, True, False, True)


@pytest.mark.parametrize("dim,interleaved", [(128, False), (64, False), (50, False), (128, True), (38, True)])
def test_rotate_forms(dim, interleaved):
    _rotate_case(400 + dim, 2, 37, 8, 2, dim, interleaved, True, True, inverse=True)
    _rotate_case(401 + dim, 2, 37, 8, 2, dim, interleaved, True, False, in_place=True)
    _rotate_case(402 + dim, 2, 37, 8, 2, dim, interleaved, False, False, in_place=True)
    _rotate_case(403 + dim, 2, 5, 8, 2, dim, interleaved, True, True, which="q")
    _rotate_case(404 + dim, 2, 5, 8, 2, dim, interleaved, True, True, which="k")


def test_rotating_back_gives_the_gradient():
    """The inverse is the transpose: against differences of the forward call, in float32 steps that bf16 holds exactly."""
    R, T, H, dim = 1, 3, 2, 64
    rot = P.Rotary(dim, base=10000.0)
    d = P.dims(R, H, H, 128, 16, 1)
    ctx = dev_i32([77])
    g = dev_bf16(random_bf16(7, (R, T, H, 128)))
    grad = torch.zeros_like(g)
    P.oasis_rotate(d, rot, T, None, ctx, g, grad, None, None, True)
    weights = O.bf16_to_f64(host_bits(g))
    for dim_at in (0, 5, 31, 32, 63, 64, 127):
        x = torch.zeros_like(g)
        x[..., dim_at] = 1.0  # linear: the difference to 0 is the derivative
        y = torch.zeros_like(g)
        P.oasis_rotate(d, rot, T, None, ctx, x, y, None, None)
        slope = np.sum(O.bf16_to_f64(host_bits(y)) * weights, -1)
        # the column's two entries are rounded to bf16, and so is the gradient
        size = np.sum(np.abs(O.bf16_to_f64(host_bits(y)) * weights), -1)
        got = O.bf16_to_f64(host_bits(grad))[..., dim_at]
        assert np.all(np.abs(got - slope) <= 2.0 ** -8 * (size + np.abs(got)) + 1e-6)


# -- append ------------------------------------------------------------------------------


def _append_case(seed, R, H, T, B, ctx, path_len=None, rot=None, packed=False, bad=False, read=True, wild=False, new_len=True,
                 pinned=False, scale=1.0):
    rng = np.random.default_rng(seed)
    note(f"append seed={seed} R={R} H={H} T={T} B={B} ctx={list(ctx)[:6]} rot={rot} packed={packed}")
    ctx = np.array(ctx, np.int32)
    NB = max(1, (int(ctx.max()) + T + B - 1) // B - (1 if bad else 0))
    NP = R * NB + 2
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    if bad:
        table[rng.random((R, NB)) < 0.2] = rng.choice([-1, -2 ** 31, NP, 2 ** 31 - 1])
    joint = random_bf16(seed + 1, (R, T, 3 * H, 128), scale=scale)
    joint[rng.random(joint.shape) < 0.05] = 0
    joint[rng.random(joint.shape) < 0.02] = 0x8000
    if wild:
        joint[rng.random(joint.shape) < 0.004] = NAN
        joint[rng.random(joint.shape) < 0.004] = INF | 0x8000
        big = rng.random(joint.shape) < 0.01
        joint[big] = 0x7F7F
    path = None
    if path_len is not None:
        path = np.full((R, T), -1, np.int32)
        for r, n in enumerate(path_len):
            path[r, :max(0, min(n, T))] = np.sort(rng.permutation(T)[:max(0, min(n, T))])
        if bad:
            path[rng.random(path.shape) < 0.1] = rng.choice([-1, T, 2 ** 31 - 1])
    pages = [rng.integers(0, 256, (NP, Q.page_bytes(H, B))).astype(np.uint8) for _ in range(2)]
    both = dev_bf16(joint)
    new_k, new_v = both[:, :, H:2 * H], both[:, :, 2 * H:]
    if not packed:
        new_k, new_v = new_k.contiguous(), new_v.contiguous()
    dev = [dev_u8(p) for p in pages]
    if pinned:
        dev = [torch.empty(p.shape, dtype=p.dtype, pin_memory=True).copy_(p) for p in dev]
    reads = [torch.full((R, T, H, 128), 7.0, dtype=torch.bfloat16, device="cuda") if read else None for _ in range(2)]
    ends = torch.full((R,), -5, dtype=torch.int32, device="cuda") if new_len else None
    rotary = None if rot is None else _rotary(*rot)
    d = P.dims(R, 2 * H, H, 128, B, NB)
    args = (d, rotary, new_k, new_v, T, None if path is None else dev_i32(path),
            None if path_len is None else dev_i32(np.array(path_len)), *dev, dev_i32(table), dev_i32(ctx), ends, *reads)
    P.oasis_append_tokens_q4(*args)
    torch.cuda.synchronize()
    want_ends, want_read, done = Q.append_tokens(joint[:, :, H:2 * H], joint[:, :, 2 * H:], path, path_len, *pages, table, ctx,
                                                 B, None if rot is None else (_turns(rot[0]), *rot[1:]))
    for got, want, n in zip(dev, pages, "kv"):
        assert np.array_equal(got.cpu().numpy(), want), f"{n} pages: {np.argwhere(got.cpu().numpy() != want)[:4]}"
    if new_len:
        assert np.array_equal(ends.cpu().numpy(), want_ends)
    for got, want in zip(reads, want_read):
        if got is not None:
            x = got.double().cpu().numpy()
            assert np.array_equal(x[done], want[done], equal_nan=True)
            assert np.all(x[~done] == 7.0)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("ctx", [[0], [1], [15, 16, 17], [31, 32, 33], [0, 100, 64], [-4, 50, 33]])
def test_append_lengths(B, ctx):
    _append_case(1000 + B + len(ctx), len(ctx), 2, 21, B, ctx)
    _append_case(1100 + B + len(ctx), len(ctx), 2, 1, B, ctx, rot=(128, False, 1.0))


@pytest.mark.parametrize("dim", [2, 6, 32, 50, 64, 96, 126, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_rotated(dim, interleaved):
    _append_case(1200 + dim, 2, 3, 19, 16, [100, 30000], rot=(dim, interleaved, 1.1), packed=True)


@pytest.mark.parametrize("H", [1, 2, 3, 8])
def test_append_accepted_paths(H):
    _append_case(1300 + H, 5, H, 16, 16, [40, 17, 0, 31, 5], [3, 16, 0, 1, 99], packed=H % 2 == 0)
    _append_case(1310 + H, 3, H, 9, 32, [40, 17, 63], [3, -2, 9], rot=(64, H == 2, 1.0), read=False, new_len=False)


def test_append_what_does_not_fit():
    _append_case(1400, 4, 2, 33, 16, [40, 90, 0, 31], [30, 33, 7, 1], bad=True)
    _append_case(1401, 4, 2, 40, 32, [40, 90, 0, 31], bad=True, rot=(128, False, 1.0))


def test_append_values_at_the_ends_of_their_range():
    _append_case(1500, 2, 2, 40, 16, [3, 20], wild=True)
    _append_case(1501, 2, 2, 40, 16, [3, 20], wild=True, rot=(128, False, 1.0))
    _append_case(1502, 2, 2, 40, 16, [3, 20], wild=True, rot=(64, True, 1.5))
    for scale in (1e-38, 1e-30, 1e30):
        _append_case(1503, 1, 2, 20, 16, [3], scale=scale)
        _append_case(1504, 1, 2, 20, 16, [3], scale=scale, rot=(128, True, 1.0))


def test_append_chunks():
    _append_case(1600, 2, 4, 300, 16, [5, 0], rot=(128, False, 1.0), packed=True)
    _append_case(1601, 1, 1, 2100, 32, [7])
    _append_case(1602, 130, 2, 9, 16, list(range(130)), [*range(10)] * 13, rot=(96, False, 1.0))


def test_append_to_pinned_pages():
    _append_case(1700, 2, 2, 20, 16, [5, 0], rot=(128, False, 1.0), pinned=True)


# -- compressed keys -----------------------------------------------------------------------


def _summary_case(seed, R, H, B, ctx, prev=None, most=1, bad=False, nan=False, pinned=False):
    rng = np.random.default_rng(seed)
    note(f"summaries seed={seed} R={R} H={H} B={B} ctx={list(ctx)[:6]} prev={prev}")
    ctx = np.array(ctx, np.int32)
    NB = max(1, (int(ctx.max()) + B - 1) // B + 1)
    NP = R * NB + 1
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    if bad:
        table[rng.random((R, NB)) < 0.3] = rng.choice([-1, -2 ** 31, NP, 2 ** 31 - 1])
    x = rng.normal(size=(NP, H, B, 128)) * np.exp(rng.normal(size=(NP, H, B, 1)) * 3)
    pages = Q.make_pages(x)
    if nan:
        at = rng.random((NP, H, B)) < 0.2
        for p, h, t in np.argwhere(at):
            Q.write_token(pages[p], H, B, h, t, np.full(128, np.nan))
    shape = (R, H, NB, 128)
    before = [random_bf16(seed + i, shape) for i in (1, 2)]
    out = [dev_bf16(b) for b in before]
    d = P.dims(R, 2 * H, H, 128, B, NB)
    dev = dev_u8(pages)
    if pinned:
        dev = torch.empty(dev.shape, dtype=dev.dtype, pin_memory=True).copy_(dev)
    P.oasis_update_summaries_q4(d, dev, dev_i32(table), None if prev is None else dev_i32(np.array(prev)), dev_i32(ctx), most,
                                *out)
    torch.cuda.synchronize()
    want = [O.bf16_to_f64(b) for b in before]
    Q.update_summaries(pages, table, prev, ctx, B, *want, most)
    for got, w in zip(out, want):
        assert np.array_equal(O.bf16_to_f64(host_bits(got)), w)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("ctx", [[0], [1], [15, 16, 17, 32, 33, 34], [-3, 200, 97]])
def test_summaries_of_whole_contexts(B, ctx):
    _summary_case(2000 + B + len(ctx), len(ctx), 2, B, ctx)
    _summary_case(2100 + B + len(ctx), len(ctx), 3, B, ctx, bad=True, nan=True)


def test_summaries_of_new_blocks():
    _summary_case(2200, 6, 2, 16, [33, 48, 49, 200, 20, 5], [32, 40, 48, 90, 25, -1], 1)
    _summary_case(2201, 6, 2, 16, [33, 48, 49, 200, 20, 5], [32, 40, 16, 90, 25, 0], 3)
    _summary_case(2202, 2, 8, 32, [333, 48], [0, 0], 1 << 30)
    _summary_case(2203, 2, 8, 32, [333, 48], None, 0, pinned=True)


# -- attention -------------------------------------------------------------------------------


def _attn_case(seed, R, Hq, Hkv, T, B, ctx, kind="random", lens=None, k=None, bad=False, lse=True, scale=None, pinned=False, spare=0,
               count=None, stream=None, spread=1.0):
    """k: blocks selected at most (None: every block); count: how many of them; kind none: no tree."""
    rng = np.random.default_rng(seed)
    ctx = np.array(ctx, np.int32)
    note(f"attention seed={seed} R={R} Hq={Hq} Hkv={Hkv} T={T} B={B} ctx={ctx.tolist()[:6]} {kind} k={k} spare={spare}")
    q = random_bf16(seed + 1, (R, T, Hq, 128), scale=1.5)
    n = [T] * R if lens is None else lens
    tk = tv = parent = None
    if kind != "none":
        tk, tv = random_bf16(seed + 2, (R, T, Hkv, 128)), random_bf16(seed + 3, (R, T, Hkv, 128))
        parent = _parents(rng, R, T, kind)
    for r in range(R):
        q[r, max(0, n[r]):] = NAN
        if tk is not None:
            tk[r, max(0, n[r]):], tv[r, max(0, n[r]):] = NAN, INF
    NB = max(1, (max(int(ctx.max()), 1) + B - 1) // B + int(rng.integers(0, 3)))
    NP = R * NB + 2
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    sizes = np.exp(rng.normal(size=(2, NP, Hkv, B, 1)) * (spread - 1.0))
    kp, vp = (Q.make_pages(rng.normal(size=(NP, Hkv, B, 128)) * s) for s in sizes)
    held = np.zeros((NP, B), bool)
    for r in range(R):
        for t in range(min(max(int(ctx[r]), 0), NB * B)):
            held[table[r, t // B], t % B] = True
    for p in (kp, vp):  # what must not count: any codes, and powers among which there are NaN
        for page, t in np.argwhere(~held):
            for h in range(Hkv):
                at, powers = Q._places(Hkv, B, h, t)
                p[page, at:at + 64] = rng.integers(0, 256, 64)
                p[page, powers] = rng.choice([255, 254, 127, 0], 4)
    if bad:
        table[rng.random((R, NB)) < 0.2] = rng.choice([-1, -2 ** 31, NP, 2 ** 31 - 1])
    if spare:
        table = np.concatenate([table, rng.choice([-1, NP, 2 ** 31 - 1], (R, spare)).astype(np.int32)], 1)
        NB += spare
    sel = cnt = None
    if k is not None:
        sel, cnt = np.full((R, Hkv, k), -1, np.int32), np.zeros((R, Hkv), np.int32)
        for r in range(R):
            nc = O.block_counts(max(0, min(int(ctx[r]), NB * B)), B)[1]
            for h in range(Hkv):
                m = min(k, nc) if count is None else min(count, nc, k)
                cnt[r, h] = m
                sel[r, h, :m] = np.sort(rng.permutation(nc)[:m])
                if bad and m > 2:  # ids that are no candidates, and counts past k
                    sel[r, h, rng.integers(0, m)] = rng.choice([-7, nc, 2 ** 31 - 1])
                    cnt[r, h] = rng.choice([m, k + 5, 2 ** 31 - 1])
    d = P.dims(R, Hq, Hkv, 128, B, NB)
    before = dev_bf16(random_bf16(seed + 6, (R, T, Hq, 128)))
    out, lse = before.clone(), (torch.full((R, T, Hq), 7.0, device="cuda") if lse else None)
    ws = torch.full((P.oasis_tree_attn_q4_workspace_bytes(d, T, k or 0),), 255, dtype=torch.uint8, device="cuda")
    pages = [dev_u8(x) for x in (kp, vp)]
    if pinned:
        pages = [torch.empty(x.shape, dtype=x.dtype, pin_memory=True).copy_(x) for x in pages]
    P.oasis_tree_attn_q4(d, dev_bf16(q), T, *pages, dev_i32(table), dev_i32(ctx), None if sel is None else dev_i32(sel),
                         None if cnt is None else dev_i32(cnt), k or 0, None if tk is None else dev_bf16(tk),
                         None if tv is None else dev_bf16(tv), None if parent is None else dev_i32(parent),
                         None if lens is None else dev_i32(np.array(lens)), scale, out, lse, ws, stream)
    torch.cuda.synchronize()
    used = sorted({int(p) for p in table.reshape(-1) if 0 <= p < NP})
    kv, vv = np.zeros((NP, Hkv, B, 128)), np.zeros((NP, Hkv, B, 128))
    kv[used], vv[used] = Q.read_pages(kp[used], Hkv, B), Q.read_pages(vp[used], Hkv, B)
    args = (q, kv, vv, table, ctx, sel, cnt, tk, tv, parent, n, B, scale)
    ref, ref_lse = Q.attend(*args)
    ref_abs, _ = Q.attend(*args, magnitude=True)
    empty = ref_lse == -np.inf
    if lse is not None:
        assert np.all(lse.cpu().numpy()[empty] == -np.inf)
        lse[torch.from_numpy(empty).cuda()] = 0.0
    _check(out, lse, ref, ref_abs, np.where(empty, 0.0, ref_lse), before)
    assert not host_bits(out)[empty].any()
    if lse is not None:
        assert torch.all(lse.cpu()[torch.from_numpy(np.isnan(ref_lse))] == 7.0)


@pytest.mark.parametrize("T", [1, 2, 5, 8, 9, 16, 17, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("kind", ["chain", "random", "none"])
def test_dense_tree_sizes(T, kind):
    _attn_case(3000 + T, 2, 8, 2, T, 16, [77, 40], kind, [T, (T + 1) // 2])


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("ctx", [[0], [1], [15, 16, 17], [31, 32, 33], [63, 64, 65], [0, 1000, 64], [-4, 500, 333], [4097]])
def test_dense_lengths(B, ctx):
    _attn_case(3100 + B + len(ctx), len(ctx), 8, 2, 3, B, ctx)
    _attn_case(3200 + B + len(ctx), len(ctx), 4, 2, 1, B, ctx, "none")


@pytest.mark.parametrize("G", [1, 3, 4, 5, 8, 16])
def test_dense_head_groups(G):
    """Rows from one tile to several groups of tiles."""
    _attn_case(3300 + G, 1, G * 2, 2, 20, 16, [700], "beam")
    _attn_case(3310 + G, 2, G * 3, 3, 3, 32, [300, 70], "random")


def test_dense_many_splits_and_roots():
    _attn_case(3400, 1, 4, 1, 7, 16, [9000])
    _attn_case(3401, 3, 4, 1, 9, 32, [9000, 12, 2500], "roots", [9, 4, 0])
    _attn_case(3402, 2, 4, 1, 1, 16, [9000, 12], "none", [1, 0])


def test_dense_wide_rows():
    _attn_case(3500, 1, 32, 2, 64, 32, [1500], "beam", [61])
    _attn_case(3501, 1, 64, 1, 64, 16, [100], "random", [63])


@pytest.mark.parametrize("G,T", [(4, 9), (3, 13), (4, 16), (5, 13), (8, 16), (4, 33), (16, 16), (9, 63), (64, 5)])
def test_rows_of_several_tiles(G, T):
    """Three, four and more row tiles, in one group and in several, with rows left over."""
    _attn_case(3510 + G * T, 2, G * 2, 2, T, 16, [777, 40], "random", [T, (T + 1) // 2])
    _attn_case(3511 + G * T, 2, G * 2, 2, T, 32, [777, 40], "none", [T, (T + 1) // 2], k=7)


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("ctx", [[0], [1], [15, 16, 17], [31, 32, 33], [63, 64, 65], [0, 1000, 64], [-4, 500, 333], [4097]])
def test_rows_of_several_tiles_lengths(B, ctx):
    _attn_case(3560 + B + len(ctx), len(ctx), 24, 2, 5, B, ctx)
    _attn_case(3570 + B + len(ctx), len(ctx), 16, 2, 20, B, ctx, "beam")
    _attn_case(3580 + B + len(ctx), len(ctx), 16, 2, 10, B, ctx, "none")


@pytest.mark.parametrize("G,T", [(5, 13), (5, 16), (6, 15), (3, 32), (7, 15), (8, 14), (11, 11), (8, 16)])
def test_five_to_eight_tiles_over_long_tables(G, T):
    """One group of so many row tiles (a table of many units), with a last tile that is full or not, and trees that leave
    whole tiles unused."""
    for k in (None, 3000):
        _attn_case(3700 + G * T, 3, G * 2, 2, T, 16, [300, 20, 0], "random", [T, T // 2, T - 1], spare=7000, k=k)
        _attn_case(3800 + G * T, 2, G * 2, 2, T, 32, [77, 1100], "beam", [3, T], spare=4000, k=k)
        _attn_case(3900 + G * T, 2, G * 2, 2, T, 16, [65, 1000], "none", spare=7000, k=k)


@pytest.mark.parametrize("G,T", [(4, 3), (20, 2), (20, 4)])
def test_long_contexts_in_one_split(G, T):
    """So many pairs that they are hardly split, or not at all, two of them with thousands of blocks: lists of blocks in
    several pieces."""
    R, B, NB, NP = 1024, 32, 2205, 2300
    ctx = np.zeros(R, np.int32)
    ctx[[3, 700]] = 2060 * 32 + 5, NB * B - 40
    rng = np.random.default_rng(G)
    q = random_bf16(3590, (R, T, G, 128))
    kp, vp = (Q.make_pages(rng.normal(size=(NP, 1, B, 128))) for _ in range(2))
    table = np.broadcast_to(rng.permutation(NP)[:NB], (R, NB)).astype(np.int32)
    sel = np.broadcast_to(np.arange(2100), (R, 1, 2100)).astype(np.int32)
    d = P.dims(R, G, 1, 128, B, NB)
    note(f"attention of long contexts G={G} T={T}")
    for k in (0, 2100):
        out, lse = torch.zeros((R, T, G, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((R, T, G), device="cuda")
        ws = torch.zeros(P.oasis_tree_attn_q4_workspace_bytes(d, T, k), dtype=torch.uint8, device="cuda")
        cnt = np.minimum(np.maximum(-(-ctx // B) - 1, 0), 2100)[:, None]
        P.oasis_tree_attn_q4(d, dev_bf16(q), T, dev_u8(kp), dev_u8(vp), dev_i32(table), dev_i32(ctx), dev_i32(sel) if k else None,
                             dev_i32(cnt) if k else None, k, None, None, None, None, None, out, lse, ws)
        some = [3, 5, 700]
        args = (q[some], Q.read_pages(kp, 1, B), Q.read_pages(vp, 1, B), table[some], ctx[some], sel[some] if k else None,
                cnt[some] if k else None, None, None, None, [T] * 3, B)
        ref, ref_lse = Q.attend(*args)
        ref_abs, _ = Q.attend(*args, magnitude=True)
        assert torch.all(lse[5] == -torch.inf) and not out[5].any()
        keep = np.array([0, 2])
        _check(out[some][keep], lse[some][keep], ref[keep], ref_abs[keep], ref_lse[keep], out[some][keep])


def test_pages_outside_the_tier():
    for k in (None, 9):
        _attn_case(3600, 3, 8, 2, 4, 16, [300, 555, 90], bad=True, k=k)
        _attn_case(3601, 2, 8, 2, 12, 32, [300, 555], bad=True, k=k)


def test_long_tables():
    """Block tables far wider than the contexts: many splits, most of them empty."""
    for k in (None, 3000):
        _attn_case(3650, 2, 8, 2, 3, 16, [300, 20], spare=6000, k=k)
        _attn_case(3651, 2, 16, 2, 9, 32, [300, 0], "beam", spare=6000, k=k)


@pytest.mark.parametrize("R,Hkv,G,T,hi", [(64, 16, 2, 3, 60), (40, 8, 4, 10, 130), (80, 8, 4, 2, 90), (12, 8, 16, 20, 300)])
def test_dense_many_pairs(R, Hkv, G, T, hi):
    """More workgroups than the chip holds at once; lengths with ties, empty and negative ones, in no order."""
    rng = np.random.default_rng(R)
    ctx = rng.integers(0, hi, R)
    ctx[::5], ctx[1::7], ctx[2], ctx[3] = hi // 2, 0, -2 ** 31, -1
    _attn_case(3700 + R, R, Hkv * G, Hkv, T, 16, list(ctx), lens=list(rng.integers(0, T + 1, R)))


@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 17, 64])
def test_selected_blocks(B, k):
    _attn_case(3800 + k, 3, 12, 2, 4, B, [1500, 16, 0], k=k)
    _attn_case(3810 + k, 2, 8, 2, 5, B, [777, 40], "none", [5, 3], k=k)
    _attn_case(3820 + k, 1, 8, 1, 40, B, [1501], "beam", k=k)


def test_selected_fewer_than_k():
    _attn_case(3900, 2, 8, 2, 3, 16, [1500, 700], k=50, count=0)
    _attn_case(3901, 2, 8, 2, 3, 16, [1500, 700], k=50, count=7)
    _attn_case(3902, 2, 8, 2, 3, 16, [0, 9], "none", k=50)
    _attn_case(3903, 1, 8, 1, 5, 16, [8000], k=499)


def test_scale_and_no_lse():
    for k in (None, 5):
        _attn_case(4000, 2, 8, 2, 4, 16, [300, 20], lse=False, scale=0.05, k=k)
        _attn_case(4001, 1, 8, 2, 4, 16, [300], scale=0.0, k=k)
        _attn_case(4002, 1, 8, 2, 4, 16, [300], scale=-0.07, k=k)
        _attn_case(4003, 2, 16, 2, 20, 32, [45, 0], "none", scale=0.0, k=k)


def test_powers_of_any_size():
    for k in (None, 5):
        _attn_case(4050, 2, 8, 2, 5, 16, [300, 20], spread=2.5, k=k)


def test_pinned_pages():
    _attn_case(4100, 2, 8, 2, 4, 16, [300, 20], pinned=True)
    _attn_case(4101, 2, 8, 2, 4, 16, [300, 20], pinned=True, k=6)


def test_on_a_stream_of_its_own():
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _attn_case(4150, 2, 8, 2, 4, 16, [300, 20], stream=side)


def test_offsets_past_32_bits():
    """Pages of more than 2^32 bytes; only the last ones are used."""
    H, B, T, L = 8, 32, 3, 90
    NP = (1 << 32) // Q.page_bytes(H, B) + 40
    kp, vp = (torch.zeros((NP, Q.page_bytes(H, B)), dtype=torch.uint8, device="cuda") for _ in range(2))
    rng = np.random.default_rng(5)
    hk, hv = (Q.make_pages(rng.normal(size=(3, H, B, 128))) for _ in range(2))
    kp[-3:], vp[-3:] = dev_u8(hk), dev_u8(hv)
    q = random_bf16(11, (1, T, 2 * H, 128))
    table, small = np.array([[NP - 1, NP - 3, NP - 2, -1]], np.int32), np.array([[2, 0, 1, -1]], np.int32)
    d = P.dims(1, 2 * H, H, 128, B, 4)
    note("offsets past 32 bits")
    new = random_bf16(12, (1, T, H, 128))
    ends = dev_i32([0])
    P.oasis_append_tokens_q4(d, None, dev_bf16(new), dev_bf16(new), T, None, None, kp, vp, dev_i32(table), dev_i32([L - T]), ends)
    Q.append_tokens(new, new, None, None, hk, hv, small, [L - T], B)
    assert np.array_equal(kp[-3:].cpu().numpy(), hk) and np.array_equal(vp[-3:].cpu().numpy(), hv)
    summaries = [torch.zeros((1, H, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    P.oasis_update_summaries_q4(d, kp, dev_i32(table), None, ends, 0, *summaries)
    want = [np.zeros((1, H, 4, 128)) for _ in range(2)]
    Q.update_summaries(hk, small, None, [L], B, *want)
    for got, w in zip(summaries, want):
        assert np.array_equal(O.bf16_to_f64(host_bits(got)), w)
    args = (q, Q.read_pages(hk, H, B), Q.read_pages(hv, H, B), small, [L])
    for sel, cnt, k in ((None, None, 0), (np.full((1, H, 1), 1, np.int32), np.ones((1, H), np.int32), 1)):
        out, lse = torch.zeros((1, T, 2 * H, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, T, 2 * H), device="cuda")
        ws = torch.zeros(P.oasis_tree_attn_q4_workspace_bytes(d, T, k), dtype=torch.uint8, device="cuda")
        P.oasis_tree_attn_q4(d, dev_bf16(q), T, kp, vp, dev_i32(table), ends, None if sel is None else dev_i32(sel),
                             None if cnt is None else dev_i32(cnt), k, None, None, None, None, None, out, lse, ws)
        ref, ref_lse = Q.attend(*args, sel, cnt, None, None, None, [T], B)
        ref_abs, _ = Q.attend(*args, sel, cnt, None, None, None, [T], B, magnitude=True)
        _check(out, lse, ref, ref_abs, ref_lse, out)
