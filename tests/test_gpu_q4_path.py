"""The 4-bit cache's calls together: prompts, steps of drafted trees with verification, captured steps, calls on two
streams, against the float64 oracle and against each other."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from oracle import q4 as Q
from paper_2608_08097_amd.path_q4 import Q4Path
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import _check
from tests.test_gpu_q4 import _rotary, _turns, dev_u8
from workloads import random_bf16

pytestmark = pytest.mark.gpu

ROT = (64, True, 1.1)


def _new_rows(seed, R, N, H):
    return random_bf16(seed, (R, N, 3 * H, 128), scale=1.2)


@pytest.mark.parametrize("B,Hq,rows", [(16, 8, 5), (32, 16, 9)])
def test_prompts_and_steps(B, Hq, rows):
    """Two layers: a prompt in two chunks, then drafted trees whose accepted rows are committed; every output, page,
    compressed key and selection."""
    R, H, T, k, NB = 2, 2, rows, 4, 24
    rng = np.random.default_rng(B)
    note(f"4-bit path B={B} Hq={Hq} T={T}")
    d = P.dims(R, Hq, H, 128, B, NB)
    NP = R * NB + 1
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    path = Q4Path(d, T, k, NP, dev_i32(table), _rotary(*ROT))
    layers = [path.new_layer() for _ in range(2)]
    rot = (_turns(ROT[0]), *ROT[1:])
    pages = [[np.zeros((NP, Q.page_bytes(H, B)), np.uint8) for _ in range(2)] for _ in layers]
    sums = [[np.zeros((R, H, NB, 128)) for _ in range(2)] for _ in layers]
    ctx, new = dev_i32(np.zeros(R)), dev_i32(np.zeros(R))
    lens = np.zeros(R, np.int32)

    def same(layer, before, after):
        st, (kp, vp), (mx, mn) = layers[layer], pages[layer], sums[layer]
        assert np.array_equal(st.k_pages.cpu().numpy(), kp) and np.array_equal(st.v_pages.cpu().numpy(), vp)
        Q.update_summaries(kp, table, before, after, B, mx, mn, 1 << 30)
        for got, want in ((st.kmax, mx), (st.kmin, mn)):
            for r in range(R):
                n = O.block_counts(int(after[r]), B)[1]
                assert np.array_equal(O.bf16_to_f64(host_bits(got))[r, :, :n], want[r, :, :n])

    for chunk, n in enumerate((B * 7 + 3, B * 5)):
        count = np.array([n, n - 9], np.int32)
        for i, st in enumerate(layers):
            joint = _new_rows(10 * chunk + i, R, n, H)
            dev = dev_bf16(joint)
            path.append(st, dev[:, :, H:2 * H], dev[:, :, 2 * H:], ctx, new, dev_i32(count))
            ends, _, _ = Q.append_tokens(joint[:, :, H:2 * H], joint[:, :, 2 * H:], None, count, *pages[i], table, lens, B, rot)
            assert np.array_equal(new.cpu().numpy(), ends)
            same(i, lens, ends)
        lens = ends
        ctx.copy_(new)
    parent = np.array([[-1, 0, 0, 1, 1, 2, 3, 5, 7][:T]] * R, np.int32)
    depth = np.array([[len(p) - 1 for p in O.tree_paths(parent, [T], T)[0]]] * R)
    for step in range(3):
        q_bits, k_bits, v_bits = (random_bf16(100 * step + j, (R, T, h, 128)) for j, h in enumerate((Hq, H, H)))
        at = (lens[:, None] + depth).astype(np.int32)
        took = np.full((R, T), -1, np.int32)
        took[0, :3], took[1, :2] = [0, 1, 3], [0, 2]
        count = np.array([3, 2], np.int32)
        for i, st in enumerate(layers):
            q, tk = path.rotate(dev_bf16(q_bits), dev_bf16(k_bits), ctx, dev_i32(at))
            rq, rk = host_bits(q), host_bits(tk)  # held to the oracle in the tests of the rotation
            tv = dev_bf16(v_bits)
            path.predict(st, q, ctx)
            sel, cnt = st.sel.cpu().numpy(), st.sel_count.cpu().numpy()
            score = O.block_scores(rq, *(O.bf16_to_f64(host_bits(x)) for x in (st.kmax, st.kmin)), lens, H, B)
            for r in range(R):
                n = O.block_counts(int(lens[r]), B)[1]
                for h in range(H):
                    assert cnt[r, h] == min(k, n)
                    best = np.sort(score[r, h, :n])[::-1][:k]
                    assert np.allclose(np.sort(score[r, h, sel[r, h, :cnt[r, h]]])[::-1], best, rtol=1e-5)
            values = [Q.read_pages(p, H, B) for p in pages[i]]
            for dense in (False, True):
                st.out.fill_(7.0)
                if dense:
                    path.attend_dense(st, q, ctx, tk, tv, dev_i32(parent))
                else:
                    path.attend(st, q, ctx, tk, tv, dev_i32(parent))
                args = (rq, *values, table, lens, None if dense else sel, None if dense else cnt, rk, v_bits, parent, [T] * R, B)
                ref, ref_lse = Q.attend(*args)
                ref_abs, _ = Q.attend(*args, magnitude=True)
                _check(st.out, st.lse, ref, ref_abs, ref_lse, st.out)
            path.commit(st, tk, tv, dev_i32(took), dev_i32(count), ctx, new)
            ends, _, _ = Q.append_tokens(rk, v_bits, took, count, *pages[i], table, lens, B)
            assert np.array_equal(new.cpu().numpy(), ends)
            same(i, lens, ends)
        lens = ends
        ctx.copy_(new)


def test_without_rotation_rows_are_as_given():
    d = P.dims(1, 4, 2, 128, 16, 4)
    path = Q4Path(d, 2, 2, 4, dev_i32([[0, 1, 2, 3]]))
    q, k = dev_bf16(random_bf16(1, (1, 2, 4, 128))), dev_bf16(random_bf16(2, (1, 2, 2, 128)))
    assert path.rotate(q, k, dev_i32([5]))[0] is q and path.rotate(q, k, dev_i32([5]))[1] is k


def _step_state(seed, R=3, Hq=16, H=4, T=5, B=16, NB=40, k=6):
    rng = np.random.default_rng(seed)
    d = P.dims(R, Hq, H, 128, B, NB)
    NP = R * NB
    path = Q4Path(d, T, k, NP, dev_i32(rng.permutation(NP).reshape(R, NB)), P.Rotary(128))
    st = path.new_layer()
    st.k_pages.copy_(dev_u8(Q.make_pages(rng.normal(size=(NP, H, B, 128)))))
    st.v_pages.copy_(dev_u8(Q.make_pages(rng.normal(size=(NP, H, B, 128)))))
    st.kmax.zero_(), st.kmin.zero_()  # rows that are not written are compared too
    ctx = dev_i32(rng.integers(200, NB * B - 40, R))
    P.oasis_update_summaries_q4(d, st.k_pages, path.block_table, None, ctx, 0, st.kmax, st.kmin)
    q, k_rows, v_rows = (dev_bf16(random_bf16(seed + j, (R, T, h, 128))) for j, h in enumerate((Hq, H, H)))
    return path, st, ctx, dev_i32(np.zeros(R)), q, k_rows, v_rows


def _step(path, st, ctx, new, q, k, v):
    q, tk = path.rotate(q, k, ctx)
    path.predict(st, q, ctx)
    path.attend(st, q, ctx, tk, v)
    path.commit(st, tk, v, None, None, ctx, new)
    return [x.clone() for x in (st.out, st.lse, st.sel, st.k_pages, st.v_pages, st.kmax, st.kmin, new)]


def test_a_captured_step_replays():
    """Several replays, each with other inputs and with eager work and synchronisations between them, against eager steps
    from the same state."""
    path, st, ctx, new, q, k, v = _step_state(50)
    keep = [x.clone() for x in (st.k_pages, st.v_pages, st.kmax, st.kmin, ctx)]
    _step(path, st, ctx, new, q, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(path, st, ctx, new, q, k, v)
    for turn in range(4):
        rng = random_bf16(900 + turn, tuple(q.shape))
        q.copy_(dev_bf16(rng))
        v.mul_(-0.5)
        start = [x.clone() for x in keep[:4]]
        for x, y in zip((st.k_pages, st.v_pages, st.kmax, st.kmin), start):
            x.copy_(y)
        ctx.copy_(keep[4] + turn)
        want = [x.clone() for x in _step(path, st, ctx, new, q, k, v)]
        torch.cuda.synchronize()
        for x, y in zip((st.k_pages, st.v_pages, st.kmax, st.kmin), start):
            x.copy_(y)
        new.zero_()
        st.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(got, want)):
            same = torch.equal(x.view(torch.int16), y.view(torch.int16)) if x.dtype == torch.bfloat16 else torch.equal(x, y)
            assert same, (turn, i)


def test_two_paths_on_two_streams():
    """Each with its own workspace, at the same time."""
    states = [_step_state(60 + i) for i in range(2)]
    start = [[x.clone() for x in (s[1].k_pages, s[1].v_pages, s[1].kmax, s[1].kmin)] for s in states]
    want = [_step(*s) for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(3):
        for s, back in zip(states, start):
            for x, y in zip((s[1].k_pages, s[1].v_pages, s[1].kmax, s[1].kmin), back):
                x.copy_(y)
        torch.cuda.synchronize()
        got = []
        for s, stream in zip(states, streams):
            with torch.cuda.stream(stream):
                got.append(_step(*s))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for x, y in zip(g, w):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_the_same_call_twice_gives_the_same_bits():
    path, st, ctx, new, q, k, v = _step_state(70, R=2, NB=400, k=100)
    rows = []
    for _ in range(3):
        path.attend_dense(st, q, ctx, k, v)
        rows.append(st.out.clone())
    assert all(torch.equal(rows[0], x) for x in rows[1:])


def test_the_native_marshalling_takes_the_plain_calls():
    """Status 0, not None, from each native function, and the Python binding's results."""
    import ctypes
    from paper_2608_08097_amd import _lib as L
    L.lib()
    path, st, ctx, new, q, k, v = _step_state(80)
    d, rot = path.dims, path.rotary
    assert L._fast.rotate(ctypes.addressof(d), ctypes.addressof(rot.struct), rot.turns, path.T, None, ctx, q, path.q, k,
                          path.tree_k, False, None) == 0
    at = dev_i32(np.zeros((3, path.T)))
    assert L._fast.rotate(ctypes.addressof(d), ctypes.addressof(rot.struct), rot.turns, path.T, at, None, q, path.q, None,
                          None, True, None) == 0
    joint = torch.zeros((3, path.T, 8, 128), dtype=torch.bfloat16, device="cuda")
    for rows in (k, joint[:, :, :4]):
        assert L._fast.append_tokens_q4(ctypes.addressof(d), ctypes.addressof(rot.struct), rot.turns, rows, rows, path.T, None,
                                        None, st.k_pages, st.v_pages, path.block_table, ctx, new, None, None, None) == 0
    assert L._fast.append_tokens_q4(ctypes.addressof(d), 0, None, k, v, path.T, None, None, st.k_pages, st.v_pages,
                                    path.block_table, ctx, None, torch.zeros_like(k), torch.zeros_like(v), None) == 0
    for prev, most in ((None, 0), (ctx, 1)):
        assert L._fast.update_summaries_q4(ctypes.addressof(d), st.k_pages, path.block_table, prev, ctx, most, st.kmax, st.kmin,
                                           None) == 0
    for sel, cnt, n, tk, tv in ((st.sel, st.sel_count, path.k, k, v), (None, None, 0, None, None)):
        assert L._fast.tree_attn_q4(ctypes.addressof(d), q, path.T, st.k_pages, st.v_pages, path.block_table, sel, cnt, n, ctx,
                                    tk, tv, None, None, None, st.out, st.lse, path.ws, None) == 0
    # unusual forms are left to the Python binding: a half-given tree, pages of other shapes, rows without order
    assert L._fast.tree_attn_q4(ctypes.addressof(d), q, path.T, st.k_pages, st.v_pages, path.block_table, None, None, 0, ctx, k,
                                None, None, None, None, st.out, st.lse, path.ws, None) is None
    assert L._fast.tree_attn_q4(ctypes.addressof(d), q, path.T, st.k_pages, st.v_pages[:-1], path.block_table, None, None, 0,
                                ctx, None, None, None, None, None, st.out, st.lse, path.ws, None) is None
    assert L._fast.append_tokens_q4(ctypes.addressof(d), 0, None, k.transpose(1, 2).contiguous().transpose(1, 2), v, path.T, None,
                                    None, st.k_pages, st.v_pages, path.block_table, ctx, new, None, None, None) is None
    torch.cuda.synchronize()
    results = []
    for fast in (L._fast, None):
        state = _step_state(81)
        keep = L._fast
        L._fast = fast
        try:
            results.append(_step(*state))
        finally:
            L._fast = keep
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*results))
