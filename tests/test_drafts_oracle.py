"""The speculative step's oracle against worked examples and the mathematics (CPU), and the entry points' refusals,
none of which reaches a HIP call."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from workloads import random_bf16


def test_paths_of_a_tree():
    parent = np.array([[-1, 0, 0, 1, 3, 9, 4]])
    assert O.tree_paths(parent, [7], 7) == [[[0], [1, 0], [2, 0], [3, 1, 0], [4, 3, 1, 0], [5], [6, 4, 3, 1, 0]]]
    assert O.tree_paths(None, [3, 0, 9], 4) == [[[0], [1, 0], [2, 1, 0]], [], [[0], [1, 0], [2, 1, 0], [3, 2, 1, 0]]]


def test_a_chain_over_the_cache_is_causal_attention():
    """The chain's tokens in the cache, one by one, and textbook attention over what each row sees."""
    T, H, B, L = 4, 2, 16, 21
    q, k, v = (random_bf16(s, (1, L + T, H, 128)) for s in (1, 2, 3))
    pages = [np.zeros((3, H, B, 128), np.uint16) for _ in range(2)]
    table = np.array([[2, 0, 1]], np.int32)
    ctx = O.append_tokens(k, v, None, [L], *pages, table, [0], B)
    assert ctx.tolist() == [L]
    out, lse = O.tree_attend(q[:, L:], *pages, table, ctx, k[:, L:], v[:, L:], None, [T], B)
    f = [torch.from_numpy(O.bf16_to_f64(x))[0].transpose(0, 1) for x in (q, k, v)]
    ref = torch.nn.functional.scaled_dot_product_attention(*f, is_causal=True).transpose(0, 1)[L:]
    assert np.allclose(out[0], ref.numpy(), rtol=0, atol=1e-12)
    logits = torch.matmul(f[0], f[1].transpose(1, 2))[:, L + 1, :L + 2] / 128 ** 0.5
    assert np.allclose(lse[0, 1], torch.logsumexp(logits, -1).numpy(), rtol=0, atol=1e-12)
    # the same over a working set whose slots hold block 0 and whose local block is block 1
    pool = [np.stack([p[2], p[0]])[None] for p in pages]
    smap = np.zeros((1, H, 1), np.int32)
    sp, sl = O.sparse_tree_attend(q[:, L:], *pool, smap, ctx, k[:, L:], v[:, L:], None, [T], B)
    assert np.allclose(sp, out, rtol=0, atol=1e-12) and np.allclose(sl, lse, rtol=0, atol=1e-12)


def test_verification_by_hand():
    p = np.array([[[0.5, 0.25, 0.25, 0.0], [0.0, 0.0, 0.5, 0.5], [0.25, 0.25, 0.25, 0.25]]])
    q = np.array([[[0.25, 0.75, 0.0, 0.0], [0.0, 0.0, 1.0, 0.0], [0.25, 0.25, 0.25, 0.25]]])
    tok = np.array([[7, 1, 2]])

    def run(ua, us, **kw):
        path, n, out = O.verify_drafts(p, kw.get("q", q), kw.get("tok", tok), kw.get("parent"), [kw.get("n", 3)],
                                       np.array([[0.0] + ua]), [us])
        return path[0, :n[0]].tolist(), out[0, :n[0]].tolist()

    assert run([0.3, 0.4], 0.6) == ([0, 1, 2], [1, 2, 2])     # 0.3 * 0.75 < 0.25, 0.4 * 1 < 0.5, then the last row
    assert run([1 / 3, 0.0], 0.0) == ([0], [0])                # 0.25 < 0.25 is false; residual [0.25, 0, 0.25, 0]
    assert run([1 / 3, 0.0], 0.5) == ([0], [2])                # 0.25 > 0.25 is false
    assert run([0.0, 0.5], 0.999) == ([0, 1], [1, 3])          # second row: residual [0, 0, 0, 0.5]
    assert run([0.0, 0.0], 0.0, n=1) == ([0], [0])
    assert run([0.0, 0.0], 0.0, n=0) == ([], [])
    # two children of the root: the first one's rejection leaves [0.25, 0, 0.25, 0] of mass 0.5 for the second
    kids = dict(parent=np.array([[-1, 0, 0]]), tok=np.array([[0, 1, 0]]))
    assert run([0.9, 0.99], 0.0, **kids) == ([0, 2], [0, 0])   # 0.99 * 0.25 * 0.5 < 0.25
    # certain drafts: token 1 rejected (0.3 >= 0.25); of mass 0.75 token 0 has 0.5
    assert run([0.3, 0.66], 0.9, q=None, **kids) == ([0, 2], [0, 3])
    assert run([0.3, 0.67], 0.9, q=None, **kids) == ([0], [2])
    same = dict(parent=np.array([[-1, 0, 0]]), tok=np.array([[0, 1, 1]]))
    assert run([0.3, 0.0], 0.6, q=None, **same) == ([0], [0])  # the same token again has no mass left
    assert run([0.0, 0.0], 0.9, tok=np.array([[0, 4, 1]])) == ([0], [2])  # no such token: passed over


@pytest.mark.parametrize("certain", [False, True])
def test_emitted_tokens_follow_the_target(certain):
    """The first emitted token's frequencies are the target's, whatever the drafts."""
    rng = np.random.default_rng(5)
    V, N, T = 5, 40000, 3
    p, q = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    target = np.broadcast_to(p, (N, T, V))
    draft = None if certain else np.broadcast_to(q, (N, T, V))
    parent = np.broadcast_to([-1, 0, 0], (N, T))
    tokens = np.broadcast_to([0, 3, 1], (N, T)) if certain else rng.choice(V, size=(N, T), p=q)
    _, _, out = O.verify_drafts(target, draft, tokens, parent, [T] * N, rng.random((N, T)), rng.random(N))
    freq = np.bincount(out[:, 0], minlength=V) / N
    assert np.all(np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / N))  # five deviations of a frequency over N draws


def test_append_skips_what_has_no_place():
    nk = random_bf16(7, (2, 3, 1, 128))
    pages = [np.zeros((4, 1, 16, 128), np.uint16) for _ in range(2)]
    table = np.array([[0, 1], [2, -1]], np.int32)
    path = np.array([[0, 2, -1], [1, 5, 2]], np.int32)
    ends = O.append_tokens(nk, nk, path, [2, 3], *pages, table, [31, 14], 16)
    assert ends.tolist() == [32, 17]
    assert np.array_equal(pages[0][1, 0, 15], nk[0, 0, 0]) and np.array_equal(pages[0][2, 0, 14], nk[1, 1, 0])
    assert np.count_nonzero(pages[0].any(axis=(1, 3))) == 2  # nothing else was written


# -- refusals ----------------------------------------------------------------------


def _ptr(n=1):
    return [ctypes.c_void_p(4096 * (i + 1)) for i in range(n)]  # aligned stand-ins, never dereferenced


def _refused(status, code, text):
    assert status == code and text in P.oasis_last_error(), (status, P.oasis_last_error())


def test_tree_attention_refusals():
    L = P.lib()
    p = _ptr(12)
    d = P.dims(2, 32, 8, 128, 16, 64)

    def paged(dims=d, T=5, num_pages=10, scale=0.1, ws=1 << 40, **bad):
        a = dict(zip(("q", "k", "v", "table", "ctx", "tk", "tv", "parent", "len", "out", "lse", "ws"), p))
        a.update(bad)
        return L.oasis_tree_attn(ctypes.byref(dims), a["q"], T, a["k"], a["v"], num_pages, a["table"], a["ctx"], a["tk"],
                                 a["tv"], a["parent"], a["len"], scale, a["out"], a["lse"], a["ws"], ws, None)

    def sparse(dims=d, T=5, ks=4096, scale=0.1, ws=1 << 40, **bad):
        a = dict(zip(("q", "k", "v", "map", "ctx", "tk", "tv", "parent", "len", "out", "lse", "ws"), p))
        a.update(bad)
        return L.oasis_sparse_tree_attn(ctypes.byref(dims), a["q"], T, a["k"], a["v"], a["map"], ks, a["ctx"], a["tk"],
                                        a["tv"], a["parent"], a["len"], scale, a["out"], a["lse"], a["ws"], ws, None)

    assert min(P.oasis_tree_attn_workspace_bytes(d, 5), P.oasis_sparse_tree_attn_workspace_bytes(d, 5, 4096)) > 16
    for f in (paged, sparse):
        _refused(f(dims=P.dims(2, 32, 8, 64, 16, 64)), 2, "head_dim")
        _refused(f(dims=P.dims(2, 32, 8, 128, 8, 64)), 2, "block_size")
        _refused(f(dims=P.dims(2, 30, 8, 128, 16, 64)), 1, "multiple")
        _refused(f(T=0), 1, "num_q_tokens < 1")
        _refused(f(T=65), 2, "num_q_tokens 65")
        _refused(f(dims=P.dims(2, 65 * 8, 8, 128, 16, 64), T=64), 2, "4160 rows")
        _refused(f(dims=P.dims(2, 32, 8, 128, 32, 1 << 27)), 2, "31 bits")
        _refused(f(scale=float("nan")), 1, "scale")
        for name, arg in (("q", "q"), ("tree_k", "tk"), ("tree_v", "tv"), ("out", "out")):
            _refused(f(**{arg: None}), 1, f"{name} is NULL")
            _refused(f(**{arg: ctypes.c_void_p(4098)}), 1, f"{name} is not 16-byte aligned")
        _refused(f(ctx=None), 1, "ctx_len is NULL")
        _refused(f(ws=16), 4, "workspace of 16 bytes")
        assert f(dims=P.dims(0, 32, 8, 128, 16, 64), q=None) == 0  # no requests: nothing to do
    _refused(paged(num_pages=0), 1, "num_pages")
    _refused(paged(k=None), 1, "k_pages is NULL")
    _refused(paged(table=None), 1, "block_table is NULL")
    _refused(sparse(ks=-1), 1, "k_slots < 0")
    _refused(sparse(map=None), 1, "slot_map is NULL")
    # positions are rounded up to whole units, and the scale multiplied by log2(e), before they are used
    longest = P.dims(1, 32, 8, 128, 16, (1 << 27) - 1)
    _refused(paged(dims=longest), 2, "31 bits")
    _refused(sparse(dims=longest), 2, "31 bits")
    for f in (paged, sparse):
        _refused(f(scale=3e38), 1, "scale")
    assert P.oasis_tree_attn_workspace_bytes(P.dims(1, 32, 8, 128, 16, (1 << 27) - 3), 5) > 0
    assert P.oasis_tree_attn_workspace_bytes(d, 65) == 0 == P.oasis_sparse_tree_attn_workspace_bytes(d, 5, -1)


def test_verification_refusals():
    L = P.lib()
    p = _ptr(10)

    def call(R=2, T=4, V=100, ts=100, ds=100, nbytes=1 << 30, **bad):
        a = dict(zip(("target", "draft", "tokens", "parent", "len", "ua", "us", "path", "n", "out"), p), ws=p[0])
        a.update(bad)
        return L.oasis_verify_drafts(R, T, V, a["target"], ts, a["draft"], ds, a["tokens"], a["parent"], a["len"], a["ua"],
                                     a["us"], a["path"], a["n"], a["out"], a["ws"], nbytes, None)

    _refused(call(R=-1), 1, "num_reqs")
    _refused(call(R=65536), 2, "num_reqs")
    _refused(call(T=0), 1, "num_q_tokens")
    _refused(call(T=65), 2, "num_q_tokens")
    _refused(call(V=0), 1, "vocab")
    _refused(call(ts=99), 1, "row stride")
    _refused(call(ds=99), 1, "row stride")
    for name, arg in (("target_probs", "target"), ("tokens", "tokens"), ("accept_u", "ua"), ("sample_u", "us"),
                      ("path", "path"), ("path_len", "n"), ("out_tokens", "out")):
        _refused(call(**{arg: None}), 1, f"{name} is NULL")
    _refused(call(nbytes=8), 4, "workspace of 8 bytes")
    _refused(call(ws=None), 4, "workspace")
    assert call(R=0) == 0 and P.oasis_verify_workspace_bytes(0, 4, 100) == 0


def test_append_refusals():
    L = P.lib()
    p = _ptr(9)
    d = P.dims(2, 32, 8, 128, 16, 64)

    def call(dims=d, N=4, pages=10, **bad):
        a = dict(zip(("nk", "nv", "path", "n", "k", "v", "table", "ctx", "new"), p))
        a.update(bad)
        return L.oasis_append_tokens(ctypes.byref(dims), a["nk"], a["nv"], N, a["path"], a["n"], a["k"], a["v"], pages,
                                     a["table"], a["ctx"], a["new"], None)

    _refused(call(N=0), 1, "num_tokens")
    _refused(call(N=1 << 24), 2, "num_tokens")
    _refused(call(pages=0), 1, "num_pages")
    _refused(call(n=None), 1, "path without path_len")
    _refused(call(new=p[7]), 1, "new_ctx_len is ctx_len")
    for name, arg in (("new_k", "nk"), ("new_v", "nv"), ("k_pages", "k"), ("v_pages", "v"), ("block_table", "table"),
                      ("ctx_len", "ctx")):
        _refused(call(**{arg: None}), 1, f"{name} is NULL")
    assert call(dims=P.dims(0, 32, 8, 128, 16, 64)) == 0


def test_the_binding_refuses_host_tensors_types_and_shapes():
    d = P.dims(1, 4, 2, 128, 16, 4)
    bf, i32 = torch.bfloat16, torch.int32
    q, tk = torch.zeros(1, 3, 4, 128, dtype=bf), torch.zeros(1, 3, 2, 128, dtype=bf)
    pages, table, ctx = torch.zeros(4, 2, 16, 128, dtype=bf), torch.zeros(1, 4, dtype=i32), torch.zeros(1, dtype=i32)
    with pytest.raises(ValueError, match="q must be a device tensor"):
        P.oasis_tree_attn(d, q, 3, pages, pages, table, ctx, tk, tk, None, None, None, q, None, None)
    with pytest.raises(ValueError, match="tree_k: 768 elements, 1024 expected"):
        P.oasis_tree_attn(d, torch.zeros(1, 4, 4, 128, dtype=bf), 4, pages, pages, table, ctx, tk, tk, None, None, None,
                          torch.zeros(1, 4, 4, 128, dtype=bf), None, None)
    with pytest.raises(ValueError, match="parent: 2 elements"):
        P.oasis_sparse_tree_attn(d, q, 3, pages[:1], pages[:1], None, 0, ctx, tk, tk, torch.zeros(2, dtype=i32), None, None,
                                 q, None, None)
    probs = torch.zeros(1, 3, 10)
    one = torch.zeros(3, dtype=i32)
    with pytest.raises(ValueError, match="target_probs must be a device tensor"):
        P.oasis_verify_drafts(probs, None, one, None, None, torch.zeros(3), torch.zeros(1), one, one[:1], one, None)
    with pytest.raises(ValueError, match="tokens: 2 elements"):
        P.oasis_verify_drafts(probs, None, one[:2], None, None, torch.zeros(3), torch.zeros(1), one, one[:1], one, None)
    with pytest.raises(ValueError, match="not whole pages|must be a device tensor"):
        P.oasis_append_tokens(d, tk, tk, 3, None, None, pages[:, :, :3].contiguous(), pages[:, :, :3].contiguous(), table,
                              ctx, None)
