"""Calls of the 4-bit cache that its entry points refuse, before anything is launched (CPU only)."""
import ctypes

import pytest
import torch

import paper_2608_08097_amd as P

R, T, HQ, H, B, NB, PAGES = 3, 4, 8, 2, 16, 64, 10
PAGE = H * B * 68
K = 60  # selected blocks: several splits
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4


def _at(byte):
    return None if byte is None else ctypes.c_void_p(byte)  # aligned stand-ins, never dereferenced


def _rotary(dim=64, interleaved=0, amplitude=1.0, turns=1 << 12):
    return P.OasisRotary(turns, dim, interleaved, amplitude)


def _d(**kw):
    a = dict(num_reqs=R, num_q_heads=HQ, num_kv_heads=H, head_dim=128, block_size=B, max_blocks=NB)
    return P.dims(**{**a, **kw})


M = 1 << 20
ROWS = R * T * H * 256
ROTATE = dict(positions=1 << 13, ctx_len=1 << 14, q=M, q_out=2 * M, k=3 * M, k_out=4 * M)


def rotate(d=None, rot=None, tokens=T, qs=HQ * 128, qos=HQ * 128, ks=H * 128, kos=H * 128, **at):
    a = {n: _at(x) for n, x in {**ROTATE, **at}.items()}
    d, rot = d or _d(), _rotary() if rot is None else rot
    st = P.lib().oasis_rotate(ctypes.byref(d), ctypes.byref(rot) if rot else None, tokens, a["positions"], a["ctx_len"], 0, a["q"],
                              qs, a["q_out"], qos, a["k"], ks, a["k_out"], kos, None)
    return st, P.oasis_last_error()


APPEND = dict(new_k=M, new_v=2 * M, path=1 << 13, path_len=1 << 14, k_pages=3 * M, v_pages=4 * M, block_table=1 << 15,
              ctx_len=1 << 16, new_ctx_len=1 << 17, read_k=5 * M, read_v=6 * M)


def append(d=None, rot=None, tokens=T, ks=H * 128, vs=H * 128, pages=PAGES, **at):
    a = {n: _at(x) for n, x in {**APPEND, **at}.items()}
    d = d or _d()
    st = P.lib().oasis_append_tokens_q4(ctypes.byref(d), ctypes.byref(rot) if rot else None, a["new_k"], ks, a["new_v"], vs, tokens,
                                        a["path"], a["path_len"], a["k_pages"], a["v_pages"], pages, a["block_table"],
                                        a["ctx_len"], a["new_ctx_len"], a["read_k"], a["read_v"], None)
    return st, P.oasis_last_error()


SUMMARY = dict(k_pages=M, block_table=1 << 13, prev_ctx_len=1 << 14, ctx_len=1 << 15, kmax=2 * M, kmin=4 * M)


def summary(d=None, pages=PAGES, most=1, **at):
    a = {n: _at(x) for n, x in {**SUMMARY, **at}.items()}
    d = d or _d()
    st = P.lib().oasis_update_summaries_q4(ctypes.byref(d), a["k_pages"], pages, a["block_table"], a["prev_ctx_len"],
                                           a["ctx_len"], most, a["kmax"], a["kmin"], None)
    return st, P.oasis_last_error()


ATTN = dict(q=M, k_pages=2 * M, v_pages=3 * M, block_table=1 << 13, ctx_len=1 << 14, sel=1 << 15, sel_count=1 << 16,
            tree_k=4 * M, tree_v=5 * M, parent=1 << 17, tree_len=1 << 18, out=6 * M, lse=7 * M, workspace=64 * M)


def attn(d=None, tokens=T, k=K, pages=PAGES, scale=0.1, ws=1 << 40, **at):
    a = {n: _at(x) for n, x in {**ATTN, **at}.items()}
    d = d or _d()
    st = P.lib().oasis_tree_attn_q4(ctypes.byref(d), a["q"], tokens, a["k_pages"], a["v_pages"], pages, a["block_table"],
                                    a["ctx_len"], a["sel"], a["sel_count"], k, a["tree_k"], a["tree_v"], a["parent"],
                                    a["tree_len"], scale, a["out"], a["lse"], a["workspace"], ws, None)
    return st, P.oasis_last_error()


CALLS = {rotate: ROTATE, append: APPEND, summary: SUMMARY, attn: ATTN}


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__)
def test_dims(call):
    for kw, want in ((dict(num_reqs=-1), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(block_size=8), UNSUPPORTED),
                     (dict(num_q_heads=7), INVALID), (dict(num_kv_heads=0), INVALID), (dict(max_blocks=0), INVALID),
                     (dict(num_reqs=40000), UNSUPPORTED)):
        st, error = call(_d(**kw))
        assert st == want and error, (kw, st, error)
    st, error = call(_d(num_reqs=0), **{n: None for n in CALLS[call]}, **({"k": 0} if call is attn else {}))
    assert st == 0 and error == ""


NULLABLE = {rotate: ["ctx_len"], append: ["path", "new_ctx_len", "read_k", "read_v"],
            summary: ["prev_ctx_len"], attn: ["parent", "tree_len", "lse"]}


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__)
def test_missing_and_misaligned_pointers(call):
    for n in CALLS[call]:
        if n in NULLABLE[call] or (call is rotate and n == "positions"):
            continue
        if call is rotate and n in ("q", "k"):
            assert rotate(q=None, q_out=None, k=None, k_out=None)[0] == INVALID
            continue
        if n == "path_len":
            st, error = call(path_len=None)
            assert st == INVALID and "path" in error
            continue
        st, error = call(**{n: None})
        assert st == (WORKSPACE if n == "workspace" else INVALID), (n, st, error)
    assert rotate(positions=None, ctx_len=None)[0] == INVALID
    for n in ("q", "q_out", "k", "k_out", "new_k", "new_v", "k_pages", "v_pages", "read_k", "read_v", "kmax", "kmin", "tree_k",
              "tree_v", "out", "workspace"):
        if n in CALLS[call]:
            st, error = call(**{n: CALLS[call][n] + 8})
            assert st == INVALID and "aligned" in error and n in error, (n, error)


def test_rotations():
    for call, kw in ((rotate, {}), (append, {})):
        for rot in (_rotary(0), _rotary(1), _rotary(65), _rotary(130), _rotary(-2), _rotary(interleaved=2),
                    _rotary(amplitude=float("nan")), _rotary(amplitude=float("inf")), _rotary(turns=None), _rotary(turns=4100)):
            st, error = call(rot=rot, **kw)
            assert st == INVALID and error, (call, rot)
    assert rotate(rot=False)[0] == INVALID


def test_rotate_more_rows_than_a_launch_has_threads_for():
    for d, tokens in ((_d(), (1 << 24) // R + 1), (_d(num_reqs=1), (1 << 24) + 1), (_d(num_reqs=1), 1 << 25)):
        st, error = rotate(d, tokens=tokens)
        assert st == UNSUPPORTED and "rows" in error, tokens


def test_strides():
    for bad in (HQ * 128 - 8, HQ * 128 + 4, 0, -HQ * 128, 1 << 62):
        for n in ("qs", "qos"):
            st, error = rotate(**{n: bad})
            assert st == INVALID and "elements apart" in error, (n, bad)
    for n in ("ks", "vs"):
        for bad in (H * 128 - 8, H * 128 + 2, 0, 1 << 62):
            st, error = append(**{n: bad})
            assert st == INVALID and "elements apart" in error, (n, bad)


def test_sizes():
    assert rotate(tokens=0)[0] == INVALID and append(tokens=0)[0] == INVALID and attn(tokens=0)[0] == INVALID
    assert rotate(tokens=1 << 30)[0] == UNSUPPORTED
    assert append(tokens=1 << 26)[0] == UNSUPPORTED
    assert attn(tokens=65)[0] == UNSUPPORTED
    assert attn(_d(num_q_heads=2 * 1025), tokens=4)[0] == UNSUPPORTED  # 4,100 rows
    for call in (append, summary, attn):
        assert call(pages=0)[0] == INVALID and call(pages=1 << 31)[0] == INVALID
        assert call(_d(max_blocks=(1 << 27)))[0] == UNSUPPORTED  # tokens past 31 bits
    assert summary(most=0)[0] == INVALID
    assert attn(k=-1)[0] == INVALID and attn(k=65537)[0] == UNSUPPORTED
    for kw in (dict(k=0), dict(sel=None), dict(sel_count=None), dict(sel=None, sel_count=None),
               dict(sel=None, sel_count=None, k=K), dict(sel=None, k=0)):
        st, error = attn(**kw)
        assert st == INVALID and "go together" in error, kw
    for scale in (float("nan"), float("inf"), 3e38):
        assert attn(scale=scale)[0] == INVALID
    for kw in (dict(tree_k=None), dict(tree_v=None)):  # both or none
        assert attn(**kw)[0] == INVALID
    need = P.oasis_tree_attn_q4_workspace_bytes(_d(), T, K)
    assert need > 0 and attn(ws=need - 1)[0] == WORKSPACE
    assert P.oasis_tree_attn_q4_workspace_bytes(_d(), 0, K) == P.oasis_tree_attn_q4_workspace_bytes(_d(), T, -1) == 0
    assert P.oasis_tree_attn_q4_workspace_bytes(_d(head_dim=64), T, K) == 0 == P.oasis_q4_page_bytes(_d(head_dim=64))


def test_rows_that_overlap():
    q, k = R * T * HQ * 256, R * T * H * 256
    for kw in (dict(q_out=M + 16), dict(q_out=M + q - 16), dict(q_out=M, qos=HQ * 128 + 8), dict(k_out=3 * M + 256),
               dict(q_out=3 * M + 256), dict(k_out=M + 256), dict(k_out=2 * M + q - 16), dict(q_out=(1 << 13)),
               dict(rot=_rotary(turns=9 * M), k_out=9 * M - k + 16)):
        st, error = rotate(**kw)
        assert st == INVALID and "overlaps" in error, (kw, error)
    # of one joint projection: side by side is fine (no refusal of the rows, but of the turns, which they hold), shifted is not
    joint, turns = (HQ + 2 * H) * 128, _rotary(turns=M + 64)
    in_place = dict(qs=joint, qos=joint, ks=joint, kos=joint, q=M, q_out=M, k=M + HQ * 256, k_out=M + HQ * 256)
    st, error = rotate(rot=turns, **in_place)
    assert st == INVALID and "overlaps turns" in error
    for kw in (dict(k_out=M + HQ * 256 - 256), dict(k_out=M + (HQ + 2 * H) * 256 - 256), dict(kos=joint + 8)):
        st, error = rotate(**{**in_place, **kw})
        assert st == INVALID and "overlaps" in error and "turns" not in error, (kw, error)


SIZES = {append: dict(new_k=ROWS, new_v=ROWS, path=4 * R * T, path_len=4 * R, k_pages=PAGES * PAGE, v_pages=PAGES * PAGE,
                      block_table=4 * R * NB, ctx_len=4 * R, new_ctx_len=4 * R, read_k=ROWS, read_v=ROWS),
         summary: dict(k_pages=PAGES * PAGE, block_table=4 * R * NB, prev_ctx_len=4 * R, ctx_len=4 * R, kmax=R * H * NB * 256,
                       kmin=R * H * NB * 256),
         attn: dict(q=R * T * HQ * 256, k_pages=PAGES * PAGE, v_pages=PAGES * PAGE, block_table=4 * R * NB, ctx_len=4 * R,
                    sel=4 * R * H * K, sel_count=4 * R * H, tree_k=ROWS, tree_v=ROWS, parent=4 * R * T, tree_len=4 * R,
                    out=R * T * HQ * 256, lse=4 * R * T * HQ, workspace=None)}
WRITTEN = {append: ["k_pages", "v_pages", "new_ctx_len", "read_k", "read_v"], summary: ["kmax", "kmin"],
           attn: ["out", "lse", "workspace"]}


@pytest.mark.parametrize("call", SIZES, ids=lambda c: c.__name__)
def test_buffers_that_overlap(call):
    sizes = dict(SIZES[call])
    if call is attn:
        sizes["workspace"] = P.oasis_tree_attn_q4_workspace_bytes(_d(), T, K)
    for out in WRITTEN[call]:
        for other, size in sizes.items():
            if other == out:
                continue
            first = CALLS[call][other]
            for at in (first, first + (size - 1) // 16 * 16, max(16, first - (sizes[out] - 1) // 16 * 16)):
                st, error = call(**{out: at})
                assert st == INVALID and "overlaps" in error and out in error, (out, other, at, st, error)


def test_the_binding():
    d = _d()
    dev = torch.zeros(4)
    with pytest.raises(ValueError, match="go together"):
        P.oasis_rotate(d, P.Rotary(64, device="cpu"), T, None, torch.zeros(R, dtype=torch.int32), dev, None, None, None)
    with pytest.raises(ValueError, match="q must be a device tensor"):
        P.oasis_rotate(d, P.Rotary(64, device="cpu"), T, None, torch.zeros(R, dtype=torch.int32),
                       torch.zeros(R, T, HQ, 128, dtype=torch.bfloat16), torch.zeros(R, T, HQ, 128, dtype=torch.bfloat16), None, None)
    pages = torch.zeros(PAGES, PAGE, dtype=torch.uint8)
    with pytest.raises(ValueError, match="differ in shape"):
        P.oasis_append_tokens_q4(d, None, dev, dev, T, None, None, pages, pages[:3], dev, dev, None)
    with pytest.raises(ValueError, match="not whole pages|elements"):
        P.oasis_update_summaries_q4(d, pages[:, :-1], torch.zeros(R, NB, dtype=torch.int32), None,
                                    torch.zeros(R, dtype=torch.int32), 1, dev, dev)
    with pytest.raises(ValueError, match="sel: "):
        P.oasis_tree_attn_q4(d, torch.zeros(R, T, HQ, 128, dtype=torch.bfloat16), T, pages, pages,
                             torch.zeros(R, NB, dtype=torch.int32), torch.zeros(R, dtype=torch.int32),
                             torch.zeros(5, dtype=torch.int32), None, 8, None, None, None, None, None,
                             torch.zeros(R, T, HQ, 128, dtype=torch.bfloat16), None, None)
