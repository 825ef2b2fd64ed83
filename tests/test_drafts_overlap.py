"""Buffers that a call of the speculative step both reads and writes are refused: its waves read them at times of their
own, so that some would see what others have written."""
import ctypes

import pytest

import paper_2608_08097_amd as P

R, T, V, NB = 3, 4, 100, 64


def _at(byte):
    return None if byte is None else ctypes.c_void_p(byte)  # aligned stand-ins, never dereferenced


VERIFY = dict(target=1 << 20, draft=2 << 20, tokens=4096, parent=8192, tree_len=12288, accept_u=16384, sample_u=20480,
              path=24576, path_len=28672, out_tokens=32768, workspace=3 << 20)


def _verify(**at):
    a = {n: _at(x) for n, x in {**VERIFY, **at}.items()}
    st = P.lib().oasis_verify_drafts(R, T, V, a["target"], V, a["draft"], V, a["tokens"], a["parent"], a["tree_len"],
                                     a["accept_u"], a["sample_u"], a["path"], a["path_len"], a["out_tokens"], a["workspace"],
                                     1 << 30, None)
    return st, P.oasis_last_error()


APPEND = dict(new_k=1 << 20, new_v=2 << 20, path=4096, path_len=8192, k=3 << 20, v=4 << 20, block_table=12288,
              ctx_len=16384, new_ctx_len=20480)


def _append(**at):
    a = {n: _at(x) for n, x in {**APPEND, **at}.items()}
    d = P.dims(R, 8, 2, 128, 16, NB)
    st = P.lib().oasis_append_tokens(ctypes.byref(d), a["new_k"], a["new_v"], T, a["path"], a["path_len"], a["k"], a["v"], 10,
                                     a["block_table"], a["ctx_len"], a["new_ctx_len"], None)
    return st, P.oasis_last_error()


@pytest.mark.parametrize("out", ["path", "path_len", "out_tokens"])
@pytest.mark.parametrize("other", ["tokens", "parent", "tree_len", "accept_u", "sample_u", "workspace", "path", "path_len",
                                   "out_tokens"])
def test_verification(out, other):
    if out == other:
        return
    n = {"path_len": 4 * R, "tree_len": 4 * R, "sample_u": 4 * R, "workspace": 4096}
    for first in (VERIFY[other], VERIFY[other] + n.get(other, 4 * R * T) - 4, VERIFY[other] - n.get(out, 4 * R * T) + 4):
        st, error = _verify(**{out: first})
        assert st == 1 and "overlaps" in error and out in error and other in error, (first, error)


@pytest.mark.parametrize("other,size", [("path", 4 * R * T), ("path_len", 4 * R), ("block_table", 4 * R * NB),
                                        ("ctx_len", 4 * R)])
def test_append(other, size):
    for first in (APPEND[other] + 4, APPEND[other] + size - 4, APPEND[other] - 4 * R + 4):
        st, error = _append(new_ctx_len=first)
        assert st == 1 and f"new_ctx_len overlaps {other}" in error, (first, error)
