"""Attention over the 4-bit cache on values at the ends of their range: NaN in the cache, infinities and NaN in the tree's
rows, the largest finite values, wild queries under a scale of 0; in every form of the kernel, in one split and several."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from oracle import q4 as Q
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import INF, NAN, _check, _inputs
from tests.test_gpu_q4 import dev_u8
from workloads import random_bf16

pytestmark = pytest.mark.gpu

H, L = 2, 300
# G, T, B, blocks of the table past the context, selected blocks: one and two row tiles a wave for itself, one and two of
# the form that shares a unit (not every place with two, and every one), each in one split and in several, and over a selection
FORMS = [(4, 3, 16, 0, 0), (4, 3, 32, 3000, 0), (4, 6, 16, 3000, 0), (4, 6, 32, 0, 0), (4, 13, 16, 0, 0), (4, 13, 32, 3000, 0),
         (8, 12, 16, 6000, 0), (8, 12, 32, 6000, 0), (4, 3, 16, 0, 30), (4, 6, 32, 0, 30), (4, 13, 16, 0, 30), (8, 12, 32, 6000, 2000),
         (8, 16, 16, 6000, 0), (8, 16, 32, 6000, 2000)]


class _Call:
    """One request of L cached tokens; k_pages, v_pages 4-bit pages in order."""

    def __init__(self, form, q, kp, vp, tk=None, tv=None, parent=None, scale=None, length=L):
        G, self.T, self.B, spare, self.k = form
        NB = -(-L // self.B)
        self.q, self.tk, self.tv, self.parent, self.scale, self.length = q, tk, tv, parent, scale, length
        self.kp, self.vp = kp, vp
        self.d = P.dims(1, G * H, H, 128, self.B, NB + spare)
        self.table = np.array([[*range(NB), *[-1] * spare]], np.int32)
        self.sel = self.cnt = None
        if self.k:  # all of them
            n = O.block_counts(length, self.B)[1]
            self.sel = np.full((1, H, self.k), -1, np.int32)
            self.sel[:, :, :n] = np.arange(n)
            self.cnt = np.full((1, H), n, np.int32)

    def run(self):
        ws = torch.full((P.oasis_tree_attn_q4_workspace_bytes(self.d, self.T, self.k),), 255, dtype=torch.uint8, device="cuda")
        note(f"4-bit values T={self.T} B={self.B} k={self.k} workspace={ws.numel()}")
        out, lse = torch.zeros(self.q.shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(self.q.shape[:3], device="cuda")
        P.oasis_tree_attn_q4(self.d, dev_bf16(self.q), self.T, dev_u8(self.kp), dev_u8(self.vp), dev_i32(self.table),
                             dev_i32([self.length]), None if self.sel is None else dev_i32(self.sel),
                             None if self.cnt is None else dev_i32(self.cnt), self.k, None if self.tk is None else dev_bf16(self.tk),
                             None if self.tv is None else dev_bf16(self.tv), None if self.parent is None else dev_i32(self.parent),
                             None, self.scale, out, lse, ws)
        torch.cuda.synchronize()
        return out, lse

    def check(self):
        args = (self.q, Q.read_pages(self.kp, H, self.B), Q.read_pages(self.vp, H, self.B), self.table, [self.length], self.sel,
                self.cnt, self.tk, self.tv, self.parent, [self.T], self.B, self.scale)
        ref, ref_lse = Q.attend(*args)
        ref_abs, _ = Q.attend(*args, magnitude=True)
        out, lse = self.run()
        _check(out, lse, ref, ref_abs, ref_lse, out)


def _pages(seed, B, scale=1.0):
    rng = np.random.default_rng(seed)
    return [Q.make_pages(rng.normal(size=(-(-L // B), H, B, 128)) * s) for s in (1.0, scale)]


def _queries(form, seed, scale=1.0):
    return random_bf16(seed, (1, form[1], form[0] * H, 128), scale=scale)


@pytest.mark.parametrize("form", FORMS)
def test_a_nan_in_the_cache_reaches_what_attends_it(form):
    G, T, B, _, _ = form
    kp, vp = _pages(1, B)
    q = _queries(form, 2)
    base, base_lse = _Call(form, q, kp, vp).run()
    row = np.full(128, 0.5)
    row[40] = np.nan  # dims 32 .. 63 of one token's value, in head 1
    Q.write_token(vp[100 // B], H, B, 1, 100 % B, row)
    out, lse = (x.cpu() for x in _Call(form, q, kp, vp).run())
    out, base = out.view(T, H, G, 128), base.cpu().view(T, H, G, 128)
    assert torch.equal(out[:, 0], base[:, 0]) and torch.equal(lse, base_lse.cpu().view(lse.shape))
    assert torch.isnan(out[:, 1, :, 32:64]).all() and torch.isfinite(out[:, 1, :, :32]).all() and torch.isfinite(out[:, 1, :, 64:]).all()
    row[:] = np.nan  # a key of head 0
    Q.write_token(kp[(L - 1) // B], H, B, 0, (L - 1) % B, row)
    out, lse = (x.cpu() for x in _Call(form, q, kp, vp).run())
    assert torch.isnan(out.view(T, H, G, 128)[:, 0]).all() and torch.isnan(lse.view(T, H, G)[:, 0]).all()
    assert torch.isfinite(lse.view(T, H, G)[:, 1]).all()


@pytest.mark.parametrize("form", FORMS)
def test_tree_rows_off_the_path_have_no_influence(form):
    G, T, B, _, _ = form
    kp, vp = _pages(3, B)
    _, q, tk, tv, parent, _ = _inputs(900 + T, 1, G * H, H, T, "random", None)
    bad = T - 2 if T > 3 else 1
    hit = np.array([bad in p for p in O.tree_paths(parent, [T], T)[0]])
    assert hit.any() and not hit.all()
    tk2, tv2 = tk.copy(), tv.copy()
    tk2[0, bad, 0, 5], tv2[0, bad, 1, 100], tv2[0, bad, 1, 7] = NAN, NAN, INF
    (o0, l0), (o1, l1) = (tuple(x.cpu()[0] for x in _Call(form, q, kp, vp, k, v, parent).run()) for k, v in ((tk, tv), (tk2, tv2)))
    assert torch.equal(o0[~hit], o1[~hit]) and torch.equal(l0[~hit], l1[~hit])
    a, b = o1[hit][:, :G], o1[hit][:, G:]
    assert torch.isnan(a).all()  # a NaN score
    assert torch.isnan(b[..., 100]).all() and torch.all(b[..., 7] == torch.inf)
    keep = [j for j in range(128) if j not in (7, 100)]
    assert torch.equal(b[..., keep], o0[hit][:, G:][..., keep])


# Tables and selections of more than 96 MiB, whose codes are read past the caches: one and two row tiles, few tokens
STREAM = [(4, 3, 16, 24000, 0), (4, 3, 32, 12000, 0), (4, 6, 16, 24000, 0), (4, 6, 32, 12000, 0), (4, 3, 16, 24000, 23500),
          (4, 3, 32, 12000, 11800), (4, 6, 16, 24000, 23500), (4, 6, 32, 12000, 11800)]


@pytest.mark.parametrize("form", STREAM)
def test_loads_past_the_caches(form):
    G, T, B, spare, k = form
    assert H * min(spare, k or spare) * B * 136 >= 96 << 20
    _, q, tk, tv, parent, _ = _inputs(920, 1, G * H, H, T, "random", None)
    _Call(form, q, *_pages(10, B), tk, tv, parent).check()
    _Call(form, q, *_pages(11, B)).check()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("signs", ["same", "mixed"])
def test_the_largest_values(form, signs):
    """All of the cache at +-6 2^125, and in the tree the largest bf16 values: finite means."""
    G, T, B, _, _ = form
    rng = np.random.default_rng(4)
    kp, _ = _pages(5, B)
    shape = (-(-L // B), H, B, 128)
    vp = Q.make_pages(6.0 * 2.0 ** 125 * (np.ones(shape) if signs == "same" else rng.choice([-1.0, 1.0], shape)))
    q = _queries(form, 6)
    _Call(form, q, kp, vp).check()
    _, _, tk, tv, parent, _ = _inputs(910, 1, G * H, H, T, "beam", None)
    tv = np.where(rng.random(tv.shape) < 0.5 if signs == "mixed" else np.zeros(tv.shape, bool), 0xFF7F, 0x7F7F).astype(np.uint16)
    _Call(form, q, kp, vp, tk, tv, parent).check()


@pytest.mark.parametrize("form", FORMS)
def test_peaked_and_flat_scores(form):
    """Logits of some hundreds, whose maximum moves from unit to unit, and logits that are all equal."""
    G, T, B, _, _ = form
    kp, vp = _pages(7, B)
    for page in range(len(kp)):  # keys grow along the context
        for h in range(H):
            for t in range(B):
                Q.write_token(kp[page], H, B, h, t, np.full(128, 0.02 * (page * B + t)) * np.where(np.arange(128) % 2, 1, -1))
    sign = np.where(np.arange(128) % 2, 1.0, -1.0)
    q = np.zeros((1, T, G * H, 128))
    q[:] = sign * np.linspace(-4, 4, T * G * H).reshape(T, G * H)[None, :, :, None]
    q = (q.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    # products of 128 equal terms of up to 24: float32 sums are off by 128 * 2^-24 of 3,072, half an exponent's last bits;
    # the scale brings them to some hundreds
    _Call(form, q, kp, vp, scale=0.002).check()
    _Call(form, np.zeros_like(q), kp, vp).check()


@pytest.mark.parametrize("form", FORMS)
def test_wild_queries_under_a_scale_of_0(form):
    G, T, B, _, _ = form
    kp, vp = _pages(8, B)
    q = _queries(form, 9)
    q[0, T - 1, 0, 17], q[0, 0, G * H - 1, 3] = NAN, INF
    out, lse = (x.cpu()[0] for x in _Call(form, q, kp, vp, scale=0.0).run())
    wild = torch.zeros((T, G * H), dtype=torch.bool)
    wild[T - 1, 0] = wild[0, G * H - 1] = True
    assert torch.isnan(out[wild]).all() and torch.isnan(lse[wild]).all()
    q[0, T - 1, 0, 17] = q[0, 0, G * H - 1, 3] = 0
    want, want_lse = (x.cpu()[0] for x in _Call(form, q, kp, vp, scale=0.0).run())
    assert torch.equal(out[~wild], want[~wild]) and torch.equal(lse[~wild], want_lse[~wild])
    q[0, :, :, 0] = NAN  # nothing attended: nothing to be NaN
    out, lse = (x.cpu() for x in _Call(form, q, kp, vp, scale=0.0, length=0).run())
    assert not host_bits(out).any() and torch.all(lse == -torch.inf)
