"""Tree attention on values at the ends of their range: infinities of negligible weight, the largest finite values, NaN
behind a scale of 0. Against the formula in float64, in every form of the kernels and however the cache is split."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from tests.gpu_util import dev_bf16, dev_i32, note, pool_v_from_htd
from tests.test_gpu_drafts import INF, NAN, _check, _magnitude
from workloads import random_bf16

pytestmark = pytest.mark.gpu

ONE = 0x3F80
BIG = 0x7F7F  # the largest finite value, (2 - 2^-7) 2^127
MINUS = 0x8000

# paged, G, T, B, blocks of the table (or slots) past the context: one and two row tiles of the register form, one and two
# a wave of the form that shares its loads, in one split and in several
FORMS = [(True, 4, 3, 16, 0), (True, 4, 3, 16, 4000), (True, 4, 6, 32, 0), (True, 4, 6, 32, 4000),
         (True, 4, 10, 16, 6000), (True, 8, 12, 16, 6000), (True, 8, 12, 32, 6000),
         (False, 4, 3, 16, 0), (False, 4, 3, 16, 2600), (False, 4, 6, 32, 0), (False, 4, 6, 32, 1300),
         (False, 4, 10, 16, 3600), (False, 8, 12, 16, 2600), (False, 8, 12, 32, 1300)]


class _Call:
    """One request of L cached tokens, two KV heads. Arrays of bf16 bits: q [1][T][Hq][128], pages (of the paged cache,
    in order, or of slots and local block) [NB][2][B][128], the tree's rows [1][T][2][128]."""

    def __init__(self, form, L, q, kp, vp, tk, tv, parent, scale=None):
        self.paged, G, self.T, self.B, spare = form
        self.L, self.q, self.kp, self.vp, self.tk, self.tv, self.parent, self.scale = L, q, kp, vp, tk, tv, parent, scale
        NB = len(kp)
        assert NB == max(1, -(-L // self.B)) and q.shape[2] == 2 * G and len(tk[0]) == self.T
        self.d = P.dims(1, 2 * G, 2, 128, self.B, NB + spare)
        if self.paged:
            self.table = np.array([[*range(NB), *[-1] * spare]], np.int32)
            self.bytes = P.oasis_tree_attn_workspace_bytes(self.d, self.T)
        else:
            self.ks = NB - 1 + spare
            self.map = np.broadcast_to(np.array([*range(NB - 1), *[-1] * spare], np.int32), (1, 2, self.ks)).copy()
            junk = np.full((spare, 2, self.B, 128), NAN, np.uint16)
            self.pk, self.pv = (np.concatenate([x[:-1], junk, x[-1:]])[None] for x in (kp, vp))
            self.bytes = P.oasis_sparse_tree_attn_workspace_bytes(self.d, self.T, self.ks)

    def run(self):
        note(f"values paged={self.paged} T={self.T} B={self.B} L={self.L} workspace={self.bytes}")
        out = torch.zeros(self.q.shape, dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros(self.q.shape[:3], device="cuda")
        ws = torch.zeros(self.bytes, dtype=torch.uint8, device="cuda")
        tree = (dev_i32([self.L]), dev_bf16(self.tk), dev_bf16(self.tv), dev_i32(self.parent), None, self.scale, out, lse, ws)
        if self.paged:
            P.oasis_tree_attn(self.d, dev_bf16(self.q), self.T, dev_bf16(self.kp), dev_bf16(self.vp), dev_i32(self.table),
                              *tree)
        else:
            P.oasis_sparse_tree_attn(self.d, dev_bf16(self.q), self.T, dev_bf16(self.pk), dev_bf16(pool_v_from_htd(self.pv)),
                                     dev_i32(self.map) if self.ks else None, self.ks, *tree)
        torch.cuda.synchronize()
        return out, lse

    def reference(self, values=lambda x: x):
        tree = (self.tk, values(self.tv), self.parent, [self.T])
        if self.paged:
            return O.tree_attend(self.q, self.kp, values(self.vp), self.table, [self.L], *tree, self.B, self.scale)
        return O.sparse_tree_attend(self.q, self.pk, values(self.pv), self.map, [self.L], *tree, self.B, self.scale)

    def check(self):
        out, lse = self.run()
        ref, ref_lse = self.reference()
        _check(out, lse, ref, self.reference(_magnitude)[0], ref_lse, out)
        return out


def _random(form, L, seed):
    _, G, T, B, _ = form
    NB = max(1, -(-L // B))
    rng = np.random.default_rng(seed)
    return dict(q=random_bf16(seed + 1, (1, T, 2 * G, 128)), kp=random_bf16(seed + 2, (NB, 2, B, 128)),
                vp=random_bf16(seed + 3, (NB, 2, B, 128)), tk=random_bf16(seed + 4, (1, T, 2, 128)),
                tv=random_bf16(seed + 5, (1, T, 2, 128)),
                parent=np.maximum(np.arange(T) - rng.integers(1, 3, (1, T)), -1).astype(np.int32))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("tree_above", [False, True])
def test_infinite_tree_values_of_negligible_weight(form, tree_above):
    """The tree's logits 260 (base 2) below the cache's, or above: a positive weight, however small, times an infinity is
    one, a NaN stays one, and the rows that do not attend them are what they are without, in one split and in several."""
    x = _random(form, 60, 4000)
    T = form[2]
    x["q"][:] = 0x4080  # 4, and 4 * 4 * 128 / sqrt(128) = 181 nats
    x["kp"][:], x["tk"][:] = (0, 0x4080) if tree_above else (0x4080, 0)
    x["parent"] = np.array([[-1, *[0] * (T - 1)]], np.int32)
    clean = _Call(form, 60, **x).check()
    x["tv"][0, 1, 0, 5], x["tv"][0, 1, 1, 7], x["tv"][0, 1, 1, 8] = INF, INF | MINUS, NAN
    out, _ = _Call(form, 60, **x).run()
    G = form[1]
    want = clean.clone()
    want[0, 1, :G, 5], want[0, 1, G:, 7], want[0, 1, G:, 8] = float("inf"), -float("inf"), float("nan")
    assert torch.equal(torch.nan_to_num(out, 77.0), torch.nan_to_num(want, 77.0))


def test_opposite_infinities_in_one_path():
    for form in FORMS[:2] + FORMS[5:6]:
        x = _random(form, 60, 4100)
        x["q"][:], x["kp"][:], x["tk"][:] = 0x4080, 0x4080, 0
        x["parent"] = (np.arange(form[2]) - 1)[None].astype(np.int32)
        x["tv"][0, 1, :, 5], x["tv"][0, 2, :, 5] = INF, INF | MINUS
        o = _Call(form, 60, **x).run()[0][0, :, :, 5]
        assert torch.isfinite(o[0]).all() and (o[1] == torch.inf).all() and torch.isnan(o[2:]).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("L", [0, 1, 47, 2500])
def test_largest_values(form, L):
    """A mean of finite values is finite: values of the largest magnitude, of one sign and of both."""
    for signs in (False, True):
        x = _random(form, L, 4200 + L)
        for v in ("vp", "tv"):
            x[v][:] = BIG | (x[v] & MINUS if signs else 0)
        _Call(form, L, **x).check()


@pytest.mark.parametrize("form", FORMS)
def test_largest_values_behind_rising_logits(form):
    """Logits that rise by less than moves a row's reference, from unit to unit: the sums are at their largest."""
    x = _random(form, 2500, 4300)
    B, rise = form[3], np.arange(len(x["kp"]) * form[3]) // 32
    x["q"][:], x["kp"][:] = 0, 0
    x["q"][..., 0] = ONE
    # 128 / sqrt(128) nats a step of 1 in q k; bf16 steps of the key's one entry
    steps = torch.tensor(np.minimum(rise * 0.75, 48.0), dtype=torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    x["kp"][..., 0] = steps.reshape(-1, B)[:, None, :]
    x["vp"][:], x["tv"][:] = BIG, BIG
    _Call(form, 2500, **x).check()


@pytest.mark.parametrize("form", FORMS)
def test_small_values(form):
    """Values of 2^-80: a sum whose terms are scaled down by some 2^20 keeps them."""
    x = _random(form, 2500, 4400)
    for v in ("vp", "tv"):
        x[v][:] = (x[v] & np.uint16(0x807F)) | np.uint16((127 - 80) << 7)
    c = _Call(form, 2500, **x)
    out, lse = c.run()
    ref, ref_lse = c.reference()
    up = 2.0 ** 80  # compared at the size that the tolerances are made for
    _check((out.float() * up).bfloat16(), lse, ref * up, c.reference(_magnitude)[0] * up, ref_lse, out)


@pytest.mark.parametrize("form", FORMS)
def test_a_scale_of_zero_keeps_nan(form):
    """0 times a NaN or an infinity in q is a NaN score of every token; the other rows weigh all tokens alike."""
    x = _random(form, 60, 4500)
    x["q"][0, 1, 0, 3], x["q"][0, 2, 1, 4], x["q"][0, 0, -1, 127] = NAN, INF, INF | MINUS
    c = _Call(form, 60, **x, scale=0.0)
    out, lse = c.run()
    bad = torch.zeros(out.shape[:3], dtype=torch.bool)
    bad[0, 1, 0] = bad[0, 2, 1] = bad[0, 0, -1] = True
    assert torch.isnan(out.cpu()[bad]).all() and torch.isnan(lse.cpu()[bad]).all()
    with np.errstate(invalid="ignore"):
        ref, ref_lse = c.reference()
        ref_abs = c.reference(_magnitude)[0]
    good = ~bad.numpy()
    assert np.isfinite(ref_lse[good]).all()
    _check(out.cpu()[torch.from_numpy(good)], lse.cpu()[torch.from_numpy(good)], ref[good], ref_abs[good], ref_lse[good],
           out.cpu()[torch.from_numpy(good)])
