"""The speculative step through ``DecodePath``: prediction and staging, attention of the drafted tree over the working
set and over every cached token, verification, and the commit of what was accepted, against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from paper_2608_08097_amd.path import DecodePath
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note, selection_diff
from tests.test_gpu_drafts import _check, _magnitude
from workloads import random_bf16

pytestmark = pytest.mark.gpu

R, HQ, H, T, B, K, V = 3, 8, 2, 6, 16, 6, 40
STEPS = 10


class _Run:
    def __init__(self, local):
        rng = np.random.default_rng(77)
        self.ctx = np.array([7, 105, 390], np.int32)
        self.NB = (int(self.ctx.max()) + STEPS * T + B - 1) // B + 1
        n = R * self.NB
        self.table = rng.permutation(n).reshape(R, self.NB).astype(np.int32)
        self.kp, self.vp = random_bf16(70, (n, H, B, 128)), random_bf16(71, (n, H, B, 128))
        self.parent = np.broadcast_to(np.array([-1, 0, 0, 1, 1, 3], np.int32), (R, T)).copy()
        self.steps = [dict(q=random_bf16(720 + i, (R, T, HQ, 128), scale=1.5), k=random_bf16(740 + i, (R, T, H, 128)),
                           v=random_bf16(760 + i, (R, T, H, 128)), tokens=rng.integers(0, 4, (R, T)).astype(np.int32),
                           ua=rng.random((R, T), dtype=np.float32), us=rng.random(R, dtype=np.float32),
                           n=rng.integers(1, T + 1, R).astype(np.int32)) for i in range(STEPS)]
        pin = lambda x: dev_bf16(x, "cpu").pin_memory()  # noqa: E731
        self.hk, self.hv = pin(self.kp), pin(self.vp)
        self.d = P.dims(R, HQ, H, 128, B, self.NB)
        self.path = DecodePath(self.d, T, K, self.hk, self.hv, dev_i32(self.table), first_draft=1, fetch_cap=4)
        if local:
            self.own = rng.permutation(n).reshape(R, self.NB).astype(np.int32)
            self.lk, self.lv = (torch.zeros((n, H, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            for r in range(R):
                self.lk[self.own[r].tolist()] = self.hk[self.table[r].tolist()].cuda()
                self.lv[self.own[r].tolist()] = self.hv[self.table[r].tolist()].cuda()
            self.path.set_local_source(self.lk, self.lv, dev_i32(self.own))
        self.st = self.path.new_layer()
        self.len = [dev_i32(self.ctx), torch.zeros(R, dtype=torch.int32, device="cuda")]
        f32 = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        self.dev = [dict(q=dev_bf16(s["q"]), k=dev_bf16(s["k"]), v=dev_bf16(s["v"]), tokens=dev_i32(s["tokens"]),
                         ua=f32(s["ua"]), us=f32(s["us"]), n=dev_i32(s["n"])) for s in self.steps]
        self.dparent = dev_i32(self.parent)
        self.head = torch.from_numpy((rng.standard_normal((HQ * 128, V)) * 0.3).astype(np.float32)).cuda()
        self.probs = torch.zeros((R, T, V), device="cuda")

    def start(self):
        ctx = self.len[0]
        self.path.build_summaries(self.st, ctx)
        self.path.predict(self.st, self.dev[0]["q"], ctx)
        self.path.stage(self.st, ctx, 0, fetch_cap=K)

    def forward(self, i, dense=False):
        s, ctx = self.dev[i], self.len[i % 2]
        (self.path.attend_tree_dense if dense else self.path.attend_tree)(
            self.st, s["q"], ctx, s["k"], s["v"], self.dparent, s["n"])

    def finish(self, i):
        s = self.dev[i]
        rows = torch.arange(T, device="cuda")[None, :, None, None] < s["n"][:, None, None, None]
        logits = torch.where(rows, self.st.out.float(), 0.0).view(R * T, -1) @ self.head
        logits[:, :4] += 7.0  # a few likely tokens, which the drafts are taken from
        self.probs.copy_(torch.softmax(logits, -1).view(R, T, V))
        self.got = self.path.verify(self.probs, None, s["tokens"], s["ua"], s["us"], self.dparent, s["n"])
        self.path.commit(self.st, s["k"], s["v"], *self.got[:2], self.len[i % 2], self.len[(i + 1) % 2])
        self.path.predict(self.st, s["q"], self.len[(i + 1) % 2])
        self.path.stage(self.st, self.len[(i + 1) % 2], i % 2 + 1, copy_local=False)


@pytest.mark.parametrize("local", [False, True])
def test_the_speculative_step_of_a_path(local):
    m = _Run(local)
    ctx = m.ctx.copy()
    note(f"speculative path local={local}")
    m.start()
    kmax, kmin = O.block_summaries(m.kp, m.table, ctx, B, m.NB)
    grown = 0
    for i, s in enumerate(m.steps):
        note(f"speculative path step {i}")
        m.st.out.fill_(3.0)
        before = m.st.out.clone()
        m.forward(i, dense=True)
        torch.cuda.synchronize()
        tree = (s["k"], s["v"], m.parent, s["n"])
        ref, ref_lse = O.tree_attend(s["q"], m.kp, m.vp, m.table, ctx, *tree, B)
        mag = (s["k"], _magnitude(s["v"]), m.parent, s["n"])
        ref_abs, _ = O.tree_attend(s["q"], m.kp, _magnitude(m.vp), m.table, ctx, *mag, B)
        _check(m.st.out, m.st.lse, ref, ref_abs, ref_lse, before)

        m.forward(i)
        torch.cuda.synchronize()
        # the working set from the tier itself: what is staged and the local block are the context as committed
        smap = m.st.slot_map.cpu().numpy()
        pk, pv = (np.zeros((R, K + 1, H, B, 128), np.uint16) for _ in range(2))
        for r in range(R):
            nb, cand, _ = O.block_counts(ctx[r], B)
            assert (smap[r] < cand).all()
            for h in range(H):
                for slot, b in [*enumerate(smap[r, h]), (K, nb - 1)]:
                    if b >= 0:
                        pk[r, slot, h], pv[r, slot, h] = m.kp[m.table[r, b], h], m.vp[m.table[r, b], h]
        ref, ref_lse = O.sparse_tree_attend(s["q"], pk, pv, smap, ctx, *tree, B)
        ref_abs, _ = O.sparse_tree_attend(s["q"], pk, _magnitude(pv), smap, ctx, *mag, B)
        _check(m.st.out, m.st.lse, ref, ref_abs, ref_lse, before)

        m.finish(i)
        torch.cuda.synchronize()
        want = O.verify_drafts(m.probs.cpu().numpy(), None, s["tokens"], m.parent, s["n"], s["ua"], s["us"])
        for x, y in zip(m.got, want):
            assert np.array_equal(x.cpu().numpy(), y)
        prev = ctx
        ctx = O.append_tokens(s["k"], s["v"], want[0], want[1], m.kp, m.vp, m.table, ctx, B)
        assert np.array_equal(m.len[(i + 1) % 2].cpu().numpy(), ctx)
        assert np.array_equal(host_bits(m.hk), m.kp) and np.array_equal(host_bits(m.hv), m.vp)
        O.update_summaries(m.kp, m.table, prev, ctx, B, kmax, kmin, T)
        ok = ~np.isnan(kmax)
        assert np.array_equal(O.bf16_to_f64(host_bits(m.st.kmax))[ok], kmax[ok])
        assert np.array_equal(O.bf16_to_f64(host_bits(m.st.kmin))[ok], kmin[ok])
        sc = O.block_scores(s["q"], kmax, kmin, ctx, H, B)
        sel, cnt = O.select_topk(sc, ctx, K, B)
        assert not selection_diff(m.st.sel.cpu().numpy(), m.st.sel_count.cpu().numpy(), sel, cnt, sc)
        grown = max(grown, int(want[1].max()))
    assert grown > 1 and (ctx // B > m.ctx // B).all()


def test_the_path_step_captured_and_replayed():
    """Two steps in a graph, replayed between eager work, against the same steps eager; the first call of a path is not
    taken into a capture."""
    m = _Run(False)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    note("a first call under capture")
    with pytest.raises(RuntimeError, match="must not be captured"):
        with torch.cuda.graph(graph, stream=side):
            m.forward(0)
    torch.cuda.synchronize()
    want = []
    m.start()
    for i in range(STEPS):
        m.forward(i)
        m.finish(i)
        torch.cuda.synchronize()
        want.append([x.clone() for x in (m.st.out, m.st.lse, *m.got, m.len[(i + 1) % 2])])

    a = _Run(False)
    a.path._speculative()
    a.start()
    feed = [{n: t.clone() for n, t in a.dev[i].items()} for i in range(2)]
    dev, a.dev = a.dev, feed
    keep = [[torch.empty_like(t) for t in want[0]] for _ in range(2)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for i in range(2):
            a.forward(i)
            a.finish(i)
            for x, y in zip(keep[i], (a.st.out, a.st.lse, *a.got, a.len[(i + 1) % 2])):
                x.copy_(y)
    for pair in range(STEPS // 2):
        for i in range(2):
            for n, t in dev[2 * pair + i].items():
                feed[i][n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        torch.ones(1000, device="cuda").cumsum(0)  # eager work in between
        for i in range(2):
            n = want[2 * pair + i]
            used = torch.arange(T, device="cuda")[None] < dev[2 * pair + i]["n"][:, None]
            for x, y in zip(keep[i][:2], n[:2]):
                assert torch.equal(x[used], y[used]), (pair, i)
            for x, y in zip(keep[i][2:], n[2:]):
                assert torch.equal(x, y), (pair, i)
    assert np.array_equal(host_bits(a.hk), host_bits(m.hk)) and np.array_equal(host_bits(a.hv), host_bits(m.hv))
