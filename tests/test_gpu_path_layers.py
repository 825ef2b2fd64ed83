"""Several layers on one ``DecodePath``, each on pages of its own: commits, staging, dense and sparse attention of one
layer are not touched by the others', against the float64 oracle; and the pipelined schedule over such layers."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from paper_2608_08097_amd.path import DecodePath
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import _check, _magnitude
from workloads import random_bf16

pytestmark = pytest.mark.gpu

R, HQ, H, T, B, K, NB = 2, 8, 2, 5, 16, 4, 20
CTX = np.array([45, 222], np.int32)
LAYERS, STEPS = 2, 4


def _pin(x):
    return dev_bf16(x, "cpu").pin_memory()


class _Layer:
    """One layer's pages, and its inputs of every step."""

    def __init__(self, i, path, table, local):
        n = R * NB
        self.kp, self.vp = random_bf16(80 + 10 * i, (n, H, B, 128)), random_bf16(81 + 10 * i, (n, H, B, 128))
        self.hk, self.hv = _pin(self.kp), _pin(self.vp)
        self.source = None
        if local:  # the same pages on the device, at other places
            own = np.random.default_rng(i).permutation(n).reshape(R, NB).astype(np.int32)
            lk, lv = (torch.zeros((n, H, B, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            for r in range(R):
                lk[own[r].tolist()] = self.hk[table[r].tolist()].cuda()
                lv[own[r].tolist()] = self.hv[table[r].tolist()].cuda()
            self.source = (lk, lv, dev_i32(own))
        self.st = path.new_layer(self.hk, self.hv, self.source)
        s = 1000 * (i + 1)
        self.q = [random_bf16(s + t, (R, T, HQ, 128), scale=1.5) for t in range(STEPS + 1)]
        self.k = [random_bf16(s + 100 + t, (R, T, H, 128)) for t in range(STEPS + 1)]
        self.v = [random_bf16(s + 200 + t, (R, T, H, 128)) for t in range(STEPS + 1)]

    def staged(self, table, ctx):
        """The working set as the layer's slot map names it, from its own pages."""
        smap = self.st.slot_map.cpu().numpy()
        pk, pv = (np.zeros((R, K + 1, H, B, 128), np.uint16) for _ in range(2))
        for r in range(R):
            nb = O.block_counts(ctx[r], B)[0]
            for h in range(H):
                for slot, b in [*enumerate(smap[r, h]), (K, nb - 1)]:
                    if b >= 0:
                        pk[r, slot, h], pv[r, slot, h] = self.kp[table[r, b], h], self.vp[table[r, b], h]
        return pk, pv, smap


def _path(table, **kw):
    unused = [torch.full((1, H, B, 128), float("nan"), dtype=torch.bfloat16).pin_memory() for _ in range(2)]
    d = P.dims(R, HQ, H, 128, B, NB)
    return DecodePath(d, T, K, *unused, dev_i32(table), first_draft=1, fetch_cap=K, **kw)


@pytest.mark.parametrize("local", [False, True])
def test_commits_of_layers_on_their_own_pages(local):
    rng = np.random.default_rng(5)
    table = rng.permutation(R * NB).reshape(R, NB).astype(np.int32)
    path = _path(table)
    layers = [_Layer(i, path, table, local) for i in range(LAYERS)]
    parent = np.broadcast_to(np.array([-1, 0, 0, 1, 2], np.int32), (R, T)).copy()
    lens, ctx = [dev_i32(CTX), dev_i32(CTX)], CTX.copy()
    dparent = dev_i32(parent)
    for x in layers:
        path.build_summaries(x.st, lens[0])
        path.predict(x.st, dev_bf16(x.q[0]), lens[0])
        path.stage(x.st, lens[0], 0)
    for i in range(STEPS):
        rows = np.sort(rng.integers(1, T, (R, T)), -1).astype(np.int32)
        rows[:, 0] = 0
        n = rng.integers(1, T + 1, R).astype(np.int32)
        prev = ctx
        for x in layers:  # every layer commits before any is looked at
            note(f"commit of a layer, step {i} local={local}")
            path.commit(x.st, dev_bf16(x.k[i]), dev_bf16(x.v[i]), dev_i32(rows), dev_i32(n), lens[i % 2], lens[(i + 1) % 2])
            path.predict(x.st, dev_bf16(x.q[i + 1]), lens[(i + 1) % 2])
            path.stage(x.st, lens[(i + 1) % 2], i + 1, copy_local=False)
        torch.cuda.synchronize()
        for x in layers:
            ctx = O.append_tokens(x.k[i], x.v[i], rows, n, x.kp, x.vp, table, prev, B)
            assert np.array_equal(lens[(i + 1) % 2].cpu().numpy(), ctx)
            assert np.array_equal(host_bits(x.hk), x.kp) and np.array_equal(host_bits(x.hv), x.vp)
            tree = (x.k[i + 1], x.v[i + 1], parent, [T] * R)
            mag = (x.k[i + 1], _magnitude(x.v[i + 1]), parent, [T] * R)
            args = (x.st, dev_bf16(x.q[i + 1]), lens[(i + 1) % 2], dev_bf16(x.k[i + 1]), dev_bf16(x.v[i + 1]), dparent)
            path.attend_tree_dense(*args)
            ref, ref_lse = O.tree_attend(x.q[i + 1], x.kp, x.vp, table, ctx, *tree, B)
            ref_abs, _ = O.tree_attend(x.q[i + 1], x.kp, _magnitude(x.vp), table, ctx, *mag, B)
            _check(x.st.out, x.st.lse, ref, ref_abs, ref_lse, x.st.out)
            path.attend_tree(*args)
            pk, pv, smap = x.staged(table, ctx)
            ref, ref_lse = O.sparse_tree_attend(x.q[i + 1], pk, pv, smap, ctx, *tree, B)
            ref_abs, _ = O.sparse_tree_attend(x.q[i + 1], pk, _magnitude(pv), smap, ctx, *mag, B)
            _check(x.st.out, x.st.lse, ref, ref_abs, ref_lse, x.st.out)


def test_pipelined_steps_of_layers_on_their_own_pages():
    """The same outputs as serial staging of each layer alone, a step behind; beside a layer on the path's tier."""
    table = np.random.default_rng(6).permutation(R * NB).reshape(R, NB).astype(np.int32)
    path = _path(table)
    layers = [_Layer(i, path, table, False) for i in range(LAYERS)]
    path.host_k, path.host_v = layers[0].hk, layers[0].hv
    shared = path.new_layer()  # on the path's tier, which holds what the first layer's own pages hold
    ctx = dev_i32(CTX)
    runs = [(x.st, x) for x in layers] + [(shared, layers[0])]
    for st, x in runs:
        path.build_summaries(st, ctx)
        path.predict(st, dev_bf16(x.q[0]), ctx)
        path.stage(st, ctx, 0)
    torch.cuda.synchronize()
    for i in range(1, STEPS):
        for st, x in runs:
            note(f"pipelined step {i}")
            path.step_pipelined(st, dev_bf16(x.q[i]), ctx, i)
        torch.cuda.synchronize()
        path.check()
        for st, x in runs[:LAYERS]:
            pk, pv, smap = x.staged(table, CTX)  # as staged behind this step: for the next one
            assert np.array_equal(host_bits(st.pool_k)[smap_used(smap)], pk[smap_used(smap)])
        assert torch.equal(shared.slot_map, layers[0].st.slot_map) and torch.equal(shared.out, layers[0].st.out)
        assert torch.equal(shared.pool_k, layers[0].st.pool_k) and torch.equal(shared.pool_v, layers[0].st.pool_v)
    path.close()


def smap_used(smap):
    """Mask [R][K + 1][H] of the slots that hold a block."""
    return np.concatenate([np.swapaxes(smap >= 0, 1, 2), np.zeros((R, 1, H), bool)], 1)
