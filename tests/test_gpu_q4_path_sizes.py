"""Steps of a 4-bit path with one token and with the widest trees, as its defaults make them, against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from oracle import q4 as Q
from paper_2608_08097_amd.path_q4 import Q4Path
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import _check
from tests.test_gpu_q4 import dev_u8
from workloads import random_bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,tree", [(1, True), (1, False), (2, True), (64, True)])
@pytest.mark.parametrize("G,B", [(1, 16), (4, 32)])
def test_steps_of_default_paths(T, tree, G, B):
    R, H, NB, k = 2, 2, 20, 4
    rng = np.random.default_rng(T + G)
    note(f"default 4-bit path T={T} G={G} B={B} tree={tree}")
    d = P.dims(R, G * H, H, 128, B, NB)
    table = rng.permutation(R * NB).reshape(R, NB).astype(np.int32)
    path = Q4Path(d, T, k, R * NB, dev_i32(table), P.Rotary(128))
    st = path.new_layer()
    kp, vp = (Q.make_pages(rng.normal(size=(R * NB, H, B, 128))) for _ in range(2))
    st.k_pages.copy_(dev_u8(kp)), st.v_pages.copy_(dev_u8(vp))
    lens = np.array([9 * B + 5, 12 * B], np.int32)
    ctx, new = dev_i32(lens), dev_i32(np.zeros(R))
    P.oasis_update_summaries_q4(d, st.k_pages, path.block_table, None, ctx, 0, st.kmax, st.kmin)
    q, rows_k, rows_v = (random_bf16(70 + T + j, (R, T, h, 128)) for j, h in enumerate((G * H, H, H)))
    dev_q, tk = path.rotate(dev_bf16(q), dev_bf16(rows_k), ctx)
    tv = dev_bf16(rows_v)
    path.predict(st, dev_q, ctx)
    rq, rk = host_bits(dev_q), host_bits(tk)
    sel, cnt = st.sel.cpu().numpy(), st.sel_count.cpu().numpy()
    score = O.block_scores(rq, *(O.bf16_to_f64(host_bits(x)) for x in (st.kmax, st.kmin)), lens, H, B, path.first_draft,
                           path.num_draft)
    for r in range(R):
        n = O.block_counts(int(lens[r]), B)[1]
        for h in range(H):
            assert cnt[r, h] == k
            best = np.sort(score[r, h, :n])[::-1][:k]
            assert np.allclose(np.sort(score[r, h, sel[r, h]])[::-1], best, rtol=1e-5)
    path.attend(st, dev_q, ctx, tk if tree else None, tv if tree else None)
    args = (rq, Q.read_pages(kp, H, B), Q.read_pages(vp, H, B), table, lens, sel, cnt, rk if tree else None, rows_v if tree else None,
            None, [T] * R, B)
    ref, ref_lse = Q.attend(*args)
    ref_abs, _ = Q.attend(*args, magnitude=True)
    _check(st.out, st.lse, ref, ref_abs, ref_lse, st.out)
    path.commit(st, tk, tv, None, None, ctx, new)
    assert np.array_equal(new.cpu().numpy(), lens + T)
    Q.append_tokens(rk, rows_v, None, None, kp, vp, table, lens, B)
    assert np.array_equal(st.k_pages.cpu().numpy(), kp) and np.array_equal(st.v_pages.cpu().numpy(), vp)
