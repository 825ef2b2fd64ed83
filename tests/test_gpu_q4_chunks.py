"""Calls of the 4-bit cache at the sizes of prompts, bit for bit: appends whose workgroups take several tokens, compressed
keys that are read and written past the caches."""
import numpy as np
import pytest
import torch

import paper_2608_08097_amd as P
from oracle import oasis_oracle as O
from oracle import q4 as Q
from tests.gpu_util import dev_bf16, dev_i32, host_bits, note
from tests.test_gpu_drafts import INF, NAN
from tests.test_gpu_q4 import _rotary, _turns, dev_u8
from workloads import random_bf16

pytestmark = pytest.mark.gpu


def _appended(rows, at, pages, table, ctx, B, row_of, put, turns=None):
    """What oracle.q4.append_tokens does, for all rows at once: rows [R][T][H][d] (float64) are written to pages (in place)
    where `put` [R][T] says so, row (r, i) being rows[r, row_of[r, i]]; the rows as read back."""
    R, T, H, _ = rows.shape
    x = np.take_along_axis(rows, row_of[:, :, None, None], 1)
    if turns is not None:
        x = Q.rotate(x, at, *turns)
    codes, powers = Q.quantise(x.reshape(R, T, H, 4, 32))
    flat = codes.reshape(R, T, H, 128)
    packed = flat[..., 0::2] | (flat[..., 1::2] << 4)
    page = np.take_along_axis(table, np.minimum(at // B, table.shape[1] - 1), 1)
    r, i = np.nonzero(put)
    for h in range(H):
        first = (h * B + at[r, i] % B) * 64
        pages[page[r, i][:, None], first[:, None] + np.arange(64)] = packed[r, i, h]
        t = at[r, i] % B
        for g in range(4):
            pages[page[r, i], H * B * 64 + h * B * 4 + t // 16 * 64 + t % 4 * 16 + g * 4 + t % 16 // 4] = powers[r, i, h, g]
    return Q.values(codes, powers).reshape(R, T, H, 128)


def _chunk(seed, R, H, T, B, ctx, lens=None, rot=None, path=False, bad=False, read=True, wild=False):
    rng = np.random.default_rng(seed)
    note(f"append of a chunk seed={seed} R={R} H={H} T={T} B={B} rot={rot} path={path} bad={bad}")
    ctx = np.array(ctx, np.int32)
    NB = (int(ctx.max()) + T + B - 1) // B - (1 if bad else 0)
    NP = R * NB + 2
    table = rng.permutation(NP)[:R * NB].reshape(R, NB).astype(np.int32)
    if bad:
        table[rng.random((R, NB)) < 0.1] = rng.choice([-1, -2 ** 31, NP, 2 ** 31 - 1])
    joint = random_bf16(seed + 1, (R, T, 3 * H, 128), scale=1.5)
    if wild:
        joint[rng.random(joint.shape) < 0.001] = NAN
        joint[rng.random(joint.shape) < 0.001] = INF | 0x8000
    n = np.full(R, T) if lens is None else np.clip(np.array(lens), 0, T)
    n = np.minimum(n, np.maximum(NB * B - ctx, 0))
    rows = np.broadcast_to(np.arange(T), (R, T)).copy()
    if path:
        rows = np.stack([rng.permutation(T) for _ in range(R)])
        rows[rng.random(rows.shape) < 0.05] = rng.choice([-1, T, -2 ** 31, 2 ** 31 - 1])
    at = ctx[:, None] + np.arange(T)
    page = np.take_along_axis(table, np.minimum(at // B, NB - 1), 1)
    put = (np.arange(T) < n[:, None]) & (rows >= 0) & (rows < T) & (page >= 0) & (page < NP)
    pages = [rng.integers(0, 256, (NP, Q.page_bytes(H, B))).astype(np.uint8) for _ in range(2)]
    both, dev = dev_bf16(joint), [dev_u8(p) for p in pages]
    reads = [torch.full((R, T, H, 128), 7.0, dtype=torch.bfloat16, device="cuda") if read else None for _ in range(2)]
    ends = dev_i32(np.full(R, -5))
    d = P.dims(R, 2 * H, H, 128, B, NB)
    P.oasis_append_tokens_q4(d, None if rot is None else _rotary(*rot), both[:, :, H:2 * H], both[:, :, 2 * H:], T,
                             dev_i32(rows) if path else None,
                             dev_i32(np.full(R, T) if lens is None else np.array(lens)) if path or lens is not None else None,
                             *dev, dev_i32(table), dev_i32(ctx), ends, *reads)
    torch.cuda.synchronize()
    assert np.array_equal(ends.cpu().numpy(), ctx + n)
    row_of = np.where(put, rows, 0)
    for j, (got, want, back) in enumerate(zip(dev, pages, reads)):
        x = O.bf16_to_f64(np.ascontiguousarray(joint[:, :, (j + 1) * H:(j + 2) * H]))
        values = _appended(x, at, want, table, ctx, B, row_of, put, None if rot is None or j else (_turns(rot[0]), *rot[1:]))
        same = got.cpu().numpy() == want
        assert same.all(), np.argwhere(~same)[:4]
        if read:
            y = back.double().cpu().numpy()
            assert np.array_equal(y[put], values[put], equal_nan=True)
            assert np.all(y[~put] == 7.0)


# A workgroup takes one token of fewer than 2,048 rows, then two, from 4,096 on four, from 8,192 on eight
@pytest.mark.parametrize("R,T", [(3, 683), (2, 1999), (4, 1025), (1, 8191), (2, 4096), (5, 1701), (1, 8207)])
@pytest.mark.parametrize("rot", [None, (128, False, 1.0), (64, False, 1.1), (50, False, 1.0), (128, True, 1.0), (38, True, 1.3)])
def test_chunks_of_every_size_of_workgroup(R, T, rot):
    H = 3 if T % 2 else 8
    _chunk(5000 + T, R, H, T, 16 if R % 2 else 32, [5 + 3000 * r for r in range(R)], [T - 5 * r for r in range(R)], rot)


@pytest.mark.parametrize("H,R,T", [(1, 2, 4099), (2, 9, 1000), (3, 2, 1700), (8, 3, 701)])
def test_chunks_with_what_is_left_out(H, R, T):
    """Paths in any order, rows and pages that are none, requests without rows and past the table's end."""
    lens = [T, 0, 1, T - 3, -4, 9, T + 9, 8, 7][:R]
    for rot in (None, (96, False, 1.0), (128, True, 1.0)):
        _chunk(5100 + H, R, H, T, 16, [70 * r for r in range(R)], lens, rot, path=True, bad=True, wild=True)
        _chunk(5200 + H, R, H, T, 32, [0] * R, None, rot, bad=True, read=False)


@pytest.mark.parametrize("H", [9, 12, 33])
def test_more_heads_than_a_workgroup_takes_at_once(H):
    for rot in (None, (128, False, 1.0), (64, True, 1.0)):
        _chunk(5300 + H, 2, H, 5, 16, [15, 40], [5, 3], rot)
        _chunk(5400 + H, 3, H, 700, 32, [0, 1, 100], None, rot)


# -- compressed keys past the caches: from 96 MiB of codes on, by each request's own count


def _wide(seed, H, B, ctx, prev=None):
    rng = np.random.default_rng(seed)
    NP, ctx = 61, np.array(ctx, np.int32)
    R, NB = len(ctx), int(ctx.max()) // B + 2
    note(f"compressed keys past the caches seed={seed} R={R} H={H} B={B} NB={NB} prev={prev}")
    x = rng.normal(size=(NP, H, B, 128)) * np.exp(rng.normal(size=(NP, H, B, 1)) * 3)
    x[rng.random((NP, H, B)) < 0.1] = np.nan
    x[7, 1] = np.nan  # nothing but NaN
    pages = Q.make_pages(x)
    table = rng.integers(0, NP, (R, NB)).astype(np.int32)
    table[rng.random((R, NB)) < 0.05] = rng.choice([-1, -2 ** 31, NP, 2 ** 31 - 1])
    out = [torch.full((R, H, NB, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    d = P.dims(R, 2 * H, H, 128, B, NB)
    P.oasis_update_summaries_q4(d, dev_u8(pages), dev_i32(table), None if prev is None else dev_i32(prev), dev_i32(ctx), 1 << 30, *out)
    torch.cuda.synchronize()
    read = Q.read_pages(pages, H, B)
    with np.errstate(invalid="ignore"):
        ends = np.fmax.reduce(read, axis=2, initial=-np.inf), np.fmin.reduce(read, axis=2, initial=np.inf)
    n_cand = np.array([O.block_counts(int(c), B)[1] for c in ctx])
    first = np.zeros(R, int) if prev is None else np.array([O.block_counts(int(c), B)[1] for c in prev])
    b = np.arange(NB)
    written = (b >= first[:, None]) & (b < n_cand[:, None]) & (table >= 0) & (table < NP)
    for got, end in zip(out, ends):
        bits = host_bits(got).transpose(0, 2, 1, 3)
        assert np.array_equal(O.bf16_to_f64(bits[written]), end[table[written]])
        assert np.all(bits[~written] == 0x40E0)
    return n_cand - first


@pytest.mark.parametrize("H,B", [(5, 16), (3, 32), (8, 16), (7, 32)])
def test_compressed_keys_past_the_caches(H, B):
    need = (96 << 20) // (2 * H * B * 68) + 1  # blocks of each of two requests
    for extra in (0, 1, 6):
        assert np.all(_wide(6000 + H + extra, H, B, [(need + extra) * B + 1, (need + 3) * B]) >= need)


@pytest.mark.parametrize("H,B", [(5, 16), (3, 32)])
def test_a_long_request_beside_short_ones(H, B):
    """One call in both forms: the long request's rows past the caches, the short ones' through them."""
    need = (96 << 20) // (4 * H * B * 68) + 1
    n = _wide(6100 + H, H, B, [100, (need + 2) * B + 5, 0, 777])
    assert n[1] >= need and max(n[0], n[2], n[3]) < need // 10
    n = _wide(6200 + H, H, B, [(need + 40) * B, (need + 40) * B, 50, (need + 40) * B], [need * B, 17, 0, 40 * B - 3])
    assert n[0] < need // 10 and n[1] >= need and n[3] >= need
