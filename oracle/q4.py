"""CPU oracle of the 4-bit cache, in float64 NumPy: rotary positions, quantisation, pages, compressed keys, attention.

Written from the definitions in include/oasis.h: a value is the nearest level of a search over all levels, a power the
first that fits of a search over all powers.
"""
from __future__ import annotations

import math

import numpy as np

from .oasis_oracle import _softmax_attend, bf16_to_f64, block_counts, tree_paths

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def frequencies(dim, base, scaling="plain", factor=1.0, first_len=0.0, low=1.0, high=32.0):
    """Turns of each pair a position, and the amplitude."""
    out = []
    if scaling == "stretched" and dim > 2:
        base = base * factor ** (dim / (dim - 2))

    def index(turns):  # of the pair that makes so many turns in first_len positions
        return dim * math.log(first_len / (turns * 2 * math.pi)) / (2 * math.log(base))

    for i in range(dim // 2):
        f = base ** (-2 * i / dim) / (2 * math.pi)
        if scaling == "linear":
            f /= factor
        elif scaling == "by_turns":
            kept = min(max((first_len * f - low) / (high - low), 0.0), 1.0)
            f = kept * f + (1 - kept) * f / factor
        elif scaling == "by_index":
            a, b = max(math.floor(index(high)), 0), min(math.ceil(index(low)), dim - 1)
            b = b if b > a else a + 0.001
            kept = min(max(1 - (i - a) / (b - a), 0.0), 1.0)
            f = kept * f + (1 - kept) * f / factor
        out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1 if scaling == "by_index" and factor > 1 else 1.0


def rotate(x, positions, turns, interleaved=False, amplitude=1.0, inverse=False):
    """Rows x [..., H][d] (float64) at positions [...], pair by pair."""
    x = np.array(x, dtype=np.float64)
    out, half = x.copy(), len(turns)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = np.asarray(positions, dtype=np.float64) * turns[i]
        angle = 2 * np.pi * (t - np.floor(t)) * (-1 if inverse else 1)
        c, s = np.cos(angle)[..., None] * amplitude, np.sin(angle)[..., None] * amplitude
        with np.errstate(invalid="ignore"):
            out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return out


def quantise(x):
    """Codes [..., 32] and power bytes [...] of groups of 32 float64 values."""
    x = np.asarray(x, dtype=np.float64)
    top = np.max(np.abs(x), axis=-1)
    finite = np.all(np.isfinite(x), axis=-1)
    e = np.full(top.shape, 125)
    for p in range(124, -127, -1):  # the smallest that fits is the last one found
        e = np.where(top <= 7.0 * 2.0 ** p, p, e)
    safe = np.where(finite[..., None], x, 0.0)
    y = np.abs(safe) * np.exp2(-e.astype(np.float64))[..., None]
    gap = np.abs(y[..., None] - LEVELS)
    code = np.full(y.shape, 0)
    best = gap[..., 0]
    for i in range(1, 8):
        better = (gap[..., i] < best) | ((gap[..., i] == best) & (i % 2 == 0))
        code, best = np.where(better, i, code), np.where(better, gap[..., i], best)
    code = code + 8 * np.signbit(safe)
    code = np.where(finite[..., None], code, 0)
    return code.astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def values(codes, powers):
    """float64 values of codes [..., 32] with power bytes [...]."""
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    p = np.where(powers == 255, np.nan, np.exp2(powers.astype(np.float64) - 127))
    return v * p[..., None]


def page_bytes(Hkv, B):
    return Hkv * B * 68


def _places(Hkv, B, h, t):
    """First byte of token t's codes and its four power bytes in a page."""
    powers = [Hkv * B * 64 + h * B * 4 + (t // 16) * 64 + (t % 4) * 16 + g * 4 + t % 16 // 4 for g in range(4)]
    return (h * B + t) * 64, powers


def write_token(page, Hkv, B, h, t, row):
    """Row [d] (float64) as token t of head h of a page (uint8, in place)."""
    codes, powers = quantise(np.reshape(row, (4, GROUP)))
    at, places = _places(Hkv, B, h, t)
    flat = codes.reshape(-1)
    page[at:at + 64] = flat[0::2] | (flat[1::2] << 4)
    for g in range(4):
        page[places[g]] = powers[g]


def read_page(page, Hkv, B):
    """float64 [Hkv][B][d] of a page."""
    out = np.empty((Hkv, B, 128))
    for h in range(Hkv):
        for t in range(B):
            at, places = _places(Hkv, B, h, t)
            b = page[at:at + 64]
            codes = np.stack([b & 15, b >> 4], -1).reshape(4, GROUP)
            out[h, t] = values(codes, page[places]).reshape(-1)
    return out


def make_pages(x):
    """4-bit pages [n][page bytes] of values [n][Hkv][B][d]."""
    n, Hkv, B, _ = x.shape
    pages = np.zeros((n, page_bytes(Hkv, B)), np.uint8)
    codes, powers = quantise(np.reshape(x, (n, Hkv, B, 4, GROUP)))
    flat = codes.reshape(n, Hkv, B, 128)
    pages[:, :Hkv * B * 64] = (flat[..., 0::2] | (flat[..., 1::2] << 4)).reshape(n, -1)
    for h in range(Hkv):
        for t in range(B):
            pages[:, _places(Hkv, B, h, t)[1]] = powers[:, h, t]
    return pages


def read_pages(pages, Hkv, B):
    return np.stack([read_page(p, Hkv, B) for p in pages]) if len(pages) else np.zeros((0, Hkv, B, 128))


def append_tokens(new_k, new_v, path, path_len, k_pages, v_pages, block_table, ctx_len, B, rot=None):
    """Rows (bf16 bits [R][T][Hkv][d]) into pages, in place; rot: (turns, interleaved, amplitude). Returns the new lengths
    and the rows as read back, NaN where none was appended."""
    R, T, H, D = new_k.shape
    cap = len(block_table[0]) * B
    ends, read = np.zeros(R, np.int32), np.full((2, R, T, H, D), np.nan)
    done = np.zeros((R, T), bool)
    for r in range(R):
        ctx = max(0, min(int(ctx_len[r]), cap))
        n = T if path_len is None else max(0, min(int(path_len[r]), T))
        n = min(n, cap - ctx)
        for i in range(n):
            row = i if path is None else int(path[r, i])
            page = int(block_table[r][(ctx + i) // B])
            if not (0 <= row < T and 0 <= page < len(k_pages)):
                continue
            k, v = bf16_to_f64(new_k[r, row]), bf16_to_f64(new_v[r, row])
            if rot is not None:
                k = rotate(k, ctx + i, *rot)
            for j, (x, pages) in enumerate(((k, k_pages), (v, v_pages))):
                for h in range(H):
                    write_token(pages[page], H, B, h, (ctx + i) % B, x[h])
                codes, powers = quantise(x.reshape(H, 4, GROUP))
                read[j, r, i] = values(codes, powers).reshape(H, D)
            done[r, i] = True
        ends[r] = ctx + n
    return ends, read, done


def update_summaries(pages, block_table, prev_ctx_len, ctx_len, B, kmax, kmin, max_new=None):
    """float64 [R][Hkv][NB][d] kmax and kmin, in place."""
    R, H, NB, _ = kmax.shape
    for r in range(R):
        end = block_counts(min(int(ctx_len[r]), NB * B), B)[1]
        first = 0 if prev_ctx_len is None else block_counts(min(int(prev_ctx_len[r]), NB * B), B)[1]
        if prev_ctx_len is not None:
            end = min(end, first + max_new)
        for b in range(first, end):
            page = int(block_table[r][b])
            if 0 <= page < len(pages):
                x = read_page(pages[page], H, B)
                with np.errstate(invalid="ignore"):
                    kmax[r, :, b] = np.fmax.reduce(x, axis=1, initial=-np.inf)
                    kmin[r, :, b] = np.fmin.reduce(x, axis=1, initial=np.inf)


def attend(q, k_values, v_values, block_table, ctx_len, sel, sel_count, tree_k, tree_v, parent, tree_len, B, scale=None,
           magnitude=False):
    """Attention over pages of values (float64 [n][Hkv][B][d]): every block (sel None) or the selected and the local one,
    and the tree's rows on each row's path (tree_k None: no tree). Rows past a tree's end are NaN; magnitude: with the
    values' magnitudes."""
    qf = bf16_to_f64(q)
    R, T, Hq, D = qf.shape
    H, NB = k_values.shape[1], len(block_table[0])
    G = Hq // H
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, lse = np.full((R, T, Hq, D), np.nan), np.full((R, T, Hq), np.nan)
    tk, tv = (None, None) if tree_k is None else (bf16_to_f64(tree_k), bf16_to_f64(tree_v))
    for r, rows in enumerate(tree_paths(parent, tree_len, T)):
        L = max(0, min(int(ctx_len[r]), NB * B))
        nb, n_cand, local = block_counts(L, B)
        for h in range(H):
            blocks = list(range(nb))
            if sel is not None:
                picked = sel[r][h][:max(0, min(int(sel_count[r][h]), len(sel[r][h])))]
                blocks = [int(b) for b in picked if 0 <= b < n_cand] + ([n_cand] if nb else [])
            ks, vs = [np.zeros((0, D))], [np.zeros((0, D))]
            for b in blocks:
                page, n = int(block_table[r][b]), local if b == n_cand else B
                if 0 <= page < len(k_values):
                    ks.append(k_values[page, h, :n])
                    vs.append(v_values[page, h, :n])
            ck, cv = np.concatenate(ks), np.concatenate(vs)
            for t, path in enumerate(rows):
                keys, vals = ck, cv
                if tk is not None:
                    keys, vals = np.concatenate([ck, tk[r, path, h]]), np.concatenate([cv, tv[r, path, h]])
                at = (r, t, slice(h * G, (h + 1) * G))
                if not len(keys):
                    out[at], lse[at] = 0.0, -np.inf
                    continue
                out[at], lse[at] = _softmax_attend(qf[r, t, h * G:(h + 1) * G], keys, np.abs(vals) if magnitude else vals,
                                                   scale)
    return out, lse
