"""Timed cases of the cache held in four bits: rotary positions, the append that quantises, compressed keys, attention.

Five operators, each through the package's public entry points:

* ``rotate``   rotary positions of a step's query and key rows (``oasis_rotate``);
* ``append``   new keys, rotated on the way, and values into 4-bit pages (``oasis_append_tokens_q4``);
* ``summary``  compressed keys (per-block minimum and maximum) of 4-bit pages (``oasis_update_summaries_q4``);
* ``dense``    attention over every cached token of 4-bit pages (``oasis_tree_attn_q4``);
* ``select``   attention over the selected blocks, read where they lie in the 4-bit pages (``oasis_tree_attn_q4``).

A 4-bit page holds, for B tokens of every KV head, codes [Hkv][B][64] (dims 2 j and 2 j + 1 in the low and high half of
byte j; a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) and then, for each 32 of a token's dims, a power of two: byte
s of [Hkv][B / 16][4][4][4], indexed by t % 4, the group of dims and t % 16 / 4, stands for 2^(s - 127).

Sizes follow the repository's own configurations (8 x 131,072 tokens; 16 x 65,536 tokens at block 32; 64 reasoning
requests) and the batches between them. A case is a dict of plain values; inputs come from its seed alone and are made
on the GPU. With ``own`` false ``run`` computes the operators in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False  # True: run() calls the framework's kernels; False: the plain forms below

D = 128       # head dimension
GROUP = 32    # dims that share a power of two
LOW = -126    # exponents of the powers of two that are written
HIGH = 125


# -- cases -------------------------------------------------------------------------


def _rotate(name, R, T, Hq, Hkv, dim, pairs, scaling, hi, packed):
    """dim: the first dims of a head that turn; pairs: half (i with i + dim / 2) or next (2 i with 2 i + 1); hi:
    contexts before the rows are uniform in [0, hi]; packed: rows lie in a projection's output, queries, keys and values
    one after the other; scaling: none, linear or turns."""
    return {"name": name, "kind": "rotate", "R": R, "T": T, "Hq": Hq, "Hkv": Hkv, "dim": dim, "pairs": pairs,
            "scaling": scaling, "hi": hi, "packed": packed}


def _append(name, R, Hkv, T, B, hi, accepted, dim, pairs, scaling, packed):
    """accepted: rows come from an accepted path; otherwise all T rows of a prompt chunk are written; dim 0: the keys
    come rotated already."""
    return {"name": name, "kind": "append", "R": R, "Hkv": Hkv, "T": T, "B": B, "hi": hi, "accepted": accepted,
            "dim": dim, "pairs": pairs, "scaling": scaling, "packed": packed}


def _summary(name, R, Hkv, B, lo, hi, new):
    """new: blocks completed since the last call, at most so many of a request; 0: every block."""
    return {"name": name, "kind": "summary", "R": R, "Hkv": Hkv, "B": B, "lo": lo, "hi": hi, "new": new}


def _attn(name, kind, R, Hq, Hkv, T, tree, B, lo, hi, k=0):
    """lo, hi: context lengths are uniform in [lo, hi]; k: blocks selected at most (kind select); tree: chain, random,
    beam, or none (the rows attend the cache alone)."""
    return {"name": name, "kind": kind, "R": R, "Hq": Hq, "Hkv": Hkv, "T": T, "tree": tree, "B": B, "lo": lo, "hi": hi,
            "k": k}


def listed():
    return [
        # the rows of one decode step of 64 requests: nothing but latency
        _rotate("rotate_step", 64, 5, 32, 8, 128, "half", "none", 16384, False),
        # a prompt chunk out of the projection's output, half of each head turned, scaled for long contexts
        _rotate("rotate_prompt", 4, 8192, 32, 8, 64, "next", "turns", 131072, True),
        # the accepted paths of a batch, their keys rotated already
        _append("append_accepted", 64, 8, 16, 16, 16384, True, 0, "half", "none", False),
        # a prompt chunk of 8,192 tokens for each of four requests, rotated and quantised out of the projection's output
        _append("append_prompt", 4, 8, 8192, 16, 8192, False, 128, "half", "linear", True),
        # the blocks that a batch completes in a step
        _summary("summary_step", 64, 8, 16, 4096, 16384, 1),
        # compressed keys of whole contexts, 8 x 131,072 tokens
        _summary("summary_build", 8, 8, 16, 131072, 131072, 0),
        # a single interactive request below the sparsification threshold, one token: nothing but latency
        _attn("dense_one", "dense", 1, 32, 8, 1, "chain", 16, 1900, 2000),
        # dense attention over long contexts: 8 x 131,072 tokens, a token and four drafted ones
        _attn("dense_long", "dense", 8, 32, 8, 5, "chain", 16, 131072, 131072),
        # a moderate batch of mixed lengths, 16-node trees (64 rows per KV head)
        _attn("dense_ragged", "dense", 24, 32, 8, 16, "random", 16, 1, 32768),
        # deep speculation on wide heads: 64-node trees, 512 rows per KV head, where arithmetic bounds
        _attn("dense_wide", "dense", 2, 64, 8, 64, "beam", 32, 65000, 65536),
        # the selected 2,048 tokens of each head of 8 x 131,072 tokens
        _attn("select_long", "select", 8, 32, 8, 5, "none", 16, 131072, 131072, 128),
        # wide heads, 4,096 selected tokens of 16 x 65,536, nine rows a head, block 32
        _attn("select_wide", "select", 16, 64, 8, 9, "chain", 32, 65536, 65536, 128),
    ]


def draw(rng):
    def log_int(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choice(["rotate", "append", "append", "summary", "dense", "dense", "dense", "select", "select"])
    while True:
        Hkv, B = rng.choice([1, 2, 4, 8, 8]), rng.choice([16, 16, 32])
        dim, pairs = rng.choice([128, 128, 96, 64, 32]), rng.choice(["half", "half", "next"])
        scaling, packed = rng.choice(["none", "linear", "turns"]), rng.random() < 0.5
        if kind == "rotate":
            G, R, T = rng.choice([1, 2, 3, 4, 4, 5, 8]), log_int(1, 128), log_int(1, 8192)
            if 256.0 * R * T * (G + 2) * Hkv > 4.5e8:
                continue
            c = _rotate("", R, T, G * Hkv, Hkv, dim, pairs, scaling, log_int(16, 1000000), packed)
        elif kind == "append":
            accepted = rng.random() < 0.5
            R, T = log_int(1, 128 if accepted else 16), log_int(1, 64) if accepted else log_int(2, 8192)
            hi = log_int(16, 16384)
            if R * T * Hkv > 4 * 8192 * 8 or 136.0 * R * Hkv * (hi + T) > 4e8:
                continue
            c = _append("", R, Hkv, T, B, hi, accepted, rng.choice([0, dim]), pairs, scaling, packed)
        elif kind == "summary":
            R, hi, new = log_int(1, 96), log_int(16, 131072), rng.choice([0, 0, 1, 4])
            if 1.0 * R * Hkv * hi > 8.4e6:
                continue
            c = _summary("", R, Hkv, B, rng.choice([hi, max(1, hi // 2), 0]), hi, new)
        else:
            tree, T = rng.choice(["chain", "random", "beam", "none"]), rng.choice([1, log_int(1, 64)])
            G, R, hi = rng.choice([1, 2, 3, 4, 4, 5, 8]), log_int(1, 96), log_int(20, 131072)
            lo = rng.choice([hi, max(1, hi // 2), 0])
            k = 0 if kind == "dense" else log_int(1, 300)
            L = hi if kind == "dense" else min(hi, (k + 1) * B)
            # tokens of the cache, operations, and the plain form's logits
            if 1.0 * R * Hkv * hi > 8.4e6 or 4.0 * R * Hkv * G * T * L * D > 2.7e11 or 4.0 * R * Hkv * G * T * L > 2.2e9:
                continue
            c = _attn("", kind, R, G * Hkv, Hkv, T, tree, B, lo, hi, k)
        del c["name"]
        return c


# -- inputs ------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _table(g, R, NB):
    """Block table [R][NB] over R * NB pages in any order."""
    return torch.randperm(R * NB, generator=g, device="cuda").view(R, NB).to(torch.int32)


def _angles(dim, scaling):
    """Turns of each pair a position, float64 [dim / 2]: base 500,000 and contexts of 8,192 stretched to 131,072."""
    base, factor, first = 500000.0, 16.0, 8192.0
    freq = [base ** (-2.0 * i / dim) / (2.0 * math.pi) for i in range(dim // 2)]
    if scaling == "linear":
        freq = [f / factor for f in freq]
    elif scaling == "turns":  # pairs of at most one turn over the first contexts are stretched, of four and more not
        ramp = [min(max((first * f - 1.0) / 3.0, 0.0), 1.0) for f in freq]
        freq = [f * (r + (1.0 - r) / factor) for f, r in zip(freq, ramp)]
    amplitude = 0.1 * math.log(factor) + 1.0 if scaling == "turns" else 1.0
    return torch.tensor(freq, dtype=torch.float64, device="cuda"), amplitude


def _outliers(g, Hkv):
    """How large a head's dims are, next to each other: a few are several times the others."""
    return torch.exp(0.6 * torch.randn((Hkv, 1, D), generator=g, device="cuda"))


def _pages(g, n, Hkv, B, spread):
    """n 4-bit pages uint8 [n][Hkv * B * 68] of quantised normal values; `spread` [Hkv][1][D]: the dims' sizes."""
    out = torch.empty((n, Hkv * B * 68), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (Hkv * B * D))
    for at in range(0, n, step):
        m = min(step, n - at)
        x = torch.randn((m, Hkv, B, D), generator=g, device="cuda") * spread
        codes, scale = _quantise(x.view(m, Hkv, B, 4, GROUP))
        out[at:at + m, :Hkv * B * 64] = _packed(codes).view(m, -1)
        out[at:at + m, Hkv * B * 64:] = _dealt(scale, B).reshape(m, -1)
    return out


def _prepare_rotate(c, seed):
    g = _gen(seed)
    R, T, Hq, Hkv = c["R"], c["T"], c["Hq"], c["Hkv"]
    s = {"case": c, "ctx": torch.randint(0, c["hi"] + 1, (R,), generator=g, device="cuda", dtype=torch.int32)}
    s["angles"], s["amplitude"] = _angles(c["dim"], c["scaling"])
    if c["packed"]:
        both = _randn(g, R, T, Hq + 2 * Hkv, D)
        s["q"], s["k"] = both[:, :, :Hq], both[:, :, Hq:Hq + Hkv]
    else:
        s["q"], s["k"] = _randn(g, R, T, Hq, D), _randn(g, R, T, Hkv, D)
    # rows of a drafted tree have positions of their own; a prompt's follow the context
    s["at"] = None
    if T <= 64:
        depth = torch.randint(0, T, (R, T), generator=g, device="cuda", dtype=torch.int32).sort(-1).values
        s["at"] = s["ctx"][:, None] + depth
    s["q_out"] = torch.zeros((R, T, Hq, D), dtype=torch.bfloat16, device="cuda")
    s["k_out"] = torch.zeros((R, T, Hkv, D), dtype=torch.bfloat16, device="cuda")
    return s


def _prepare_append(c, seed):
    g = _gen(seed)
    R, Hkv, T, B = c["R"], c["Hkv"], c["T"], c["B"]
    NB = (c["hi"] + T + B - 1) // B
    s = {"case": c, "NB": NB, "table": _table(g, R, NB)}
    s["ctx"] = torch.randint(0, c["hi"] + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    if c["packed"]:  # as many query heads as key heads stand before them
        both = _randn(g, R, T, 3 * Hkv, D)
        s["new_k"], s["new_v"] = both[:, :, Hkv:2 * Hkv], both[:, :, 2 * Hkv:]
    else:
        s["new_k"], s["new_v"] = _randn(g, R, T, Hkv, D), _randn(g, R, T, Hkv, D)
    s["new_k"] *= _outliers(g, Hkv)[:, 0].to(torch.bfloat16)
    s["angles"], s["amplitude"] = _angles(c["dim"], c["scaling"]) if c["dim"] else (None, 1.0)
    # what the pages hold already is of no matter to an append, but it stays
    for n in ("k", "v"):
        s[n] = torch.randint(1, 200, (R * NB, Hkv * B * 68), generator=g, device="cuda", dtype=torch.uint8)
    s["path"], s["path_len"] = None, None
    if c["accepted"]:  # an ascending path through the tree, row 0 first
        s["path_len"] = torch.randint(1, min(T, 8) + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
        order = torch.rand((R, T), generator=g, device="cuda")
        order[:, 0] = -1.0
        rows = order.argsort(-1)
        keep = torch.arange(T, device="cuda") < s["path_len"][:, None]
        rows = torch.where(keep, rows, torch.full_like(rows, T)).sort(-1).values
        s["path"] = torch.where(keep, rows, torch.full_like(rows, -1)).to(torch.int32)
    for n in ("read_k", "read_v"):
        s[n] = torch.zeros((R, T, Hkv, D), dtype=torch.bfloat16, device="cuda")
    s["new_ctx"] = torch.zeros((R,), dtype=torch.int32, device="cuda")
    return s


def _prepare_summary(c, seed):
    g = _gen(seed)
    R, Hkv, B, hi = c["R"], c["Hkv"], c["B"], c["hi"]
    NB = (hi + B - 1) // B
    s = {"case": c, "NB": NB, "table": _table(g, R, NB)}
    s["k"] = _pages(g, R * NB, Hkv, B, _outliers(g, Hkv))
    s["ctx"] = torch.randint(c["lo"], hi + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    s["prev"] = None
    if c["new"]:
        back = torch.randint(1, c["new"] * B + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
        s["prev"] = (s["ctx"] - back).clamp(min=0)
    for n in ("kmax", "kmin"):
        s[n] = torch.zeros((R, Hkv, NB, D), dtype=torch.bfloat16, device="cuda")
    return s


def _trees(g, c):
    """Parents [R][T] and rows in use [R]: chains, two children a node (beam) or any earlier row near by (random)."""
    R, T = c["R"], c["T"]
    t = torch.arange(T, device="cuda")
    if c["tree"] == "beam":
        parent = torch.div(t + 1, 2, rounding_mode="floor").sub(1).expand(R, T)
    elif c["tree"] == "random":
        back = torch.randint(1, 5, (R, T), generator=g, device="cuda")
        parent = (t - back).clamp(min=0)
        parent[:, 0] = -1
    else:
        parent = (t - 1).expand(R, T)
    length = torch.full((R,), T, device="cuda")
    if R > 2:  # some drafters stopped early
        cut = torch.randint(0, max(1, T // 2) + 1, (R,), generator=g, device="cuda")
        length = length - torch.where(torch.rand((R,), generator=g, device="cuda") < 0.25, cut, torch.zeros_like(cut))
    return parent.to(torch.int32).contiguous(), length.to(torch.int32)


def _prepare_attn(c, seed):
    g = _gen(seed)
    R, Hq, Hkv, T, B, k = c["R"], c["Hq"], c["Hkv"], c["T"], c["B"], c["k"]
    NB = max(1, (c["hi"] + B - 1) // B)
    s = {"case": c, "NB": NB, "table": _table(g, R, NB)}
    s["ctx"] = torch.randint(c["lo"], c["hi"] + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    s["k"], s["v"] = _pages(g, R * NB, Hkv, B, _outliers(g, Hkv)), _pages(g, R * NB, Hkv, B, torch.ones((1, 1, 1), device="cuda"))
    s["parent"], s["len"] = _trees(g, c)
    s["q"] = _randn(g, R, T, Hq, D) * 1.5  # peaked logits
    s["tree_k"], s["tree_v"] = None, None
    if c["tree"] == "none":
        s["parent"] = None
    else:
        s["tree_k"], s["tree_v"] = _randn(g, R, T, Hkv, D), _randn(g, R, T, Hkv, D)
    s["sel"], s["count"] = None, None
    if k:  # the best blocks by a random score, ascending; all of them where there are no more than k
        nc = ((s["ctx"] + B - 1) // B - 1).clamp(min=0)
        score = torch.rand((R, Hkv, NB), generator=g, device="cuda")
        score.masked_fill_(torch.arange(NB, device="cuda") >= nc[:, None, None], -1.0)
        best = score.topk(min(k, NB), -1)
        ids = torch.where(best.values >= 0, best.indices, NB).sort(-1).values
        ids = torch.nn.functional.pad(torch.where(ids < NB, ids, -1), (0, k - ids.shape[-1]), value=-1)
        s["sel"] = ids.to(torch.int32).contiguous()
        s["count"] = (ids >= 0).sum(-1).to(torch.int32)
    s["out"] = torch.zeros((R, T, Hq, D), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((R, T, Hq), dtype=torch.float32, device="cuda")
    return s


def prepare(case, seed):
    return {"rotate": _prepare_rotate, "append": _prepare_append, "summary": _prepare_summary, "dense": _prepare_attn,
            "select": _prepare_attn}[case["kind"]](case, seed)


# -- four bits -----------------------------------------------------------------------


def _quantise(x):
    """Codes (uint8, as x) and bytes of the powers of two (uint8, x without its last dimension) of groups [..., 32]:
    the smallest 2^e whose seven-fold reaches the group's largest value, and the nearest value, ties to an even code."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.875, e - 3, e - 2)
    e = torch.where(top == 0, torch.full_like(e, LOW), e).clamp(LOW, HIGH)
    y = torch.ldexp(x.double(), -e[..., None]) if x.dtype == torch.float64 else x * torch.exp2(-e.double()).float()[..., None]
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for edge, up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= edge) if up else (a > edge)
    return code | (torch.signbit(x).to(torch.uint8) << 3), (e + 127).to(torch.uint8)


def _packed(codes):
    """Two codes a byte, the even dim in the low half."""
    pair = codes.reshape(*codes.shape[:-1], -1, 2)
    return pair[..., 0] | (pair[..., 1] << 4)


def _dealt(scale, B):
    """Bytes [..., B][4] in the pages' order [..., B / 16][t % 4][group][t % 16 / 4]."""
    x = scale.view(*scale.shape[:-2], B // 16, 4, 4, 4)  # [t / 16][t % 16 / 4][t % 4][group]
    return x.movedim(-3, -1)


def _values(pages, Hkv, B):
    """float32 [n][Hkv][B][D] of 4-bit pages."""
    n = pages.shape[0]
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    levels = torch.cat([levels, -levels])
    codes = pages[:, :Hkv * B * 64].reshape(n, Hkv, B, 64)
    x = torch.stack([levels[(codes & 15).int()], levels[(codes >> 4).int()]], -1).view(n, Hkv, B, 4, GROUP)
    s = pages[:, Hkv * B * 64:].reshape(n, Hkv, B // 16, 4, 4, 4).movedim(-1, -3).reshape(n, Hkv, B, 4)
    return (x * torch.exp2(s.float() - 127.0)[..., None]).view(n, Hkv, B, D)


# -- plain forms -------------------------------------------------------------------


def _turned(x, at, c, angles, amplitude):
    """float64 [..., H][D] of rows x [R][T][H][D] at positions at [R][T]."""
    x = x.double()
    if not c["dim"]:
        return x
    half = c["dim"] // 2
    phase = at.double()[..., None] * angles
    phase = 2.0 * math.pi * (phase - phase.floor())
    co, si = (torch.cos(phase) * amplitude)[:, :, None], (torch.sin(phase) * amplitude)[:, :, None]
    if c["pairs"] == "half":
        a, b = x[..., :half], x[..., half:c["dim"]]
        y = torch.cat([a * co - b * si, b * co + a * si], -1)
    else:
        a, b = x[..., 0:c["dim"]:2], x[..., 1:c["dim"]:2]
        y = torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)
    return torch.cat([y, x[..., c["dim"]:]], -1)


def _plain_rotate(s):
    c = s["case"]
    at = s["at"] if s["at"] is not None else s["ctx"][:, None] + torch.arange(c["T"], device="cuda")
    return [_turned(s[n], at, c, s["angles"], s["amplitude"]).to(torch.bfloat16) for n in ("q", "k")]


def _plain_append(s):
    c = s["case"]
    R, Hkv, T, B = c["R"], c["Hkv"], c["T"], c["B"]
    i = torch.arange(T, device="cuda").expand(R, T)
    n = torch.full((R,), T, device="cuda") if s["path_len"] is None else s["path_len"].long()
    used = i < n[:, None]
    i = torch.where(used, i, 0)  # past the path's end: its first row once more
    rows = (i if s["path"] is None else s["path"].long().gather(1, i))[..., None, None].expand(R, T, Hkv, D)
    pos = s["ctx"].long()[:, None] + i
    page = s["table"].long().gather(1, torch.div(pos, B, rounding_mode="floor"))[..., None]
    head, t = torch.arange(Hkv, device="cuda"), (pos % B)[..., None]
    at = (head * B + t)[..., None] * 64 + torch.arange(64, device="cuda")  # [R][T][Hkv][64]
    group = torch.arange(4, device="cuda")
    sub = head * (B // 16) + torch.div(t, 16, rounding_mode="floor")  # 16 tokens of a head
    at_s = Hkv * B * 64 + ((sub * 4 + t % 4)[..., None] * 4 + group) * 4 + torch.div(t % 16, 4, rounding_mode="floor")[..., None]
    read = []
    for name, new in (("k", "new_k"), ("v", "new_v")):
        x = s[new].gather(1, rows)
        x = _turned(x, pos, c, s["angles"], s["amplitude"]) if name == "k" and c["dim"] else x.float()
        codes, scale = _quantise(x.view(R, T, Hkv, 4, GROUP))
        codes = codes.view(R, T, Hkv, D)
        s[name].index_put_((page[..., None], at), _packed(codes))
        s[name].index_put_((page[..., None], at_s), scale)
        levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
        back = torch.cat([levels, -levels])[codes.int()].view(R, T, Hkv, 4, GROUP)
        back = (back * torch.exp2(scale.float() - 127.0)[..., None]).view(R, T, Hkv, D)
        read.append(torch.where(used[..., None, None], back, torch.zeros_like(back)).to(torch.bfloat16))
    return {"k": s["k"], "v": s["v"], "read_k": read[0], "read_v": read[1], "new_ctx": (s["ctx"].long() + n).int()}


def _plain_summary(s):
    c = s["case"]
    R, Hkv, B, NB = c["R"], c["Hkv"], c["B"], s["NB"]
    nc = ((s["ctx"].long() + B - 1) // B - 1).clamp(min=0)
    if c["new"]:
        first = ((s["prev"].long() + B - 1) // B - 1).clamp(min=0)
        b = first[:, None] + torch.arange(c["new"], device="cuda")
    else:
        b = torch.arange(NB, device="cuda").expand(R, NB)
    valid = b < nc[:, None]
    b = b.clamp(max=NB - 1)
    x = _values(s["k"][s["table"].long().gather(1, b).view(-1)], Hkv, B).view(R, -1, Hkv, B, D)
    r, h = torch.arange(R, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[:, None]
    keep = valid[:, None, :, None]
    for name, y in (("kmax", x.amax(3)), ("kmin", x.amin(3))):
        y = torch.where(keep, y.transpose(1, 2).to(torch.bfloat16), s[name][r, h, b[:, None]])
        # blocks past the last one stand on it: their old rows must not win
        put = torch.where(valid, b, NB)
        wide = torch.cat([s[name], torch.zeros_like(s[name][:, :, :1])], 2)
        wide[r, h, put[:, None]] = y
        s[name].copy_(wide[:, :, :NB])
    return [s["kmax"], s["kmin"]]


def _ancestors(parent, length):
    """[R][T][T]: row t attends drafted token j (itself and the rows above it)."""
    R, T = parent.shape
    t = torch.arange(T, device=parent.device)
    up = ((parent[..., None] == t) & (t < t[:, None])).float()
    a = up + torch.eye(T, device=parent.device)
    for _ in range(6):  # paths of up to 64 rows
        a = (torch.matmul(a, a) > 0).float()
    return (a > 0) & (t < length[:, None, None])


def _plain_attn(s):
    c = s["case"]
    R, Hq, Hkv, T, B = c["R"], c["Hq"], c["Hkv"], c["T"], c["B"]
    G, ctx, NB = Hq // Hkv, s["ctx"].long(), s["NB"]
    if not c["k"]:
        table = s["table"].view(-1).long()
        k, v = (_values(s[n][table], Hkv, B).view(R, NB, Hkv, B, D).transpose(1, 2).reshape(R, Hkv, -1, D) for n in ("k", "v"))
        seen = (torch.arange(NB * B, device="cuda") < ctx[:, None])[:, None].expand(R, Hkv, -1)
    else:  # the selected blocks and, behind them, the local one
        local = ((ctx + B - 1) // B - 1).clamp(min=0)
        blocks = torch.cat([s["sel"].long(), local[:, None, None].expand(R, Hkv, 1)], -1)
        pages = s["table"].long()[torch.arange(R, device="cuda")[:, None, None], blocks.clamp(min=0)]
        head = torch.arange(Hkv, device="cuda")[:, None]
        size = B * 64
        parts = []
        for n in ("k", "v"):  # each head's part of its pages, as pages of one head
            codes = s[n][:, :Hkv * size].view(-1, Hkv, size)[pages, head]
            scale = s[n][:, Hkv * size:].view(-1, Hkv, B * 4)[pages, head]
            parts.append(_values(torch.cat([codes, scale], -1).view(-1, B * 68), 1, B).view(R, Hkv, -1, D))
        k, v = parts
        pos = torch.arange(B, device="cuda")
        tail = (ctx - local * B)[:, None, None]
        seen = torch.cat([(s["sel"] >= 0)[..., None].expand(-1, -1, -1, B).reshape(R, Hkv, -1),
                          (pos < tail).expand(R, Hkv, B)], -1)
    q = s["q"].float().view(R, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, T * G, D)
    scale = 1.0 / math.sqrt(D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    x.masked_fill_(~seen[:, :, None], -math.inf)
    m = x.amax(-1)
    y = None
    if s["tree_k"] is not None:
        tk, tv = (s[n].float().transpose(1, 2).contiguous() for n in ("tree_k", "tree_v"))
        y = torch.matmul(q, tk.transpose(2, 3).contiguous()).mul_(scale)
        mask = _ancestors(s["parent"], s["len"])[:, :, None].expand(R, T, G, T).reshape(R, 1, T * G, T)
        y = y.masked_fill(~mask, -math.inf)
        m = torch.maximum(m, y.amax(-1))
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)[..., None]  # rows that attend nothing
    x.sub_(m).exp_()
    l, o = x.sum(-1, keepdim=True), torch.matmul(x, v)
    if y is not None:
        y = (y - m).exp()
        l, o = l + y.sum(-1, keepdim=True), o + torch.matmul(y, tv)
    o = torch.where(l > 0, o / l, torch.zeros_like(o))
    lse = (m + l.log())[..., 0]
    used = torch.arange(T, device="cuda") < s["len"][:, None]
    o = o.view(R, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(R, T, Hq, D)
    lse = lse.view(R, Hkv, T, G).permute(0, 2, 1, 3).reshape(R, T, Hq)
    return [torch.where(used[..., None, None], o, torch.zeros_like(o)).to(torch.bfloat16),
            torch.where(used[..., None], lse, torch.zeros_like(lse))]


# -- the framework's calls ---------------------------------------------------------


def _rotary(P, s):
    c = s["case"]
    return P.Rotary.from_turns(s["angles"], interleaved=c["pairs"] == "next", amplitude=s["amplitude"]) if c["dim"] else None


def _own_rotate(s):
    import paper_2608_08097_amd as P
    c = s["case"]
    if "d" not in s:  # kept by a program between its calls
        s["d"], s["rot"] = P.dims(c["R"], c["Hq"], c["Hkv"], D, 16, 1), _rotary(P, s)
    P.oasis_rotate(s["d"], s["rot"], c["T"], s["at"], s["ctx"], s["q"], s["q_out"], s["k"], s["k_out"])
    return [s["q_out"], s["k_out"]]


def _own_append(s):
    import paper_2608_08097_amd as P
    c = s["case"]
    if "d" not in s:
        s["d"], s["rot"] = P.dims(c["R"], c["Hkv"], c["Hkv"], D, c["B"], s["NB"]), _rotary(P, s)
    P.oasis_append_tokens_q4(s["d"], s["rot"], s["new_k"], s["new_v"], c["T"], s["path"], s["path_len"], s["k"], s["v"],
                             s["table"], s["ctx"], s["new_ctx"], s["read_k"], s["read_v"])
    return {n: s[n] for n in ("k", "v", "read_k", "read_v", "new_ctx")}


def _own_summary(s):
    import paper_2608_08097_amd as P
    c = s["case"]
    if "d" not in s:
        s["d"] = P.dims(c["R"], c["Hkv"], c["Hkv"], D, c["B"], s["NB"])
    P.oasis_update_summaries_q4(s["d"], s["k"], s["table"], s["prev"], s["ctx"], c["new"], s["kmax"], s["kmin"])
    return [s["kmax"], s["kmin"]]


def _own_attn(s):
    import paper_2608_08097_amd as P
    c, T = s["case"], s["case"]["T"]
    if "d" not in s:
        s["d"] = P.dims(c["R"], c["Hq"], c["Hkv"], D, c["B"], s["NB"])
        s["ws"] = torch.empty(P.oasis_tree_attn_q4_workspace_bytes(s["d"], T, c["k"]), dtype=torch.uint8, device="cuda")
    P.oasis_tree_attn_q4(s["d"], s["q"], T, s["k"], s["v"], s["table"], s["ctx"], s["sel"], s["count"], c["k"], s["tree_k"],
                         s["tree_v"], s["parent"], s["len"], None, s["out"], s["lse"], s["ws"])
    return [s["out"], s["lse"]]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rotate": _own_rotate, "append": _own_append, "summary": _own_summary, "dense": _own_attn,
                "select": _own_attn}[kind](state)
    return {"rotate": _plain_rotate, "append": _plain_append, "summary": _plain_summary, "dense": _plain_attn,
            "select": _plain_attn}[kind](state)


# -- what a pass cannot do without ---------------------------------------------------


def work(case):
    c = case
    R, Hkv = c["R"], c["Hkv"]
    if c["kind"] == "rotate":  # rows in and out, their positions
        rows, heads = R * c["T"], c["Hq"] + Hkv
        return {"bytes": rows * (heads * 4.0 * D + 4) + 4.0 * c["dim"], "flops": rows * heads * 3.0 * c["dim"]}
    if c["kind"] == "append":  # bf16 rows in; 4-bit rows and the rows as they read out
        n = R * (0.5 * (1 + min(c["T"], 8)) if c["accepted"] else c["T"]) * 2 * Hkv
        return {"bytes": n * (2.0 * D + 68 + 2.0 * D + 4), "flops": n * D * 4.0}
    if c["kind"] == "summary":  # 4-bit keys of the blocks in, two bf16 rows of each out
        L = 0.5 * (c["lo"] + c["hi"])
        # a length that grew by 1 to new * B tokens completes half as many blocks more or less
        n = R * Hkv * max(0.5, 0.5 * (c["new"] * c["B"] + 1) / c["B"] if c["new"] else L / c["B"] - 1.0)
        return {"bytes": n * (c["B"] * 68.0 + 4.0 * D), "flops": n * c["B"] * D * 2.0}
    L, B = 0.5 * (c["lo"] + c["hi"]), c["B"]
    if c["k"]:
        top = (c["k"] + 0.5) * B  # mean of min(length, selected and local tokens) over [lo, hi]
        if c["hi"] > top:
            share = (c["hi"] - max(c["lo"], top)) / (c["hi"] - c["lo"]) if c["hi"] > c["lo"] else 1.0
            L = share * top + (1 - share) * 0.5 * (c["lo"] + top)
    T, Hq = c["T"], c["Hq"]
    tree = 0 if c["tree"] == "none" else T
    size = R * (2 * 68.0 * Hkv * L + 512.0 * Hkv * tree + T * Hq * (2 * 2 * D + 4) + 8 * T)
    return {"bytes": size, "flops": 4.0 * R * T * Hq * D * (L + 0.5 * tree)}


# -- from the definitions, in 64 bits --------------------------------------------------


_LEVEL = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_turned(x, at, c, angles, amplitude):
    """Pairs as complex numbers, multiplied by one of the unit circle: x [n][H][D] at positions at [n]."""
    x, dim = x.double(), c["dim"]
    if not dim:
        return x
    z = torch.polar(torch.full((len(at), dim // 2), amplitude, dtype=torch.float64, device="cuda"),
                    torch.remainder(at.double()[:, None] * angles, 1.0) * (2.0 * math.pi))[:, None]
    out = x.clone()
    pair = (slice(0, dim // 2), slice(dim // 2, dim)) if c["pairs"] == "half" else (slice(0, dim, 2), slice(1, dim, 2))
    y = torch.complex(x[..., pair[0]].contiguous(), x[..., pair[1]].contiguous()) * z
    out[..., pair[0]], out[..., pair[1]] = y.real, y.imag
    return out


def _exact_rotate(c, s):
    out = []
    for n in ("q", "k"):
        rows = []
        for r in range(c["R"]):
            at = s["ctx"][r] + torch.arange(c["T"], device="cuda") if s["at"] is None else s["at"][r]
            rows.append(_exact_turned(s[n][r], at, c, s["angles"], s["amplitude"]).cpu())
        out.append(torch.stack(rows))
    return out


def _nearest(x):
    """Code and exponent of groups [..., 32] by search: over the exponents for the first that fits, over the levels for
    the nearest (of two as near the one with an even code)."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, LOW)
    guess = torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -140))) - 4
    for step in range(5, -1, -1):  # the largest exponent that does not fit, plus one
        t = guess + step
        e = torch.where((top <= 7.0 * torch.exp2(t)), torch.maximum(t, torch.full_like(t, LOW)), e)
    e = torch.where(top == 0, torch.full_like(e, LOW), e.clamp(LOW, HIGH))
    y = (x * torch.exp2(-e)).abs()
    best, code = torch.full_like(y, math.inf), torch.zeros(y.shape, dtype=torch.int64, device=y.device)
    for i, level in enumerate(_LEVEL):
        off = (y - level).abs()
        better = (off < best) | ((off == best) & (i % 2 == 0))
        best, code = torch.where(better, off, best), torch.where(better, i, code)
    value = torch.tensor(_LEVEL, dtype=torch.float64, device=x.device)[code] * torch.exp2(e)
    minus = torch.signbit(x)
    return code + 8 * minus.long(), e[..., 0].long() + 127, torch.where(minus, -value, value)


def _exact_append(c, s):
    R, Hkv, T, B = c["R"], c["Hkv"], c["T"], c["B"]
    out = {"k": s["k"].clone(), "v": s["v"].clone()}
    read = {n: torch.zeros((R, T, Hkv, D), dtype=torch.float64, device="cuda") for n in ("k", "v")}
    ctx, ends = s["ctx"].tolist(), []
    for r in range(R):
        rows = list(range(T)) if s["path"] is None else s["path"][r, :int(s["path_len"][r])].tolist()
        at = ctx[r] + torch.arange(len(rows), device="cuda")
        for n in ("k", "v"):
            x = s["new_" + n][r, rows]
            x = _exact_turned(x, at, c, s["angles"], s["amplitude"]) if n == "k" else x.double()
            code, byte, value = _nearest(x.view(len(rows), Hkv, 4, GROUP))
            code, read[n][r, :len(rows)] = code.view(len(rows), Hkv, D), value.view(len(rows), Hkv, D)
            codes = out[n][:, :Hkv * B * 64].unflatten(1, (Hkv, B, 64))
            scales = out[n][:, Hkv * B * 64:].unflatten(1, (Hkv, B // 16, 4, 4, 4))
            i = 0
            while i < len(rows):  # the tokens that fall into one block
                b, o = divmod(ctx[r] + i, B)
                m = min(B - o, len(rows) - i)
                page = int(s["table"][r, b])
                codes[page, :, o:o + m] = (code[i:i + m, :, 0::2] + 16 * code[i:i + m, :, 1::2]).to(torch.uint8).transpose(0, 1)
                t = torch.arange(o, o + m, device="cuda")
                scales[page, :, t // 16, t % 4, :, t % 16 // 4] = byte[i:i + m].to(torch.uint8)
                i += m
        ends.append(ctx[r] + len(rows))
    return {**out, "read_k": read["k"], "read_v": read["v"], "new_ctx": torch.tensor(ends, dtype=torch.int32)}


def _exact_block(pages, h, Hkv, B):
    """float64 [n * B][D]: KV head h of whole pages."""
    n = len(pages)
    byte = pages[:, h * B * 64:(h + 1) * B * 64].long().view(n, B, 64)
    code = torch.stack([byte % 16, byte // 16], -1).view(n, B, D)
    power = pages[:, Hkv * B * 64 + h * B * 4:Hkv * B * 64 + (h + 1) * B * 4].double().view(n, B // 16, 4, 4, 4)
    power = power.permute(0, 1, 4, 2, 3).reshape(n, B, 4).repeat_interleave(GROUP, -1)
    value = torch.tensor(_LEVEL, dtype=torch.float64, device="cuda")[code % 8] * torch.exp2(power - 127.0)
    return torch.where(code < 8, value, -value).view(n * B, D)


def _exact_summary(c, s):
    R, Hkv, B = c["R"], c["Hkv"], c["B"]
    out = [s["kmax"].double(), s["kmin"].double()]
    ctx = s["ctx"].tolist()
    for r in range(R):
        end = max(0, -(-ctx[r] // B) - 1)
        first = 0
        if c["new"]:
            first = max(0, -(-int(s["prev"][r]) // B) - 1)
            end = min(end, first + c["new"])
        if end <= first:
            continue
        for h in range(Hkv):
            x = _exact_block(s["k"][s["table"][r, first:end].long()], h, Hkv, B).view(-1, B, D)
            out[0][r, h, first:end], out[1][r, h, first:end] = x.max(1).values, x.min(1).values
    return out


def _exact_attn(c, s):
    R, Hq, Hkv, T, B = c["R"], c["Hq"], c["Hkv"], c["T"], c["B"]
    G = Hq // Hkv
    out, lse = torch.zeros((R, T, Hq, D), dtype=torch.float64), torch.zeros((R, T, Hq), dtype=torch.float64)
    length, ctx = s["len"].tolist(), s["ctx"].tolist()
    parent = None if s["parent"] is None else s["parent"].tolist()
    for r in range(R):
        n, L = length[r], ctx[r]
        nb = -(-L // B)
        see = torch.zeros((n, n), dtype=torch.bool)
        for t in range(n if parent is not None else 0):
            j = t
            while 0 <= j < n:  # t, its parent, and so on up to the root
                see[t, j] = True
                j = parent[r][j]
        see = see.cuda()
        for h in range(Hkv):
            blocks = list(range(nb)) if not c["k"] else s["sel"][r, h, :int(s["count"][r, h])].tolist() + list(range(max(0, nb - 1), nb))
            pages = s["table"][r, torch.tensor(blocks, dtype=torch.long, device="cuda")].long()
            some = len(blocks) * B - (nb * B - L)  # the last block is the only one that may be part full
            k, v = _exact_block(s["k"][pages], h, Hkv, B)[:some], _exact_block(s["v"][pages], h, Hkv, B)[:some]
            if parent is not None:
                k = torch.cat([k, s["tree_k"][r, :n, h].double()])
                v = torch.cat([v, s["tree_v"][r, :n, h].double()])
            kt = k.T.contiguous()
            for g in range(G):
                z = s["q"][r, :n, h * G + g].double() @ kt / math.sqrt(D)
                if parent is not None:
                    z[:, k.shape[0] - n:][~see] = -math.inf
                e = torch.logsumexp(z, -1) if k.shape[0] else torch.full((n,), -math.inf, dtype=torch.float64, device="cuda")
                if k.shape[0]:
                    out[r, :n, h * G + g] = (torch.exp(z - e[:, None]) @ v).cpu()
                lse[r, :n, h * G + g] = e.cpu()
    return [out, lse]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("dense", "select"):
        # about 1e12 operations a second in 64 bits, and some 40 us for each of the loops' turns
        if work(case)["flops"] / 1e12 + case["R"] * case["Hq"] * 4e-4 > 15:
            return None
        return _exact_attn(case, s)
    return {"rotate": _exact_rotate, "append": _exact_append, "summary": _exact_summary}[case["kind"]](case, s)
