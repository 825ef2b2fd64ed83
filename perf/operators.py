"""Timed cases of the speculative step: attention of a drafted token tree, its verification, the append of what is accepted.

Four operators, each through the package's public entry points:

* ``tree``    attention of a tree of drafted tokens over the paged cache (``oasis_tree_attn``);
* ``sparse``  the same over the block-sparse working set (``oasis_sparse_tree_attn``);
* ``verify``  acceptance of the drafted tokens and the next token, from given random numbers (``oasis_verify_drafts``);
* ``append``  the accepted tokens' keys and values into the paged cache (``oasis_append_tokens``).

A tree is a list of parents: row 0 is the token being verified, row t > 0 a drafted token that follows row parent[t].
Sizes follow the repository's own configurations (8 x 131,072 tokens; 16 x 65,536 tokens at block 32; 64 reasoning
requests) and the batches between them. A case is a dict of plain values; inputs come from its seed alone and are made
on the GPU. With ``own`` false ``run`` computes the operators in elementary torch operations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: run() calls the framework's kernels; False: the plain forms below

D = 128  # head dimension


# -- cases -------------------------------------------------------------------------


def _attn(name, kind, R, Hq, Hkv, T, tree, B, lo, hi, budget=0):
    """lo, hi: context lengths are uniform in [lo, hi]; budget: tokens in the slots of a working set (kind sparse)."""
    return {"name": name, "kind": kind, "R": R, "Hq": Hq, "Hkv": Hkv, "T": T, "tree": tree, "B": B, "lo": lo, "hi": hi,
            "budget": budget}


def _verify(name, R, T, tree, V, draft):
    """draft: the drafter's probabilities are given (its tokens were sampled); otherwise its tokens are its best ones."""
    return {"name": name, "kind": "verify", "R": R, "T": T, "tree": tree, "V": V, "draft": draft}


def _append(name, R, Hkv, T, B, lo, hi, accepted):
    """accepted: rows come from an accepted path; otherwise all T rows of a prompt chunk are written."""
    return {"name": name, "kind": "append", "R": R, "Hkv": Hkv, "T": T, "B": B, "lo": lo, "hi": hi, "accepted": accepted}


def listed():
    return [
        # a single interactive request below the sparsification threshold, one drafted token: nothing but latency
        _attn("tree_one", "tree", 1, 32, 8, 2, "chain", 16, 1900, 2000),
        # dense verification of long contexts: 8 x 131,072 tokens, four drafted tokens
        _attn("tree_long", "tree", 8, 32, 8, 5, "chain", 16, 131072, 131072),
        # a moderate batch of mixed lengths, 16-node trees (64 rows per KV head)
        _attn("tree_ragged", "tree", 24, 32, 8, 16, "random", 16, 1, 32768),
        # deep speculation on wide heads: 64-node trees, 512 rows per KV head, where arithmetic bounds
        _attn("tree_wide", "tree", 2, 64, 8, 64, "beam", 32, 65000, 65536),
        # the working set of 8 x 131,072 tokens, four drafted tokens
        _attn("sparse_long", "sparse", 8, 32, 8, 5, "chain", 16, 131072, 131072, 2048),
        # wide heads over the working set of 16 x 65,536 tokens: 32-node trees, 256 rows per KV head, block 32
        _attn("sparse_wide", "sparse", 16, 64, 8, 32, "beam", 32, 65536, 65536, 4096),
        # a full batch early in decoding: short prompts, so most slots are free; small trees
        _attn("sparse_short", "sparse", 64, 32, 8, 7, "random", 16, 200, 3000, 2048),
        # one request, a chain of four drafted tokens with the drafter's probabilities
        _verify("verify_one", 1, 5, "chain", 32000, True),
        # a batch with sampled trees: rejected siblings leave a residual that the next one is held to
        _verify("verify_trees", 48, 16, "random", 50261, True),
        # a large vocabulary, wide trees of the drafter's best tokens
        _verify("verify_wide", 32, 32, "beam", 131072, False),
        # the accepted paths of a batch into the paged cache
        _append("append_accepted", 64, 8, 16, 16, 4096, 16384, True),
        # a prompt chunk of 8,192 tokens for each of four requests
        _append("append_prompt", 4, 8, 8192, 16, 0, 8192, False),
    ]


def draw(rng):
    def log_int(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choice(["tree"] * 4 + ["sparse"] * 3 + ["verify"] * 3 + ["append"] * 2)
    while True:
        Hkv, B, tree = rng.choice([1, 2, 4, 8, 8]), rng.choice([16, 16, 32]), rng.choice(["chain", "random", "beam"])
        T = log_int(1, 64)
        if kind in ("tree", "sparse"):
            G, R, hi = rng.choice([1, 2, 3, 4, 4, 5, 8]), log_int(1, 96), log_int(20, 131072)
            lo = rng.choice([hi, max(1, hi // 2), 0])
            budget = rng.choice([512, 1024, 2048, 4096]) if kind == "sparse" else 0
            L = min(hi, budget + B) if kind == "sparse" else hi
            # bytes of the cache, operations, and the plain form's logits and gathered cache
            if 512.0 * R * Hkv * L > 4.3e9 or 4.0 * R * Hkv * G * T * L * D > 2.7e11 or 4.0 * R * Hkv * G * T * L > 2.2e9:
                continue
            if kind == "sparse" and 512.0 * R * Hkv * budget > 8e8:
                continue
            c = _attn("", kind, R, G * Hkv, Hkv, T, tree, B, lo, hi, budget)
        elif kind == "verify":
            R, V = log_int(1, 128), log_int(1000, 160000)
            if 4.0 * R * T * V > 6e8:
                continue
            c = _verify("", R, T, tree, V, rng.random() < 0.6)
        else:
            accepted = rng.random() < 0.6
            R, T, hi = log_int(1, 128 if accepted else 16), T if accepted else log_int(2, 8192), log_int(16, 16384)
            if 512.0 * R * Hkv * (hi + T) > 8e8:
                continue
            c = _append("", R, Hkv, T, B, rng.choice([0, hi // 2, hi]), hi, accepted)
        del c["name"]
        return c


# -- inputs ------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _lengths(g, c):
    return torch.randint(c["lo"], c["hi"] + 1, (c["R"],), generator=g, device="cuda", dtype=torch.int32)


def _trees(g, c):
    """Parents [R][T] and rows in use [R]: chains, two children a node (beam) or any earlier row near by (random)."""
    R, T = c["R"], c["T"]
    t = torch.arange(T, device="cuda")
    if c["tree"] == "chain":
        parent = (t - 1).expand(R, T)
    elif c["tree"] == "beam":
        parent = torch.div(t + 1, 2, rounding_mode="floor").sub(1).expand(R, T)
    else:
        back = torch.randint(1, 5, (R, T), generator=g, device="cuda")
        parent = (t - back).clamp(min=0)
        parent[:, 0] = -1
    length = torch.full((R,), T, device="cuda")
    if R > 2:  # some drafters stopped early
        cut = torch.randint(0, max(1, T // 2) + 1, (R,), generator=g, device="cuda")
        length = length - torch.where(torch.rand((R,), generator=g, device="cuda") < 0.25, cut, torch.zeros_like(cut))
    return parent.to(torch.int32).contiguous(), length.to(torch.int32)


def _tables(g, R, NB):
    """Block table [R][NB] over R * NB pages in any order."""
    return torch.randperm(R * NB, generator=g, device="cuda").view(R, NB).to(torch.int32)


def _prepare_attn(c, seed):
    g = _gen(seed)
    R, Hq, Hkv, T, B = c["R"], c["Hq"], c["Hkv"], c["T"], c["B"]
    s = {"case": c, "ctx": _lengths(g, c), "NB": max(1, (c["hi"] + B - 1) // B)}
    s["parent"], s["len"] = _trees(g, c)
    s["q"] = _randn(g, R, T, Hq, D) * 2.0  # peaked logits: deviation 2
    s["tree_k"], s["tree_v"] = _randn(g, R, T, Hkv, D), _randn(g, R, T, Hkv, D)
    if c["kind"] == "tree":
        s["table"] = _tables(g, R, s["NB"])
        s["k"], s["v"] = _randn(g, R * s["NB"], Hkv, B, D), _randn(g, R * s["NB"], Hkv, B, D)
    else:
        ks = s["ks"] = c["budget"] // B
        s["k"], s["v"] = _randn(g, R, ks + 1, Hkv, B, D), _randn(g, R, ks + 1, Hkv, D, B)
        # the first candidates where they fit, else ascending blocks spread over the context
        nc = ((s["ctx"] + B - 1) // B - 1).clamp(min=0).long()[:, None, None]
        slot = torch.arange(ks, device="cuda").expand(R, Hkv, ks)
        start = (torch.rand((R, Hkv, 1), generator=g, device="cuda") * s["NB"]).long()
        ids = torch.where(nc > ks, (start + slot * (nc // max(1, ks)).clamp(min=1)) % nc.clamp(min=1), slot)
        s["slot_map"] = torch.where(slot < nc, ids, torch.full_like(ids, -1)).to(torch.int32).contiguous()
    s["out"] = torch.zeros((R, T, Hq, D), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((R, T, Hq), dtype=torch.float32, device="cuda")
    return s


def _prepare_verify(c, seed):
    g = _gen(seed)
    R, T, V = c["R"], c["T"], c["V"]
    s = {"case": c}
    s["parent"], s["len"] = _trees(g, c)
    logits = torch.randn((R, T, V), generator=g, device="cuda").mul_(3.0)
    s["target"] = torch.softmax(logits, -1)
    # the drafter's logits: the target's and as much noise as leaves most of its tokens accepted
    logits.add_(torch.randn((R, T, V), generator=g, device="cuda"), alpha=0.7)
    at = s["parent"].long().clamp(min=0)
    if c["draft"]:
        s["draft"] = torch.softmax(logits, -1)
        pick = torch.multinomial(s["draft"].view(R * T, V), T, replacement=True, generator=g).view(R, T, T)
    else:
        s["draft"] = None
        pick = logits.topk(min(T, V), -1).indices
        pick = torch.nn.functional.pad(pick, (0, T - pick.shape[-1]))
    # row t's token: its parent's pick number (t's place among its siblings)
    same = (s["parent"][:, :, None] == s["parent"][:, None, :]).long()
    place = torch.tril(same, -1).sum(-1)
    s["tokens"] = pick.gather(1, at[:, :, None].expand(R, T, T)).gather(2, place[:, :, None])[..., 0].to(torch.int32)
    s["accept_u"] = torch.rand((R, T), generator=g, device="cuda")
    s["sample_u"] = torch.rand((R,), generator=g, device="cuda")
    for n in ("path", "out_tokens"):
        s[n] = torch.zeros((R, T), dtype=torch.int32, device="cuda")
    s["path_len"] = torch.zeros((R,), dtype=torch.int32, device="cuda")
    return s


def _prepare_append(c, seed):
    g = _gen(seed)
    R, Hkv, T, B = c["R"], c["Hkv"], c["T"], c["B"]
    NB = (c["hi"] + T + B - 1) // B
    s = {"case": c, "NB": NB, "ctx": _lengths(g, c), "table": _tables(g, R, NB)}
    s["new_k"], s["new_v"] = _randn(g, R, T, Hkv, D), _randn(g, R, T, Hkv, D)
    s["k"], s["v"] = _randn(g, R * NB, Hkv, B, D), _randn(g, R * NB, Hkv, B, D)
    s["path"], s["path_len"] = None, None
    if c["accepted"]:  # an ascending path through the tree, row 0 first
        s["path_len"] = torch.randint(1, min(T, 8) + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
        order = torch.rand((R, T), generator=g, device="cuda")
        order[:, 0] = -1.0
        rows = order.argsort(-1)
        keep = torch.arange(T, device="cuda") < s["path_len"][:, None]
        rows = torch.where(keep, rows, torch.full_like(rows, T)).sort(-1).values
        s["path"] = torch.where(keep, rows, torch.full_like(rows, -1)).to(torch.int32)
    s["new_ctx"] = torch.zeros((R,), dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    return {"tree": _prepare_attn, "sparse": _prepare_attn, "verify": _prepare_verify,
            "append": _prepare_append}[case["kind"]](case, seed)


# -- plain forms -------------------------------------------------------------------


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
    G, ctx = Hq // Hkv, s["ctx"].long()
    if c["kind"] == "tree":
        table = s["table"].long()
        k = s["k"][table].float().permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D)  # [R][Hkv][NB * B][d]
        v = s["v"][table].float().permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D)
        seen = (torch.arange(k.shape[2], device="cuda") < ctx[:, None])[:, None].expand(R, Hkv, -1)
    else:
        k = s["k"].float().permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D)  # [R][Hkv][(ks + 1) * B][d]
        v = s["v"].float().permute(0, 2, 1, 4, 3).reshape(R, Hkv, -1, D)
        local = ctx - ((ctx + B - 1) // B - 1).clamp(min=0) * B
        slots = (s["slot_map"] >= 0)[..., None].expand(R, Hkv, s["ks"], B).reshape(R, Hkv, -1)
        own_block = (torch.arange(B, device="cuda") < local[:, None])[:, None].expand(R, Hkv, B)
        seen = torch.cat([slots, own_block], -1)
    q = s["q"].float().view(R, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, T * G, D)
    tk, tv = s["tree_k"].float().transpose(1, 2).contiguous(), s["tree_v"].float().transpose(1, 2).contiguous()
    scale = 1.0 / math.sqrt(D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    x.masked_fill_(~seen[:, :, None], -math.inf)
    y = torch.matmul(q, tk.transpose(2, 3).contiguous()).mul_(scale)
    mask = _ancestors(s["parent"], s["len"])[:, :, None].expand(R, T, G, T).reshape(R, 1, T * G, T)
    y = y.masked_fill(~mask, -math.inf)
    m = torch.maximum(x.amax(-1), y.amax(-1))[..., None]
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)  # rows past the tree's end, dropped below
    x.sub_(m).exp_()
    y = (y - m).exp()
    l = x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
    o = (torch.matmul(x, v) + torch.matmul(y, tv)) / l
    lse = (m + l.log())[..., 0]
    used = torch.arange(T, device="cuda") < s["len"][:, None]
    o = o.view(R, Hkv, T, G, D).permute(0, 2, 1, 3, 4).reshape(R, T, Hq, D)
    lse = lse.view(R, Hkv, T, G).permute(0, 2, 1, 3).reshape(R, T, Hq)
    return [torch.where(used[..., None, None], o, torch.zeros_like(o)).to(torch.bfloat16),
            torch.where(used[..., None], lse, torch.zeros_like(lse))]


def _plain_verify(s):
    c = s["case"]
    R, T, V = c["R"], c["T"], c["V"]
    r = torch.arange(R, device="cuda")
    at = torch.zeros(R, dtype=torch.long, device="cuda")        # the node that the walk stands on
    steps = (s["len"] > 0).long()                                # rows on the path so far
    path = torch.full((R, T + 1), -1, dtype=torch.long, device="cuda")
    path[:, 0] = torch.where(steps > 0, 0, -1)
    toks = torch.full((R, T + 1), -1, dtype=torch.long, device="cuda")
    coef = torch.zeros(R, dtype=torch.float64, device="cuda")   # what of the draft's row is taken off the target's
    mass = torch.ones(R, dtype=torch.float64, device="cuda")    # of the residual
    gone = torch.zeros((R, V), dtype=torch.bool, device="cuda")  # rejected at this node (drafts without probabilities)

    def residual(coef):
        p = s["target"][r, at].double()
        if s["draft"] is None:
            return p.masked_fill(gone, 0.0)
        return (p - coef[:, None] * s["draft"][r, at].double()).clamp(min=0.0)

    for t in range(1, T):
        x = s["tokens"][:, t].long()
        child = (s["parent"][:, t] == at) & (t < s["len"])
        wx = residual(coef)[r, x]
        qx = 1.0 if s["draft"] is None else s["draft"][r, at, x].double()
        yes = child & (s["accept_u"][:, t].double() * qx * mass < wx)
        no = child & ~yes
        if s["draft"] is None:
            mass = torch.where(no, mass - wx, mass)
            gone[r, x] |= no
        else:
            coef = torch.where(no, coef + mass, coef)
            mass = torch.where(no, residual(coef).sum(-1), mass)
        path[r, torch.where(yes, steps, T)] = t
        toks[r, torch.where(yes, steps - 1, T)] = x
        steps, at = steps + yes.long(), torch.where(yes, t, at)
        coef, mass = torch.where(yes, 0.0, coef), torch.where(yes, 1.0, mass)
        gone &= ~yes[:, None]
    w = residual(coef)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, s["target"][r, at].double())
    total = w.cumsum(-1)
    nxt = (total > s["sample_u"].double()[:, None] * w.sum(-1, keepdim=True)).int().argmax(-1)
    toks[r, torch.where(steps > 0, steps - 1, T)] = nxt
    return [path[:, :T].int(), steps.int(), toks[:, :T].int()]


def _plain_append(s):
    c = s["case"]
    R, Hkv, T, B = c["R"], c["Hkv"], c["T"], c["B"]
    i = torch.arange(T, device="cuda").expand(R, T)
    n = torch.full((R,), T, device="cuda") if s["path_len"] is None else s["path_len"].long()
    i = torch.where(i < n[:, None], i, 0)  # past the path's end: its first row once more
    rows = i if s["path"] is None else s["path"].long().gather(1, i)
    pos = s["ctx"].long()[:, None] + i
    page = s["table"].long().gather(1, torch.div(pos, B, rounding_mode="floor"))
    at = (page[..., None] * Hkv + torch.arange(Hkv, device="cuda")) * B + (pos % B)[..., None]  # [R][T][Hkv]
    pick = rows[..., None, None].expand(R, T, Hkv, D)
    s["k"].view(-1, D).index_put_((at,), s["new_k"].gather(1, pick))
    s["v"].view(-1, D).index_put_((at,), s["new_v"].gather(1, pick))
    return [s["k"], s["v"], (s["ctx"].long() + n).int()]


# -- the framework's calls ---------------------------------------------------------


def _own_attn(s):
    import paper_2608_08097_amd as P
    c, T = s["case"], s["case"]["T"]
    if "d" not in s:  # kept by a program between its calls
        s["d"] = P.dims(c["R"], c["Hq"], c["Hkv"], D, c["B"], s["NB"])
        need = (P.oasis_tree_attn_workspace_bytes(s["d"], T) if c["kind"] == "tree"
                else P.oasis_sparse_tree_attn_workspace_bytes(s["d"], T, s["ks"]))
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    if c["kind"] == "tree":
        P.oasis_tree_attn(s["d"], s["q"], T, s["k"], s["v"], s["table"], s["ctx"], s["tree_k"], s["tree_v"], s["parent"],
                          s["len"], None, s["out"], s["lse"], s["ws"])
    else:
        P.oasis_sparse_tree_attn(s["d"], s["q"], T, s["k"], s["v"], s["slot_map"], s["ks"], s["ctx"], s["tree_k"],
                                 s["tree_v"], s["parent"], s["len"], None, s["out"], s["lse"], s["ws"])
    return [s["out"], s["lse"]]


def _own_verify(s):
    import paper_2608_08097_amd as P
    if "ws" not in s:
        need = P.oasis_verify_workspace_bytes(s["case"]["R"], s["case"]["T"], s["case"]["V"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    P.oasis_verify_drafts(s["target"], s["draft"], s["tokens"], s["parent"], s["len"], s["accept_u"], s["sample_u"],
                          s["path"], s["path_len"], s["out_tokens"], s["ws"])
    return [s["path"], s["path_len"], s["out_tokens"]]


def _own_append(s):
    import paper_2608_08097_amd as P
    c = s["case"]
    if "d" not in s:
        s["d"] = P.dims(c["R"], c["Hkv"], c["Hkv"], D, c["B"], s["NB"])
    P.oasis_append_tokens(s["d"], s["new_k"], s["new_v"], c["T"], s["path"], s["path_len"], s["k"], s["v"], s["table"],
                          s["ctx"], s["new_ctx"])
    return [s["k"], s["v"], s["new_ctx"]]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"tree": _own_attn, "sparse": _own_attn, "verify": _own_verify, "append": _own_append}[kind](state)
    return {"tree": _plain_attn, "sparse": _plain_attn, "verify": _plain_verify, "append": _plain_append}[kind](state)


# -- what a pass cannot do without ---------------------------------------------------


def work(case):
    c = case
    if c["kind"] == "verify":  # the last node's row of each table and the scalars of the walk
        rows = 2 if c["draft"] else 1
        return {"bytes": c["R"] * (4.0 * c["V"] * rows + 28.0 * c["T"]), "flops": 3.0 * c["R"] * c["V"]}
    L = 0.5 * (c["lo"] + c["hi"])
    if c["kind"] == "append":
        n = 0.5 * (1 + min(c["T"], 8)) if c["accepted"] else c["T"]
        return {"bytes": c["R"] * n * (2 * 512.0 * c["Hkv"] + 8), "flops": 0.0}
    if c["kind"] == "sparse":
        top = c["budget"] + c["B"]  # mean of min(length, budget and the local block) over [lo, hi]
        if c["hi"] > top:
            share = (c["hi"] - max(c["lo"], top)) / max(1, c["hi"] - c["lo"]) if c["hi"] > c["lo"] else 1.0
            L = share * top + (1 - share) * 0.5 * (c["lo"] + top)
    T, R, Hkv, Hq = c["T"], c["R"], c["Hkv"], c["Hq"]
    size = R * (512.0 * Hkv * (L + T) + T * Hq * (2 * 2 * D + 4) + 8 * T)
    return {"bytes": size, "flops": 4.0 * R * T * Hq * D * (L + 0.5 * T)}


# -- from the definitions, in 64 bits --------------------------------------------------


def _exact_attn(c, s):
    R, Hq, Hkv, T, B = c["R"], c["Hq"], c["Hkv"], c["T"], c["B"]
    G = Hq // Hkv
    out, lse = torch.zeros((R, T, Hq, D), dtype=torch.float64), torch.zeros((R, T, Hq), dtype=torch.float64)
    parent, length, ctx = s["parent"].tolist(), s["len"].tolist(), s["ctx"].tolist()
    for r in range(R):
        n, L = length[r], ctx[r]
        see = torch.zeros((n, n), dtype=torch.bool)
        for t in range(n):
            j = t
            while 0 <= j < n:  # t, its parent, and so on up to the root
                see[t, j] = True
                j = parent[r][j]
        see = see.cuda()
        for h in range(Hkv):
            if c["kind"] == "tree":
                blocks = s["table"][r, :(L + B - 1) // B].long()
                k, v = s["k"][blocks, h].reshape(-1, D)[:L], s["v"][blocks, h].reshape(-1, D)[:L]
            else:
                full = [i for i, b in enumerate(s["slot_map"][r, h].tolist()) if b >= 0]
                tail = L - B * max(0, (L + B - 1) // B - 1)
                k = torch.cat([s["k"][r, full, h].reshape(-1, D), s["k"][r, s["ks"], h, :tail]])
                v = torch.cat([s["v"][r, full, h].transpose(1, 2).reshape(-1, D), s["v"][r, s["ks"], h].T[:tail]])
            k = torch.cat([k, s["tree_k"][r, :n, h]]).double()
            v = torch.cat([v, s["tree_v"][r, :n, h]]).double()
            kt = k.T.contiguous()
            for g in range(G):
                z = s["q"][r, :n, h * G + g].double() @ kt / math.sqrt(D)
                z[:, k.shape[0] - n:][~see] = -math.inf
                e = torch.logsumexp(z, -1)
                out[r, :n, h * G + g] = (torch.exp(z - e[:, None]) @ v).cpu()
                lse[r, :n, h * G + g] = e.cpu()
    return [out, lse]


def _exact_verify(c, s):
    R, T, V = c["R"], c["T"], c["V"]
    path, count, toks = np.full((R, T), -1), np.zeros(R, int), np.full((R, T), -1)
    parent, tokens = s["parent"].cpu().numpy(), s["tokens"].cpu().numpy()
    length, us = s["len"].tolist(), s["sample_u"].double().cpu().numpy()
    ua = s["accept_u"].double().cpu().numpy()
    for r in range(R):
        if length[r] < 1:
            continue
        node, rows, emitted = 0, [0], []
        while True:
            w = s["target"][r, node].double().cpu().numpy()
            q = None if s["draft"] is None else s["draft"][r, node].double().cpu().numpy()
            whole, mass, found = w, 1.0, None
            for t in range(node + 1, length[r]):
                if parent[r, t] != node:
                    continue
                x = tokens[r, t]
                if ua[r, t] * (1.0 if q is None else q[x]) * mass < w[x]:
                    found = t
                    break
                if q is None:
                    mass, w = mass - w[x], w.copy()
                    w[x] = 0.0
                else:
                    w = np.maximum(w - mass * q, 0.0)
                    mass = math.fsum(w)
            if found is None:
                break
            node = found
            rows.append(node)
            emitted.append(tokens[r, node])
        if not w.sum() > 0:
            w = whole
        emitted.append(int(np.argmax(np.cumsum(w) > us[r] * math.fsum(w))))
        path[r, :len(rows)], toks[r, :len(emitted)], count[r] = rows, emitted, len(rows)
    return [torch.from_numpy(a.astype(np.int32)) for a in (path, count, toks)]


def _exact_append(c, s):
    k, v, B = s["k"].clone(), s["v"].clone(), c["B"]
    ctx = s["ctx"].tolist()
    ends = []
    for r in range(c["R"]):
        rows = list(range(c["T"])) if s["path"] is None else s["path"][r, :int(s["path_len"][r])].tolist()
        i = 0
        while i < len(rows):  # the tokens that fall into one block
            b, o = divmod(ctx[r] + i, B)
            n = min(B - o, len(rows) - i)
            page = int(s["table"][r, b])
            k[page, :, o:o + n] = s["new_k"][r, rows[i:i + n]].transpose(0, 1)
            v[page, :, o:o + n] = s["new_v"][r, rows[i:i + n]].transpose(0, 1)
            i += n
        ends.append(ctx[r] + len(rows))
    return [k.double(), v.double(), torch.tensor(ends, dtype=torch.int32)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("tree", "sparse"):
        # about 1e12 operations a second in 64 bits, and some 40 us for each of the loops' turns
        if work(case)["flops"] / 1e12 + case["R"] * case["Hq"] * 3e-4 > 15:
            return None
        return _exact_attn(case, s)
    return _exact_verify(case, s) if case["kind"] == "verify" else _exact_append(case, s)
