"""Decode path over a cache that stays in HBM at four bits: no host tier and no working set.

Paper §4.2.1 ranks blocks from the draft queries and attends the best of them; here the selected blocks are read where
they lie in the 4-bit pages, so that nothing is staged (§4.2.3) and a step attends its own selection. This module owns
the buffers of the layers and issues the library calls in order; every computation happens in liboasis.so (through
``_lib``).
"""
from __future__ import annotations

import math

import torch

from . import _lib as L


class Q4Layer:
    """Pages, compressed keys, selection and outputs of one layer."""

    def __init__(self, d: L.OasisDims, num_q_tokens: int, k: int, num_pages: int, device: str | torch.device = "cuda"):
        R, Hq, Hkv, D, NB = d.num_reqs, d.num_q_heads, d.num_kv_heads, d.head_dim, d.max_blocks
        dev, bf, i32 = torch.device(device), torch.bfloat16, torch.int32
        page = L.oasis_q4_page_bytes(d)
        self.k_pages = torch.zeros((num_pages, page), dtype=torch.uint8, device=dev)
        self.v_pages = torch.zeros((num_pages, page), dtype=torch.uint8, device=dev)
        self.kmax = torch.empty((R, Hkv, NB, D), dtype=bf, device=dev)
        self.kmin = torch.empty((R, Hkv, NB, D), dtype=bf, device=dev)
        self.scores = torch.empty((R, Hkv, NB), dtype=torch.float32, device=dev)
        self.sel = torch.full((R, Hkv, k), -1, dtype=i32, device=dev)
        self.sel_count = torch.zeros((R, Hkv), dtype=i32, device=dev)
        self.out = torch.empty((R, num_q_tokens, Hq, D), dtype=bf, device=dev)
        self.lse = torch.empty((R, num_q_tokens, Hq), dtype=torch.float32, device=dev)


class Q4Path:
    """Issues append -> (rotate -> predict -> attend) -> commit for layers on 4-bit pages.

    ``block_table`` is the device page table ``[R][NBmax]`` of every layer; two requests may share pages that neither
    appends to. ``rotary`` (None: keys and queries come with their positions) turns the keys that ``append`` writes and the
    rows that ``rotate`` is given. ``predict`` ranks blocks from the ``num_draft`` rows from ``first_draft`` on: by default
    from all but the first, or a step's only one, as many as the scorer takes (64 with the heads that share a KV head). The
    layers' calls share one workspace and one pair of rotated rows, so they must run in order, on one stream or behind
    each other's events.
    """

    def __init__(self, d: L.OasisDims, num_q_tokens: int, k: int, num_pages: int, block_table: torch.Tensor,
                 rotary: L.Rotary | None = None, first_draft: int | None = None, num_draft: int | None = None,
                 scale: float | None = None):
        self.dims, self.T, self.k, self.num_pages = d, int(num_q_tokens), int(k), int(num_pages)
        self.block_table, self.rotary = block_table, rotary
        self.first_draft = int(first_draft if first_draft is not None else self.T > 1)
        most = max(1, 64 // (d.num_q_heads // d.num_kv_heads))  # (more heads: the scorer says so)
        self.num_draft = int(num_draft if num_draft is not None else min(self.T - self.first_draft, most))
        self.scale = scale if scale is not None else 1.0 / math.sqrt(d.head_dim)
        dev = block_table.device
        need = max(L.oasis_tree_attn_q4_workspace_bytes(d, self.T, self.k), L.oasis_tree_attn_q4_workspace_bytes(d, self.T, 0))
        self.ws = torch.empty(need, dtype=torch.uint8, device=dev)
        # the step's rotated query and key rows
        self.q = torch.empty((d.num_reqs, self.T, d.num_q_heads, d.head_dim), dtype=torch.bfloat16, device=dev)
        self.tree_k = torch.empty((d.num_reqs, self.T, d.num_kv_heads, d.head_dim), dtype=torch.bfloat16, device=dev)

    def new_layer(self) -> Q4Layer:
        return Q4Layer(self.dims, self.T, self.k, self.num_pages, self.block_table.device)

    def append(self, st: Q4Layer, new_k: torch.Tensor, new_v: torch.Tensor, ctx_len: torch.Tensor, new_ctx_len: torch.Tensor,
               lengths: torch.Tensor | None = None, read_k: torch.Tensor | None = None, read_v: torch.Tensor | None = None,
               stream=None):
        """A chunk of new rows [R][N][Hkv][d] (of request r the first ``lengths[r]``, None: all) at ``ctx_len``: rotated,
        quantised and written, the lengths that follow, and the compressed keys of the blocks that it completes.
        ``read_k`` and ``read_v`` receive the rows as the cache holds them."""
        n = int(new_k.shape[1])
        L.oasis_append_tokens_q4(self.dims, self.rotary, new_k, new_v, n, None, lengths, st.k_pages, st.v_pages,
                                 self.block_table, ctx_len, new_ctx_len, read_k, read_v, stream)
        self._summaries(st, ctx_len, new_ctx_len, n, stream)

    def _summaries(self, st: Q4Layer, ctx_len, new_ctx_len, n: int, stream):
        L.oasis_update_summaries_q4(self.dims, st.k_pages, self.block_table, ctx_len, new_ctx_len,
                                    -(-n // self.dims.block_size), st.kmax, st.kmin, stream)

    def rotate(self, q: torch.Tensor, k: torch.Tensor, ctx_len: torch.Tensor, positions: torch.Tensor | None = None,
               stream=None) -> tuple[torch.Tensor, torch.Tensor]:
        """The step's query rows [R][T][Hq][d] and key rows [R][T][Hkv][d] at their positions (int32 [R][T]; None: a chain
        from ``ctx_len`` on), in buffers that the next call writes again; without a rotary table they are as given."""
        if self.rotary is None:
            return q, k
        L.oasis_rotate(self.dims, self.rotary, self.T, positions, ctx_len, q, self.q, k, self.tree_k, False, stream)
        return self.q, self.tree_k

    def predict(self, st: Q4Layer, q: torch.Tensor, ctx_len: torch.Tensor, stream=None):
        """Rank the layer's blocks from the draft rows of q and select the best ones of each KV head."""
        L.oasis_score_blocks(self.dims, q, self.T, self.first_draft, self.num_draft, st.kmax, st.kmin, ctx_len, st.scores,
                             stream)
        L.oasis_select_topk(self.dims, st.scores, ctx_len, self.k, st.sel, st.sel_count, stream)

    def attend(self, st: Q4Layer, q: torch.Tensor, ctx_len: torch.Tensor, tree_k: torch.Tensor | None = None,
               tree_v: torch.Tensor | None = None, parent: torch.Tensor | None = None, tree_len: torch.Tensor | None = None,
               stream=None):
        """Attention of the T rows over the layer's selection and local block, and (tree_k, tree_v) over the rows on their
        own path, into ``st.out`` and ``st.lse``."""
        L.oasis_tree_attn_q4(self.dims, q, self.T, st.k_pages, st.v_pages, self.block_table, ctx_len, st.sel, st.sel_count,
                             self.k, tree_k, tree_v, parent, tree_len, self.scale, st.out, st.lse, self.ws, stream)

    def attend_dense(self, st: Q4Layer, q: torch.Tensor, ctx_len: torch.Tensor, tree_k: torch.Tensor | None = None,
                     tree_v: torch.Tensor | None = None, parent: torch.Tensor | None = None,
                     tree_len: torch.Tensor | None = None, stream=None):
        """The same over every cached token."""
        L.oasis_tree_attn_q4(self.dims, q, self.T, st.k_pages, st.v_pages, self.block_table, ctx_len, None, None, 0, tree_k,
                             tree_v, parent, tree_len, self.scale, st.out, st.lse, self.ws, stream)

    def commit(self, st: Q4Layer, tree_k: torch.Tensor, tree_v: torch.Tensor, path: torch.Tensor | None,
               path_len: torch.Tensor | None, ctx_len: torch.Tensor, new_ctx_len: torch.Tensor, stream=None):
        """Append the accepted rows (``path``, as the verification gives it; None: all T, a chain) with keys that are
        rotated already, write the lengths that follow, and bring the compressed keys up to them."""
        L.oasis_append_tokens_q4(self.dims, None, tree_k, tree_v, self.T, path, path_len, st.k_pages, st.v_pages,
                                 self.block_table, ctx_len, new_ctx_len, None, None, stream)
        self._summaries(st, ctx_len, new_ctx_len, self.T, stream)
