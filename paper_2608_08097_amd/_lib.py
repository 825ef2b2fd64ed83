"""ctypes binding of liboasis.so: the C ABI declared in include/oasis.h, one
Python function per entry point, with the same names.

Marshalling only: the functions check that tensors sit where the C ABI expects
them (device or pinned host), have the right dtype and are contiguous, then
pass raw pointers and the current HIP stream. Every step of the path runs in
the library's kernels; there is no fallback. If the library is not built, the
first call raises.

The calls a decode step makes many times first go to ``_fastcall`` (built
beside the library), which makes the same checks and the call natively and
returns None for arguments it does not accept as they are; those, and every
error, take the Python code below it. So does every call, with a warning when
the library is loaded, where ``_fastcall`` is missing or does not fit.
"""
from __future__ import annotations

import ctypes
import math
import os
import warnings

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "liboasis.so")

STATUS = {0: "OASIS_OK", 1: "OASIS_ERR_INVALID_ARG", 2: "OASIS_ERR_UNSUPPORTED",
          3: "OASIS_ERR_HIP", 4: "OASIS_ERR_WORKSPACE"}

EXPORTS = (
    "oasis_last_error", "oasis_abi_version", "oasis_build_summaries", "oasis_update_summaries",
    "oasis_copy_blocks", "oasis_score_blocks", "oasis_score_select",
    "oasis_select_topk", "oasis_stage_blocks",
    "oasis_attn_workspace_bytes", "oasis_sparse_decode_attn", "oasis_sparse_decode_attn_noalloc",
    "oasis_union_selection",
    "oasis_tree_attn_workspace_bytes", "oasis_tree_attn", "oasis_sparse_tree_attn_workspace_bytes",
    "oasis_sparse_tree_attn", "oasis_verify_workspace_bytes", "oasis_verify_drafts", "oasis_append_tokens",
    "oasis_q4_page_bytes", "oasis_rotary_turns", "oasis_rotate", "oasis_append_tokens_q4", "oasis_update_summaries_q4",
    "oasis_tree_attn_q4_workspace_bytes", "oasis_tree_attn_q4",
    "oasis_pipeline_create", "oasis_pipeline_set_layer", "oasis_pipeline_set_local_source",
    "oasis_pipeline_set_plan_stream", "oasis_pipeline_set_fused_prediction", "oasis_pipeline_step",
    "oasis_pipeline_join", "oasis_pipeline_check", "oasis_pipeline_set_wait_limit",
    "oasis_pipeline_set_prediction_order",
    "oasis_pipeline_destroy", "oasis_pipeline_profile_begin", "oasis_pipeline_profile_end",
)


class OasisError(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__(f"{fn}: {STATUS.get(status, status)}: {msg}")
        self.status = status


class OasisDims(ctypes.Structure):
    _fields_ = [("num_reqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("max_blocks", ctypes.c_int32)]

    def __repr__(self):
        return "OasisDims(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class OasisLayerBuffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("kmax", "kmin", "scores", "sel", "sel_count", "slot_map",
                                               "slot_stamp", "pool_k", "pool_v", "moved", "out", "lse",
                                               "workspace")] + [("workspace_bytes", ctypes.c_size_t)]


class OasisRotary(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("amplitude", ctypes.c_double)]


def dims(num_reqs, num_q_heads, num_kv_heads, head_dim, block_size, max_blocks) -> OasisDims:
    return OasisDims(int(num_reqs), int(num_q_heads), int(num_kv_heads), int(head_dim), int(block_size),
                     int(max_blocks))


_lib = None
_fast = None  # the _fastcall module, bound to the loaded library (None: calls are marshalled in Python)
_BUILD_HINT = "Build it with __graft_entry__.build() or python -m paper_2608_08097_amd.build_lib"
ABI_VERSION = 7  # OASIS_ABI_VERSION of include/oasis.h

_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_DIMS = ctypes.POINTER(OasisDims)


def lib() -> ctypes.CDLL:
    """Load liboasis.so (once); raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing. {_BUILD_HINT}")
        L = ctypes.CDLL(LIB_PATH)
        L.oasis_last_error.restype = ctypes.c_char_p
        L.oasis_last_error.argtypes = []
        L.oasis_abi_version.restype = _I32
        L.oasis_abi_version.argtypes = []
        if L.oasis_abi_version() != ABI_VERSION:
            raise RuntimeError(f"{LIB_PATH} has ABI version {L.oasis_abi_version()}, this binding expects "
                               f"{ABI_VERSION}: rebuild it")
        L.oasis_build_summaries.restype = _I32
        L.oasis_build_summaries.argtypes = [_DIMS, _P, _I64, _P, _P, _P, _P, _P]
        L.oasis_update_summaries.restype = _I32
        L.oasis_update_summaries.argtypes = [_DIMS, _P, _I64, _P, _P, _P, _I32, _P, _P, _P]
        L.oasis_copy_blocks.restype = _I32
        L.oasis_copy_blocks.argtypes = [_DIMS, _P, _P, _I64, _P, _P, _P, _I64, _P, _P, _P, _I32, _P]
        L.oasis_score_blocks.restype = _I32
        L.oasis_score_blocks.argtypes = [_DIMS, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P]
        L.oasis_select_topk.restype = _I32
        L.oasis_select_topk.argtypes = [_DIMS, _P, _P, _I32, _P, _P, _P]
        L.oasis_stage_blocks.restype = _I32
        L.oasis_stage_blocks.argtypes = [_DIMS, _P, _P, _I64, _P, _P, _P, _P, _P, _I32, _P, _P, _I32, _I32, _I32,
                                         _P, _P, _P, _P]
        L.oasis_score_select.restype = _I32
        L.oasis_score_select.argtypes = [_DIMS, _P, _I32, _I32, _I32, _P, _P, _P, _I32, _P, _P, _P, _P]
        L.oasis_union_selection.restype = _I32
        L.oasis_union_selection.argtypes = [_DIMS, _P, _P, _I32, _P, _P, _P]
        L.oasis_attn_workspace_bytes.restype = _SZ
        L.oasis_attn_workspace_bytes.argtypes = [_DIMS, _I32, _I32]
        L.oasis_sparse_decode_attn.restype = _I32
        L.oasis_sparse_decode_attn.argtypes = [_DIMS, _P, _I32, _P, _P, _P, _I32, _P, ctypes.c_float, _P, _P,
                                               _P, _SZ, _P]
        L.oasis_sparse_decode_attn_noalloc.restype = _I32
        L.oasis_sparse_decode_attn_noalloc.argtypes = [_DIMS, _P, _I32, _P, _P, _P, _I32, _P, ctypes.c_float, _P,
                                                       _P, _P]
        L.oasis_tree_attn_workspace_bytes.restype = _SZ
        L.oasis_tree_attn_workspace_bytes.argtypes = [_DIMS, _I32]
        L.oasis_tree_attn.restype = _I32
        L.oasis_tree_attn.argtypes = [_DIMS, _P, _I32, _P, _P, _I64, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P,
                                      _SZ, _P]
        L.oasis_sparse_tree_attn_workspace_bytes.restype = _SZ
        L.oasis_sparse_tree_attn_workspace_bytes.argtypes = [_DIMS, _I32, _I32]
        L.oasis_sparse_tree_attn.restype = _I32
        L.oasis_sparse_tree_attn.argtypes = [_DIMS, _P, _I32, _P, _P, _P, _I32, _P, _P, _P, _P, _P, ctypes.c_float, _P,
                                             _P, _P, _SZ, _P]
        L.oasis_verify_workspace_bytes.restype = _SZ
        L.oasis_verify_workspace_bytes.argtypes = [_I32, _I32, _I32]
        L.oasis_verify_drafts.restype = _I32
        L.oasis_verify_drafts.argtypes = [_I32, _I32, _I32, _P, _I64, _P, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ,
                                          _P]
        L.oasis_append_tokens.restype = _I32
        L.oasis_append_tokens.argtypes = [_DIMS, _P, _P, _I32, _P, _P, _P, _P, _I64, _P, _P, _P, _P]
        rot, f64 = ctypes.POINTER(OasisRotary), ctypes.c_double
        L.oasis_q4_page_bytes.restype = _SZ
        L.oasis_q4_page_bytes.argtypes = [_DIMS]
        L.oasis_rotary_turns.restype = _I32
        L.oasis_rotary_turns.argtypes = [_I32, f64, _I32, f64, f64, f64, f64, _P, ctypes.POINTER(f64)]
        L.oasis_rotate.restype = _I32
        L.oasis_rotate.argtypes = [_DIMS, rot, _I32, _P, _P, _I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]
        L.oasis_append_tokens_q4.restype = _I32
        L.oasis_append_tokens_q4.argtypes = [_DIMS, rot, _P, _I64, _P, _I64, _I32, _P, _P, _P, _P, _I64, _P, _P, _P, _P,
                                             _P, _P]
        L.oasis_update_summaries_q4.restype = _I32
        L.oasis_update_summaries_q4.argtypes = [_DIMS, _P, _I64, _P, _P, _P, _I32, _P, _P, _P]
        L.oasis_tree_attn_q4_workspace_bytes.restype = _SZ
        L.oasis_tree_attn_q4_workspace_bytes.argtypes = [_DIMS, _I32, _I32]
        L.oasis_tree_attn_q4.restype = _I32
        L.oasis_tree_attn_q4.argtypes = [_DIMS, _P, _I32, _P, _P, _I64, _P, _P, _P, _P, _I32, _P, _P, _P, _P,
                                         ctypes.c_float, _P, _P, _P, _SZ, _P]
        L.oasis_pipeline_create.restype = _I32
        L.oasis_pipeline_create.argtypes = [_DIMS, _I32, _I32, _I32, _I32, _I32, ctypes.c_float, _P, _P, _I64, _P,
                                            _I32, _P, _P, ctypes.POINTER(_P)]
        L.oasis_pipeline_set_fused_prediction.restype = _I32
        L.oasis_pipeline_set_fused_prediction.argtypes = [_P, _I32]
        L.oasis_pipeline_set_layer.restype = _I32
        L.oasis_pipeline_set_layer.argtypes = [_P, _I32, ctypes.POINTER(OasisLayerBuffers)]
        L.oasis_pipeline_set_local_source.restype = _I32
        L.oasis_pipeline_set_local_source.argtypes = [_P, _P, _P, _I64, _P]
        L.oasis_pipeline_set_plan_stream.restype = _I32
        L.oasis_pipeline_set_plan_stream.argtypes = [_P, _I32]
        L.oasis_pipeline_step.restype = _I32
        L.oasis_pipeline_step.argtypes = [_P, _I32, _P, _P, _P, _I32, _I32, _I32, _P, _P]
        L.oasis_pipeline_join.restype = _I32
        L.oasis_pipeline_join.argtypes = [_P, _P]
        L.oasis_pipeline_check.restype = _I32
        L.oasis_pipeline_check.argtypes = [_P]
        L.oasis_pipeline_set_prediction_order.restype = _I32
        L.oasis_pipeline_set_prediction_order.argtypes = [_P, _I32]
        L.oasis_pipeline_set_wait_limit.restype = _I32
        L.oasis_pipeline_set_wait_limit.argtypes = [_P, ctypes.c_uint32]
        L.oasis_pipeline_destroy.restype = None
        L.oasis_pipeline_destroy.argtypes = [_P]
        L.oasis_pipeline_profile_begin.restype = _I32
        L.oasis_pipeline_profile_begin.argtypes = [_P, _I32]
        L.oasis_pipeline_profile_end.restype = _I32
        L.oasis_pipeline_profile_end.argtypes = [_P, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float),
                                                   ctypes.POINTER(_I32)]
        _bind_fast(L)
        _lib = L
    return _lib


def _load_fast():
    from . import _fastcall
    return _fastcall


def _bind_fast(L: ctypes.CDLL) -> None:
    """Point the native marshalling at the entry points of the loaded library. Without a module that fits it
    (not built, built for another PyTorch, or left over from another ABI version) every call is marshalled by
    the Python code below: the same kernels and results, some microseconds more of host time a call."""
    global _fast
    _fast = None
    try:
        fast = _load_fast()
        built_for = fast.abi_version
        fits = built_for == ABI_VERSION
        bind_drafts, bind_q4 = (fast.bind_drafts, fast.bind_q4) if fits else (None, None)
    except (ImportError, AttributeError) as e:
        warnings.warn(f"native marshalling not loaded ({e}): calls go through the slower Python binding. {_BUILD_HINT}",
                      RuntimeWarning, stacklevel=2)
        return
    if built_for != ABI_VERSION:
        warnings.warn(f"{fast.__file__} was built for ABI version {built_for}, the library has {ABI_VERSION}: calls "
                      f"go through the slower Python binding. {_BUILD_HINT}", RuntimeWarning, stacklevel=2)
        return
    fast.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.oasis_sparse_decode_attn, L.oasis_score_blocks, L.oasis_select_topk, L.oasis_score_select,
        L.oasis_stage_blocks)))
    bind_drafts(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.oasis_tree_attn, L.oasis_sparse_tree_attn, L.oasis_verify_drafts, L.oasis_append_tokens)))
    bind_q4(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.oasis_rotate, L.oasis_append_tokens_q4, L.oasis_update_summaries_q4, L.oasis_tree_attn_q4)))
    _fast = fast


def _handle(stream):
    """The stream as the native marshalling takes it: a handle, or None for the current stream."""
    return None if stream is None else _stream(stream)


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise OasisError(fn, status, lib().oasis_last_error().decode())


def _stream(stream) -> int | None:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _dev(t: torch.Tensor | None, name: str, dtypes, nullable: bool = False):
    if t is None:
        if nullable:
            return None
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype} not in {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _host_or_dev(t: torch.Tensor, name: str, dtypes):
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype} not in {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if not t.is_cuda and not t.is_pinned():
        raise ValueError(f"{name} must be pinned host memory or a device tensor")
    return t.data_ptr()


def _need(t: torch.Tensor | None, numel: int, name: str) -> None:
    """Element count the C ABI will address for this argument (no kernel may go past it)."""
    if t is not None and t.numel() != numel:
        raise ValueError(f"{name}: {t.numel()} elements, {numel} expected")


_BF16 = (torch.bfloat16, torch.uint16, torch.int16)
_I32T = (torch.int32,)
_F32 = (torch.float32,)


def oasis_abi_version() -> int:
    return int(lib().oasis_abi_version())


def oasis_last_error() -> str:
    return lib().oasis_last_error().decode()


def oasis_build_summaries(d: OasisDims, k_pages, block_table, ctx_len, kmax, kmin, stream=None) -> None:
    R, H, NB, D = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim
    _need(k_pages, k_pages.shape[0] * H * d.block_size * D, "k_pages")
    _need(block_table, R * NB, "block_table")
    _need(ctx_len, R, "ctx_len")
    _need(kmax, R * H * NB * D, "kmax")
    _need(kmin, R * H * NB * D, "kmin")
    _check("oasis_build_summaries", lib().oasis_build_summaries(
        ctypes.byref(d), _host_or_dev(k_pages, "k_pages", _BF16), int(k_pages.shape[0]),
        _dev(block_table, "block_table", _I32T), _dev(ctx_len, "ctx_len", _I32T),
        _dev(kmax, "kmax", _BF16), _dev(kmin, "kmin", _BF16), _stream(stream)))


def oasis_update_summaries(d: OasisDims, k_pages, block_table, prev_ctx_len, ctx_len, max_new_blocks: int,
                           kmax, kmin, stream=None) -> None:
    R, H, NB, D = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim
    _need(k_pages, k_pages.shape[0] * H * d.block_size * D, "k_pages")
    _need(block_table, R * NB, "block_table")
    _need(prev_ctx_len, R, "prev_ctx_len")
    _need(ctx_len, R, "ctx_len")
    _need(kmax, R * H * NB * D, "kmax")
    _need(kmin, R * H * NB * D, "kmin")
    _check("oasis_update_summaries", lib().oasis_update_summaries(
        ctypes.byref(d), _host_or_dev(k_pages, "k_pages", _BF16), int(k_pages.shape[0]),
        _dev(block_table, "block_table", _I32T), _dev(prev_ctx_len, "prev_ctx_len", _I32T),
        _dev(ctx_len, "ctx_len", _I32T), int(max_new_blocks), _dev(kmax, "kmax", _BF16), _dev(kmin, "kmin", _BF16),
        _stream(stream)))


def oasis_copy_blocks(d: OasisDims, src_k, src_v, src_block_table, dst_k, dst_v, dst_block_table, prev_ctx_len,
                      ctx_len, max_blocks: int, stream=None) -> None:
    R, H, NB, D, B = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim, d.block_size
    for t, name in ((src_k, "src_k"), (src_v, "src_v"), (dst_k, "dst_k"), (dst_v, "dst_v")):
        if t.dim() < 1 or t.numel() % (H * B * D):
            raise ValueError(f"{name}: not whole pages of [Hkv][B][d]")
    if src_k.shape != src_v.shape or dst_k.shape != dst_v.shape:
        raise ValueError("K and V tiers differ in shape")
    _need(src_block_table, R * NB, "src_block_table")
    _need(dst_block_table, R * NB, "dst_block_table")
    _need(prev_ctx_len, R, "prev_ctx_len")
    _need(ctx_len, R, "ctx_len")
    _check("oasis_copy_blocks", lib().oasis_copy_blocks(
        ctypes.byref(d), _host_or_dev(src_k, "src_k", _BF16), _host_or_dev(src_v, "src_v", _BF16),
        src_k.numel() // (H * B * D), _dev(src_block_table, "src_block_table", _I32T),
        _host_or_dev(dst_k, "dst_k", _BF16), _host_or_dev(dst_v, "dst_v", _BF16), dst_k.numel() // (H * B * D),
        _dev(dst_block_table, "dst_block_table", _I32T), _dev(prev_ctx_len, "prev_ctx_len", _I32T, nullable=True),
        _dev(ctx_len, "ctx_len", _I32T), int(max_blocks), _stream(stream)))


def oasis_score_blocks(d: OasisDims, q, num_q_tokens: int, first_draft: int, num_draft: int,
                       kmax, kmin, ctx_len, scores, stream=None) -> None:
    if _fast is not None and type(d) is OasisDims:
        st = _fast.score_blocks(ctypes.addressof(d), q, num_q_tokens, first_draft, num_draft, kmax, kmin, ctx_len,
                                scores, _handle(stream))
        if st is not None:
            return _check("oasis_score_blocks", st)
    R, H, NB, D = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim
    _need(q, R * num_q_tokens * d.num_q_heads * D, "q")
    _need(kmax, R * H * NB * D, "kmax")
    _need(kmin, R * H * NB * D, "kmin")
    _need(ctx_len, R, "ctx_len")
    _need(scores, R * H * NB, "scores")
    _check("oasis_score_blocks", lib().oasis_score_blocks(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), int(first_draft), int(num_draft),
        _dev(kmax, "kmax", _BF16), _dev(kmin, "kmin", _BF16), _dev(ctx_len, "ctx_len", _I32T),
        _dev(scores, "scores", _F32), _stream(stream)))


def oasis_select_topk(d: OasisDims, scores, ctx_len, k: int, sel, sel_count, stream=None) -> None:
    if _fast is not None and type(d) is OasisDims:
        st = _fast.select_topk(ctypes.addressof(d), scores, ctx_len, k, sel, sel_count, _handle(stream))
        if st is not None:
            return _check("oasis_select_topk", st)
    R, H = d.num_reqs, d.num_kv_heads
    _need(scores, R * H * d.max_blocks, "scores")
    _need(ctx_len, R, "ctx_len")
    _need(sel, R * H * k, "sel")
    _need(sel_count, R * H, "sel_count")
    _check("oasis_select_topk", lib().oasis_select_topk(
        ctypes.byref(d), _dev(scores, "scores", _F32), _dev(ctx_len, "ctx_len", _I32T), int(k),
        _dev(sel, "sel", _I32T), _dev(sel_count, "sel_count", _I32T), _stream(stream)))


def oasis_score_select(d: OasisDims, q, num_q_tokens: int, first_draft: int, num_draft: int, kmax, kmin, ctx_len,
                       k: int, scores, sel, sel_count, stream=None) -> None:
    """Scores and top-K in one kernel (the same results as oasis_score_blocks + oasis_select_topk)."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.score_select(ctypes.addressof(d), q, num_q_tokens, first_draft, num_draft, kmax, kmin, ctx_len, k,
                                scores, sel, sel_count, _handle(stream))
        if st is not None:
            return _check("oasis_score_select", st)
    R, H, NB, D = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim
    _need(q, R * num_q_tokens * d.num_q_heads * D, "q")
    _need(kmax, R * H * NB * D, "kmax")
    _need(kmin, R * H * NB * D, "kmin")
    _need(ctx_len, R, "ctx_len")
    _need(scores, R * H * NB, "scores")
    _need(sel, R * H * k, "sel")
    _need(sel_count, R * H, "sel_count")
    _check("oasis_score_select", lib().oasis_score_select(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), int(first_draft), int(num_draft),
        _dev(kmax, "kmax", _BF16), _dev(kmin, "kmin", _BF16), _dev(ctx_len, "ctx_len", _I32T), int(k),
        _dev(scores, "scores", _F32), _dev(sel, "sel", _I32T), _dev(sel_count, "sel_count", _I32T),
        _stream(stream)))


def oasis_stage_blocks(d: OasisDims, host_k, host_v, host_block_table, ctx_len, sel, sel_count, scores, k: int,
                       slot_map, slot_stamp, step: int, fetch_cap: int, copy_local: bool, pool_k, pool_v,
                       moved, stream=None) -> None:
    if host_k.shape != host_v.shape:
        raise ValueError("host_k and host_v differ in shape")
    if _fast is not None and type(d) is OasisDims:
        st = _fast.stage_blocks(ctypes.addressof(d), host_k, host_v, host_k.shape[0], host_block_table, ctx_len, sel,
                                sel_count, scores, k, slot_map, slot_stamp, step, fetch_cap, copy_local, pool_k,
                                pool_v, moved, _handle(stream))
        if st is not None:
            return _check("oasis_stage_blocks", st)
    R, H, B, D = d.num_reqs, d.num_kv_heads, d.block_size, d.head_dim
    _need(host_k, host_k.shape[0] * H * B * D, "host_k")
    _need(host_block_table, R * d.max_blocks, "host_block_table")
    _need(ctx_len, R, "ctx_len")
    for t, n in ((sel, "sel"), (slot_map, "slot_map"), (slot_stamp, "slot_stamp")):
        _need(t, R * H * k, n)
    _need(sel_count, R * H, "sel_count")
    _need(scores, R * H * d.max_blocks, "scores")
    _need(moved, R * H, "moved")
    _need(pool_k, R * (k + 1) * H * B * D, "pool_k")
    _need(pool_v, R * (k + 1) * H * B * D, "pool_v")
    _check("oasis_stage_blocks", lib().oasis_stage_blocks(
        ctypes.byref(d), _host_or_dev(host_k, "host_k", _BF16), _host_or_dev(host_v, "host_v", _BF16),
        int(host_k.shape[0]), _dev(host_block_table, "host_block_table", _I32T), _dev(ctx_len, "ctx_len", _I32T),
        _dev(sel, "sel", _I32T, nullable=True), _dev(sel_count, "sel_count", _I32T, nullable=True),
        _dev(scores, "scores", (torch.float32,), nullable=True), int(k),
        _dev(slot_map, "slot_map", _I32T, nullable=True), _dev(slot_stamp, "slot_stamp", _I32T, nullable=True),
        int(step), int(fetch_cap), 1 if copy_local else 0, _dev(pool_k, "pool_k", _BF16),
        _dev(pool_v, "pool_v", _BF16), _dev(moved, "moved", _I32T, nullable=True), _stream(stream)))


def oasis_union_selection(d: OasisDims, sel, sel_count, k: int, union_ids, union_count, stream=None) -> None:
    R, H = d.num_reqs, d.num_kv_heads
    _need(sel, R * H * k, "sel")
    _need(sel_count, R * H, "sel_count")
    _need(union_ids, R * H * k, "union_ids")
    _need(union_count, R, "union_count")
    _check("oasis_union_selection", lib().oasis_union_selection(
        ctypes.byref(d), _dev(sel, "sel", _I32T), _dev(sel_count, "sel_count", _I32T), int(k),
        _dev(union_ids, "union_ids", _I32T), _dev(union_count, "union_count", _I32T), _stream(stream)))


def oasis_attn_workspace_bytes(d: OasisDims, num_q_tokens: int, k_slots: int) -> int:
    return int(lib().oasis_attn_workspace_bytes(ctypes.byref(d), int(num_q_tokens), int(k_slots)))


def oasis_sparse_decode_attn(d: OasisDims, q, num_q_tokens: int, pool_k, pool_v, slot_map, k_slots: int,
                             ctx_len, scale: float | None, out, lse, workspace, stream=None) -> None:
    if _fast is not None and type(d) is OasisDims:
        st = _fast.sparse_decode_attn(ctypes.addressof(d), q, num_q_tokens, pool_k, pool_v, slot_map, k_slots, ctx_len,
                                      scale, out, lse, workspace, _handle(stream))
        if st is not None:
            return _check("oasis_sparse_decode_attn", st)
    if scale is None:
        scale = 1.0 / math.sqrt(d.head_dim)
    R, H, B, D = d.num_reqs, d.num_kv_heads, d.block_size, d.head_dim
    _need(q, R * num_q_tokens * d.num_q_heads * D, "q")
    _need(out, R * num_q_tokens * d.num_q_heads * D, "out")
    _need(lse, R * num_q_tokens * d.num_q_heads, "lse")
    _need(pool_k, R * (k_slots + 1) * H * B * D, "pool_k")
    _need(pool_v, R * (k_slots + 1) * H * B * D, "pool_v")
    _need(slot_map, R * H * k_slots, "slot_map")
    _need(ctx_len, R, "ctx_len")
    _check("oasis_sparse_decode_attn", lib().oasis_sparse_decode_attn(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), _dev(pool_k, "pool_k", _BF16),
        _dev(pool_v, "pool_v", _BF16), _dev(slot_map, "slot_map", _I32T, nullable=k_slots == 0), int(k_slots),
        _dev(ctx_len, "ctx_len", _I32T), float(scale), _dev(out, "out", _BF16),
        _dev(lse, "lse", _F32, nullable=True),
        _dev(workspace, "workspace", (torch.uint8,), nullable=workspace is None or workspace.numel() == 0),
        int(workspace.numel()) if workspace is not None else 0, _stream(stream)))


NOALLOC_SCRATCH_BYTES = 16 << 20  # OASIS_NOALLOC_SCRATCH_BYTES of include/oasis.h


def oasis_sparse_decode_attn_noalloc(d: OasisDims, q, num_q_tokens: int, pool_k, pool_v, slot_map, k_slots: int,
                                     ctx_len, scale: float | None, out, lse, stream=None) -> None:
    """oasis_sparse_decode_attn with the library's own scratch instead of a workspace (allocates nothing)."""
    if scale is None:
        scale = 1.0 / math.sqrt(d.head_dim)
    R, H, B, D = d.num_reqs, d.num_kv_heads, d.block_size, d.head_dim
    _need(q, R * num_q_tokens * d.num_q_heads * D, "q")
    _need(out, R * num_q_tokens * d.num_q_heads * D, "out")
    _need(lse, R * num_q_tokens * d.num_q_heads, "lse")
    _need(pool_k, R * (k_slots + 1) * H * B * D, "pool_k")
    _need(pool_v, R * (k_slots + 1) * H * B * D, "pool_v")
    _need(slot_map, R * H * k_slots, "slot_map")
    _need(ctx_len, R, "ctx_len")
    _check("oasis_sparse_decode_attn_noalloc", lib().oasis_sparse_decode_attn_noalloc(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), _dev(pool_k, "pool_k", _BF16),
        _dev(pool_v, "pool_v", _BF16), _dev(slot_map, "slot_map", _I32T, nullable=k_slots == 0), int(k_slots),
        _dev(ctx_len, "ctx_len", _I32T), float(scale), _dev(out, "out", _BF16),
        _dev(lse, "lse", _F32, nullable=True), _stream(stream)))


# --- speculative step ----------------------------------------------------------


def _one_device(**tensors) -> None:
    """The device tensors of a call are all on the current device, whose stream it takes."""
    dev = torch.cuda.current_device() if torch.cuda.is_initialized() else None
    for name, t in tensors.items():
        if t is not None and t.is_cuda and t.device.index != dev:
            raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")


def _pages(d: OasisDims, t: torch.Tensor, name: str) -> int:
    """Number of pages [Hkv][B][d] of a tier."""
    per = d.num_kv_heads * d.block_size * d.head_dim
    if t.dim() < 1 or per < 1 or t.numel() % per:
        raise ValueError(f"{name}: not whole pages of [Hkv][B][d]")
    return t.numel() // per


def _bytes(t: torch.Tensor | None) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def oasis_tree_attn_workspace_bytes(d: OasisDims, num_q_tokens: int) -> int:
    return int(lib().oasis_tree_attn_workspace_bytes(ctypes.byref(d), int(num_q_tokens)))


def _tree_needs(d: OasisDims, T: int, q, ctx_len, tree_k, tree_v, parent, tree_len, out, lse) -> None:
    R, Hq, H, D = d.num_reqs, d.num_q_heads, d.num_kv_heads, d.head_dim
    for t, n, name in ((q, R * T * Hq * D, "q"), (out, R * T * Hq * D, "out"), (lse, R * T * Hq, "lse"),
                       (tree_k, R * T * H * D, "tree_k"), (tree_v, R * T * H * D, "tree_v"), (ctx_len, R, "ctx_len"),
                       (parent, R * T, "parent"), (tree_len, R, "tree_len")):
        _need(t, n, name)


def oasis_tree_attn(d: OasisDims, q, num_q_tokens: int, k_pages, v_pages, block_table, ctx_len, tree_k, tree_v,
                    parent, tree_len, scale: float | None, out, lse, workspace, stream=None) -> None:
    """Attention of a drafted token tree over the paged cache (parent None: a chain; tree_len None: every row)."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.tree_attn(ctypes.addressof(d), q, num_q_tokens, k_pages, v_pages, block_table, ctx_len, tree_k, tree_v,
                             parent, tree_len, scale, out, lse, workspace, _handle(stream))
        if st is not None:
            return _check("oasis_tree_attn", st)
    if scale is None:
        scale = 1.0 / math.sqrt(d.head_dim)
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages differ in shape")
    _tree_needs(d, int(num_q_tokens), q, ctx_len, tree_k, tree_v, parent, tree_len, out, lse)
    _need(block_table, d.num_reqs * d.max_blocks, "block_table")
    _one_device(q=q, k_pages=k_pages, v_pages=v_pages, block_table=block_table, ctx_len=ctx_len, tree_k=tree_k,
                tree_v=tree_v, parent=parent, tree_len=tree_len, out=out, lse=lse, workspace=workspace)
    _check("oasis_tree_attn", lib().oasis_tree_attn(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), _host_or_dev(k_pages, "k_pages", _BF16),
        _host_or_dev(v_pages, "v_pages", _BF16), _pages(d, k_pages, "k_pages"),
        _dev(block_table, "block_table", _I32T), _dev(ctx_len, "ctx_len", _I32T), _dev(tree_k, "tree_k", _BF16),
        _dev(tree_v, "tree_v", _BF16), _dev(parent, "parent", _I32T, nullable=True),
        _dev(tree_len, "tree_len", _I32T, nullable=True), float(scale), _dev(out, "out", _BF16),
        _dev(lse, "lse", _F32, nullable=True),
        _dev(workspace, "workspace", (torch.uint8,), nullable=True), _bytes(workspace), _stream(stream)))


def oasis_sparse_tree_attn_workspace_bytes(d: OasisDims, num_q_tokens: int, k_slots: int) -> int:
    return int(lib().oasis_sparse_tree_attn_workspace_bytes(ctypes.byref(d), int(num_q_tokens), int(k_slots)))


def oasis_sparse_tree_attn(d: OasisDims, q, num_q_tokens: int, pool_k, pool_v, slot_map, k_slots: int, ctx_len, tree_k,
                           tree_v, parent, tree_len, scale: float | None, out, lse, workspace, stream=None) -> None:
    """Attention of a drafted token tree over the working set (parent None: a chain; tree_len None: every row)."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.sparse_tree_attn(ctypes.addressof(d), q, num_q_tokens, pool_k, pool_v, slot_map, k_slots, ctx_len,
                                    tree_k, tree_v, parent, tree_len, scale, out, lse, workspace, _handle(stream))
        if st is not None:
            return _check("oasis_sparse_tree_attn", st)
    if scale is None:
        scale = 1.0 / math.sqrt(d.head_dim)
    R, H, B, D = d.num_reqs, d.num_kv_heads, d.block_size, d.head_dim
    _tree_needs(d, int(num_q_tokens), q, ctx_len, tree_k, tree_v, parent, tree_len, out, lse)
    _need(pool_k, R * (k_slots + 1) * H * B * D, "pool_k")
    _need(pool_v, R * (k_slots + 1) * H * B * D, "pool_v")
    _need(slot_map, R * H * k_slots, "slot_map")
    _one_device(q=q, pool_k=pool_k, pool_v=pool_v, slot_map=slot_map, ctx_len=ctx_len, tree_k=tree_k, tree_v=tree_v,
                parent=parent, tree_len=tree_len, out=out, lse=lse, workspace=workspace)
    _check("oasis_sparse_tree_attn", lib().oasis_sparse_tree_attn(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), _dev(pool_k, "pool_k", _BF16),
        _dev(pool_v, "pool_v", _BF16), _dev(slot_map, "slot_map", _I32T, nullable=k_slots == 0), int(k_slots),
        _dev(ctx_len, "ctx_len", _I32T), _dev(tree_k, "tree_k", _BF16), _dev(tree_v, "tree_v", _BF16),
        _dev(parent, "parent", _I32T, nullable=True), _dev(tree_len, "tree_len", _I32T, nullable=True), float(scale),
        _dev(out, "out", _BF16), _dev(lse, "lse", _F32, nullable=True),
        _dev(workspace, "workspace", (torch.uint8,), nullable=True), _bytes(workspace), _stream(stream)))


def oasis_verify_workspace_bytes(num_reqs: int, num_q_tokens: int, vocab: int) -> int:
    return int(lib().oasis_verify_workspace_bytes(int(num_reqs), int(num_q_tokens), int(vocab)))


def _prob_rows(t: torch.Tensor, name: str, shape):
    """Address and row stride of probabilities [R][T][V]: rows dense, evenly spaced (a padded vocabulary may be
    sliced off)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype is not torch.float32:
        raise TypeError(f"{name}: dtype {t.dtype}, torch.float32 expected")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, {tuple(shape)} expected")
    R, T, V = shape
    row = t.stride(1) if T > 1 else (t.stride(0) if R > 1 else V)
    if (V > 1 and t.stride(2) != 1) or row < V or (R > 1 and t.stride(0) != T * row):
        raise ValueError(f"{name}: rows must be contiguous and evenly spaced")
    return t.data_ptr(), row


def oasis_verify_drafts(target_probs, draft_probs, tokens, parent, tree_len, accept_u, sample_u, path, path_len,
                        out_tokens, workspace, stream=None) -> None:
    """Accepted path, emitted tokens and next token of each request's drafted tree (target_probs and draft_probs
    fp32 [R][T][V]; draft_probs None: certain drafts; parent None: a chain; tree_len None: every row)."""
    if _fast is not None:
        st = _fast.verify_drafts(target_probs, draft_probs, tokens, parent, tree_len, accept_u, sample_u, path, path_len,
                                 out_tokens, workspace, _handle(stream))
        if st is not None:
            return _check("oasis_verify_drafts", st)
    if target_probs.dim() != 3:
        raise ValueError(f"target_probs: {target_probs.dim()} dimensions, [R][T][V] expected")
    R, T, V = target_probs.shape
    for t, n, name in ((tokens, R * T, "tokens"), (parent, R * T, "parent"), (tree_len, R, "tree_len"),
                       (accept_u, R * T, "accept_u"), (sample_u, R, "sample_u"), (path, R * T, "path"),
                       (path_len, R, "path_len"), (out_tokens, R * T, "out_tokens")):
        _need(t, n, name)
    _one_device(target_probs=target_probs, draft_probs=draft_probs, tokens=tokens, parent=parent, tree_len=tree_len,
                accept_u=accept_u, sample_u=sample_u, path=path, path_len=path_len, out_tokens=out_tokens,
                workspace=workspace)
    tp, ts = _prob_rows(target_probs, "target_probs", (R, T, V))
    dp, ds = (None, 0) if draft_probs is None else _prob_rows(draft_probs, "draft_probs", (R, T, V))
    _check("oasis_verify_drafts", lib().oasis_verify_drafts(
        R, T, V, tp, ts, dp, ds, _dev(tokens, "tokens", _I32T), _dev(parent, "parent", _I32T, nullable=True),
        _dev(tree_len, "tree_len", _I32T, nullable=True), _dev(accept_u, "accept_u", _F32),
        _dev(sample_u, "sample_u", _F32), _dev(path, "path", _I32T), _dev(path_len, "path_len", _I32T),
        _dev(out_tokens, "out_tokens", _I32T), _dev(workspace, "workspace", (torch.uint8,), nullable=True),
        _bytes(workspace), _stream(stream)))


def oasis_append_tokens(d: OasisDims, new_k, new_v, num_tokens: int, path, path_len, k_pages, v_pages, block_table,
                        ctx_len, new_ctx_len, stream=None) -> None:
    """Rows path[r][:path_len[r]] of new_k / new_v into the paged cache at ctx_len[r] (path None: rows 0, 1, ...;
    path_len None then: all of them)."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.append_tokens(ctypes.addressof(d), new_k, new_v, num_tokens, path, path_len, k_pages, v_pages,
                                 block_table, ctx_len, new_ctx_len, _handle(stream))
        if st is not None:
            return _check("oasis_append_tokens", st)
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages differ in shape")
    R, H, D, N = d.num_reqs, d.num_kv_heads, d.head_dim, int(num_tokens)
    for t, n, name in ((new_k, R * N * H * D, "new_k"), (new_v, R * N * H * D, "new_v"), (path, R * N, "path"),
                       (path_len, R, "path_len"), (block_table, R * d.max_blocks, "block_table"),
                       (ctx_len, R, "ctx_len"), (new_ctx_len, R, "new_ctx_len")):
        _need(t, n, name)
    _one_device(new_k=new_k, new_v=new_v, path=path, path_len=path_len, k_pages=k_pages, v_pages=v_pages,
                block_table=block_table, ctx_len=ctx_len, new_ctx_len=new_ctx_len)
    _check("oasis_append_tokens", lib().oasis_append_tokens(
        ctypes.byref(d), _dev(new_k, "new_k", _BF16), _dev(new_v, "new_v", _BF16), N,
        _dev(path, "path", _I32T, nullable=True), _dev(path_len, "path_len", _I32T, nullable=True),
        _host_or_dev(k_pages, "k_pages", _BF16), _host_or_dev(v_pages, "v_pages", _BF16), _pages(d, k_pages, "k_pages"),
        _dev(block_table, "block_table", _I32T), _dev(ctx_len, "ctx_len", _I32T),
        _dev(new_ctx_len, "new_ctx_len", _I32T, nullable=True), _stream(stream)))


# --- the cache in four bits --------------------------------------------------------

ROTARY_PLAIN = 0      # OASIS_ROTARY_PLAIN
ROTARY_LINEAR = 1     # OASIS_ROTARY_LINEAR
ROTARY_STRETCHED = 2  # OASIS_ROTARY_STRETCHED
ROTARY_BY_TURNS = 3   # OASIS_ROTARY_BY_TURNS
ROTARY_BY_INDEX = 4   # OASIS_ROTARY_BY_INDEX


def oasis_rotary_turns(rotary_dim: int, base: float = 10000.0, scaling: int = ROTARY_PLAIN, factor: float = 1.0,
                       first_len: float = 0.0, low: float = 1.0, high: float = 32.0) -> tuple[list[float], float]:
    """Turns of each pair a position, and the amplitude, of rotary positions scaled for long contexts. ``low`` and ``high``
    are by default those usual for ROTARY_BY_INDEX; ROTARY_BY_TURNS usually takes 1 and 4."""
    n = int(rotary_dim)
    turns, amplitude = (ctypes.c_double * max(1, n // 2))(), ctypes.c_double()
    _check("oasis_rotary_turns", lib().oasis_rotary_turns(n, base, int(scaling), factor, first_len, low, high, turns,
                                                          ctypes.byref(amplitude)))
    return list(turns), amplitude.value


class Rotary:
    """Rotary positions: the table of turns on the device, and how pairs lie in a head. Kept by the caller, for as long
    as calls that it was given to are under way."""

    def __init__(self, rotary_dim: int = 128, base: float = 10000.0, interleaved: bool = False,
                 scaling: int = ROTARY_PLAIN, factor: float = 1.0, first_len: float = 0.0, low: float = 1.0,
                 high: float = 32.0, device: str | torch.device = "cuda"):
        turns, amplitude = oasis_rotary_turns(rotary_dim, base, scaling, factor, first_len, low, high)
        self._set(torch.tensor(turns, dtype=torch.float64, device=device), interleaved, amplitude)

    @classmethod
    def from_turns(cls, turns: torch.Tensor, interleaved: bool = False, amplitude: float = 1.0) -> "Rotary":
        """From a float64 device tensor of turns a position, one for each pair."""
        self = cls.__new__(cls)
        self._set(turns, interleaved, amplitude)
        return self

    def _set(self, turns, interleaved, amplitude):
        self.turns = turns
        self.struct = OasisRotary(_dev(turns, "turns", (torch.float64,)) if turns.is_cuda else None, 2 * turns.numel(),
                                  1 if interleaved else 0, float(amplitude))


def _rows(t: torch.Tensor, name: str, shape):
    """Address and row stride of heads [R][T][H][d]: contiguous, or 4-dimensional with dense heads and rows evenly
    spaced (a slice of a joint projection's output)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in _BF16:
        raise TypeError(f"{name}: dtype {t.dtype} not in {_BF16}")
    R, T, H, D = shape
    if t.is_contiguous():
        _need(t, R * T * H * D, name)
        return t.data_ptr(), H * D
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, {tuple(shape)} expected")
    row = t.stride(1) if T > 1 else (t.stride(0) if R > 1 else H * D)
    if (D > 1 and t.stride(3) != 1) or (H > 1 and t.stride(2) != D) or (R > 1 and t.stride(0) != T * row):
        raise ValueError(f"{name}: heads must be contiguous and rows evenly spaced")
    return t.data_ptr(), row


def oasis_q4_page_bytes(d: OasisDims) -> int:
    """Bytes of a 4-bit page: pages are uint8 tensors of whole ones, [num_pages][page bytes]."""
    return int(lib().oasis_q4_page_bytes(ctypes.byref(d)))


def _q4_pages(d: OasisDims, t: torch.Tensor, name: str) -> int:
    per = d.num_kv_heads * d.block_size * 68
    if t.dim() < 1 or per < 1 or t.numel() % per:
        raise ValueError(f"{name}: not whole pages of {per} bytes")
    return t.numel() // per


_U8 = (torch.uint8,)


def oasis_rotate(d: OasisDims, rotary: Rotary, num_tokens: int, positions, ctx_len, q, q_out, k, k_out,
                 inverse: bool = False, stream=None) -> None:
    """Rotary positions of query rows [R][T][Hq][d] and key rows [R][T][Hkv][d] (either may be None) at positions [R][T]
    (None: ctx_len[r] + t); an output may be its own input. inverse: backwards, which takes a gradient of the turned
    rows to that of the rows."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.rotate(ctypes.addressof(d), ctypes.addressof(rotary.struct), rotary.turns, num_tokens, positions, ctx_len,
                          q, q_out, k, k_out, inverse, _handle(stream))
        if st is not None:
            return _check("oasis_rotate", st)
    R, T, D = d.num_reqs, int(num_tokens), d.head_dim
    _need(positions, R * T, "positions")
    _need(ctx_len, R, "ctx_len")
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("q and q_out, and k and k_out, go together")
    args = []
    for t, n, h in ((q, "q", d.num_q_heads), (q_out, "q_out", d.num_q_heads), (k, "k", d.num_kv_heads),
                    (k_out, "k_out", d.num_kv_heads)):
        args += (None, 0) if t is None else _rows(t, n, (R, T, h, D))
    _one_device(turns=rotary.turns, positions=positions, ctx_len=ctx_len, q=q, q_out=q_out, k=k, k_out=k_out)
    _check("oasis_rotate", lib().oasis_rotate(
        ctypes.byref(d), ctypes.byref(rotary.struct), T, _dev(positions, "positions", _I32T, nullable=True),
        _dev(ctx_len, "ctx_len", _I32T, nullable=True), 1 if inverse else 0, *args, _stream(stream)))


def oasis_append_tokens_q4(d: OasisDims, rotary: Rotary | None, new_k, new_v, num_tokens: int, path, path_len, k_pages,
                           v_pages, block_table, ctx_len, new_ctx_len, read_k=None, read_v=None, stream=None) -> None:
    """oasis_append_tokens into 4-bit pages (uint8), the keys turned to their positions first (rotary None: as they
    are); read_k and read_v receive the rows as the cache holds them."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.append_tokens_q4(ctypes.addressof(d), 0 if rotary is None else ctypes.addressof(rotary.struct),
                                    None if rotary is None else rotary.turns, new_k, new_v, num_tokens, path, path_len,
                                    k_pages, v_pages, block_table, ctx_len, new_ctx_len, read_k, read_v, _handle(stream))
        if st is not None:
            return _check("oasis_append_tokens_q4", st)
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages differ in shape")
    R, H, D, N = d.num_reqs, d.num_kv_heads, d.head_dim, int(num_tokens)
    for t, n, name in ((path, R * N, "path"), (path_len, R, "path_len"), (block_table, R * d.max_blocks, "block_table"),
                       (ctx_len, R, "ctx_len"), (new_ctx_len, R, "new_ctx_len"), (read_k, R * N * H * D, "read_k"),
                       (read_v, R * N * H * D, "read_v")):
        _need(t, n, name)
    rows = (*_rows(new_k, "new_k", (R, N, H, D)), *_rows(new_v, "new_v", (R, N, H, D)))
    _one_device(turns=None if rotary is None else rotary.turns, new_k=new_k, new_v=new_v, path=path, path_len=path_len,
                k_pages=k_pages, v_pages=v_pages, block_table=block_table, ctx_len=ctx_len, new_ctx_len=new_ctx_len,
                read_k=read_k, read_v=read_v)
    _check("oasis_append_tokens_q4", lib().oasis_append_tokens_q4(
        ctypes.byref(d), None if rotary is None else ctypes.byref(rotary.struct), *rows, N,
        _dev(path, "path", _I32T, nullable=True), _dev(path_len, "path_len", _I32T, nullable=True),
        _host_or_dev(k_pages, "k_pages", _U8), _host_or_dev(v_pages, "v_pages", _U8), _q4_pages(d, k_pages, "k_pages"),
        _dev(block_table, "block_table", _I32T), _dev(ctx_len, "ctx_len", _I32T),
        _dev(new_ctx_len, "new_ctx_len", _I32T, nullable=True), _dev(read_k, "read_k", _BF16, nullable=True),
        _dev(read_v, "read_v", _BF16, nullable=True), _stream(stream)))


def oasis_update_summaries_q4(d: OasisDims, k_pages, block_table, prev_ctx_len, ctx_len, max_new_blocks: int, kmax, kmin,
                              stream=None) -> None:
    """Compressed keys of 4-bit pages: of the blocks completed since prev_ctx_len, or (None) of every block."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.update_summaries_q4(ctypes.addressof(d), k_pages, block_table, prev_ctx_len, ctx_len, max_new_blocks,
                                       kmax, kmin, _handle(stream))
        if st is not None:
            return _check("oasis_update_summaries_q4", st)
    R, H, NB, D = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim
    for t, n, name in ((block_table, R * NB, "block_table"), (prev_ctx_len, R, "prev_ctx_len"), (ctx_len, R, "ctx_len"),
                       (kmax, R * H * NB * D, "kmax"), (kmin, R * H * NB * D, "kmin")):
        _need(t, n, name)
    _one_device(k_pages=k_pages, block_table=block_table, prev_ctx_len=prev_ctx_len, ctx_len=ctx_len, kmax=kmax, kmin=kmin)
    _check("oasis_update_summaries_q4", lib().oasis_update_summaries_q4(
        ctypes.byref(d), _host_or_dev(k_pages, "k_pages", _U8), _q4_pages(d, k_pages, "k_pages"),
        _dev(block_table, "block_table", _I32T), _dev(prev_ctx_len, "prev_ctx_len", _I32T, nullable=True),
        _dev(ctx_len, "ctx_len", _I32T), int(max_new_blocks), _dev(kmax, "kmax", _BF16), _dev(kmin, "kmin", _BF16),
        _stream(stream)))


def oasis_tree_attn_q4_workspace_bytes(d: OasisDims, num_q_tokens: int, k: int) -> int:
    return int(lib().oasis_tree_attn_q4_workspace_bytes(ctypes.byref(d), int(num_q_tokens), int(k)))


def oasis_tree_attn_q4(d: OasisDims, q, num_q_tokens: int, k_pages, v_pages, block_table, ctx_len, sel, sel_count, k: int,
                       tree_k, tree_v, parent, tree_len, scale: float | None, out, lse, workspace, stream=None) -> None:
    """Attention over the 4-bit cache: of the blocks selected for each KV head (sel, sel_count, k: the selection's
    output) and the local one, or (None, None, 0) of every block, and of a drafted tree's rows (tree_k and tree_v None:
    the cache alone; parent None: a chain; tree_len None: every row)."""
    if _fast is not None and type(d) is OasisDims:
        st = _fast.tree_attn_q4(ctypes.addressof(d), q, num_q_tokens, k_pages, v_pages, block_table, sel, sel_count, k, ctx_len,
                                tree_k, tree_v, parent, tree_len, scale, out, lse, workspace, _handle(stream))
        if st is not None:
            return _check("oasis_tree_attn_q4", st)
    if scale is None:
        scale = 1.0 / math.sqrt(d.head_dim)
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages differ in shape")
    RH = d.num_reqs * d.num_kv_heads
    _tree_needs(d, int(num_q_tokens), q, ctx_len, tree_k, tree_v, parent, tree_len, out, lse)
    _need(block_table, d.num_reqs * d.max_blocks, "block_table")
    _need(sel, RH * int(k), "sel")
    _need(sel_count, RH, "sel_count")
    _one_device(q=q, k_pages=k_pages, v_pages=v_pages, block_table=block_table, ctx_len=ctx_len, sel=sel,
                sel_count=sel_count, tree_k=tree_k, tree_v=tree_v, parent=parent, tree_len=tree_len, out=out, lse=lse,
                workspace=workspace)
    _check("oasis_tree_attn_q4", lib().oasis_tree_attn_q4(
        ctypes.byref(d), _dev(q, "q", _BF16), int(num_q_tokens), _host_or_dev(k_pages, "k_pages", _U8),
        _host_or_dev(v_pages, "v_pages", _U8), _q4_pages(d, k_pages, "k_pages"), _dev(block_table, "block_table", _I32T),
        _dev(ctx_len, "ctx_len", _I32T), _dev(sel, "sel", _I32T, nullable=True),
        _dev(sel_count, "sel_count", _I32T, nullable=True), int(k), _dev(tree_k, "tree_k", _BF16, nullable=True),
        _dev(tree_v, "tree_v", _BF16, nullable=True), _dev(parent, "parent", _I32T, nullable=True),
        _dev(tree_len, "tree_len", _I32T, nullable=True), float(scale), _dev(out, "out", _BF16),
        _dev(lse, "lse", _F32, nullable=True), _dev(workspace, "workspace", _U8, nullable=True), _bytes(workspace),
        _stream(stream)))


# --- native step issuer --------------------------------------------------------

_PIPE_SIZES: dict[int, tuple[int, int, int]] = {}  # handle -> element counts of q, ctx_len, moved

def oasis_pipeline_create(d: OasisDims, num_q_tokens: int, first_draft: int, num_draft: int, k: int,
                          fetch_cap: int, scale: float | None, host_k, host_v, host_block_table, max_layers: int,
                          pred_stream=None, xfer_stream=None) -> int:
    """Returns the pipeline handle (an address); release it with oasis_pipeline_destroy."""
    if scale is None:
        scale = 1.0 / math.sqrt(d.head_dim)
    if host_k.shape != host_v.shape:
        raise ValueError("host_k and host_v differ in shape")
    _need(host_k, host_k.shape[0] * d.num_kv_heads * d.block_size * d.head_dim, "host_k")
    _need(host_block_table, d.num_reqs * d.max_blocks, "host_block_table")
    h = ctypes.c_void_p()
    _check("oasis_pipeline_create", lib().oasis_pipeline_create(
        ctypes.byref(d), int(num_q_tokens), int(first_draft), int(num_draft), int(k), int(fetch_cap), float(scale),
        _host_or_dev(host_k, "host_k", _BF16), _host_or_dev(host_v, "host_v", _BF16), int(host_k.shape[0]),
        _dev(host_block_table, "host_block_table", _I32T),
        int(max_layers), None if pred_stream is None else _stream(pred_stream),
        None if xfer_stream is None else _stream(xfer_stream), ctypes.byref(h)))
    _PIPE_SIZES[h.value] = (d.num_reqs * int(num_q_tokens) * d.num_q_heads * d.head_dim, d.num_reqs,
                            d.num_reqs * d.num_kv_heads)
    return h.value


PLAN_ON_TRANSFER = 0    # OASIS_PLAN_ON_TRANSFER
PLAN_ON_PREDICTION = 1  # OASIS_PLAN_ON_PREDICTION


def oasis_pipeline_set_plan_stream(handle: int, where: int) -> None:
    """Plan each step's transfer on the transfer stream (PLAN_ON_TRANSFER) or in the top-K kernel
    on the prediction stream (PLAN_ON_PREDICTION)."""
    _check("oasis_pipeline_set_plan_stream", lib().oasis_pipeline_set_plan_stream(handle, int(where)))


FUSED_PREDICTION_AUTO = 0  # OASIS_FUSED_PREDICTION_AUTO
FUSED_PREDICTION_OFF = 1   # OASIS_FUSED_PREDICTION_OFF
FUSED_PREDICTION_ON = 2    # OASIS_FUSED_PREDICTION_ON


def oasis_pipeline_set_fused_prediction(handle: int, mode: int) -> None:
    """Score and select (and plan) in one kernel per step: AUTO (many short rows), OFF or ON."""
    _check("oasis_pipeline_set_fused_prediction", lib().oasis_pipeline_set_fused_prediction(handle, int(mode)))


def oasis_pipeline_set_local_source(handle: int, d: OasisDims, k_pages, v_pages, block_table) -> None:
    """Pages a growing step refreshes the local block from (all None: the host tier)."""
    if k_pages is None and v_pages is None and block_table is None:
        _check("oasis_pipeline_set_local_source", lib().oasis_pipeline_set_local_source(handle, None, None, 0, None))
        return
    if k_pages is None or v_pages is None or block_table is None:
        raise ValueError("k_pages, v_pages and block_table must all be given or all be None")
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages differ in shape")
    _need(k_pages, k_pages.shape[0] * d.num_kv_heads * d.block_size * d.head_dim, "k_pages")
    _need(block_table, d.num_reqs * d.max_blocks, "block_table")
    _check("oasis_pipeline_set_local_source", lib().oasis_pipeline_set_local_source(
        handle, _host_or_dev(k_pages, "k_pages", _BF16), _host_or_dev(v_pages, "v_pages", _BF16),
        int(k_pages.shape[0]), _dev(block_table, "block_table", _I32T)))


def oasis_pipeline_set_layer(handle: int, layer: int, d: OasisDims, num_q_tokens: int, k: int, kmax, kmin, scores,
                             sel, sel_count, slot_map, slot_stamp, pool_k, pool_v, moved, out, lse,
                             workspace) -> None:
    R, H, NB, D, B = d.num_reqs, d.num_kv_heads, d.max_blocks, d.head_dim, d.block_size
    T, Hq = int(num_q_tokens), d.num_q_heads
    for t, n, name in ((kmax, R * H * NB * D, "kmax"), (kmin, R * H * NB * D, "kmin"), (scores, R * H * NB, "scores"),
                       (sel, R * H * k, "sel"), (sel_count, R * H, "sel_count"), (slot_map, R * H * k, "slot_map"),
                       (slot_stamp, R * H * k, "slot_stamp"), (pool_k, R * (k + 1) * H * B * D, "pool_k"),
                       (pool_v, R * (k + 1) * H * B * D, "pool_v"), (moved, R * H, "moved"),
                       (out, R * T * Hq * D, "out"), (lse, R * T * Hq, "lse")):
        _need(t, n, name)
    b = OasisLayerBuffers(
        _dev(kmax, "kmax", _BF16), _dev(kmin, "kmin", _BF16), _dev(scores, "scores", _F32),
        _dev(sel, "sel", _I32T), _dev(sel_count, "sel_count", _I32T), _dev(slot_map, "slot_map", _I32T),
        _dev(slot_stamp, "slot_stamp", _I32T), _dev(pool_k, "pool_k", _BF16), _dev(pool_v, "pool_v", _BF16),
        _dev(moved, "moved", _I32T, nullable=True), _dev(out, "out", _BF16), _dev(lse, "lse", _F32, nullable=True),
        _dev(workspace, "workspace", (torch.uint8,), nullable=True),
        0 if workspace is None else workspace.numel() * workspace.element_size())
    _check("oasis_pipeline_set_layer", lib().oasis_pipeline_set_layer(handle, int(layer), ctypes.byref(b)))


def oasis_pipeline_step(handle: int, layer: int, q, ctx_len, step: int, growing: bool, moved=None,
                        stream=None, prev_ctx_len=None, max_new_blocks: int = 1) -> None:
    """One layer's pipelined step (q, ctx_len, prev_ctx_len, moved: device tensors of the pipeline's
    shapes); with prev_ctx_len the compressed keys of newly completed blocks are added first."""
    nq, nr, nm = _PIPE_SIZES[handle]
    _need(q, nq, "q")
    _need(ctx_len, nr, "ctx_len")
    _need(prev_ctx_len, nr, "prev_ctx_len")
    _need(moved, nm, "moved")
    _check("oasis_pipeline_step", lib().oasis_pipeline_step(
        handle, int(layer), _dev(q, "q", _BF16), _dev(ctx_len, "ctx_len", _I32T),
        _dev(prev_ctx_len, "prev_ctx_len", _I32T, nullable=True), int(max_new_blocks), int(step),
        1 if growing else 0, _dev(moved, "moved", _I32T, nullable=True), _stream(stream)))


def oasis_pipeline_join(handle: int, stream=None) -> None:
    _check("oasis_pipeline_join", lib().oasis_pipeline_join(handle, _stream(stream)))


def oasis_pipeline_check(handle: int) -> None:
    """Synchronize the device; raise if a transfer of the pipeline gave up waiting for its prediction."""
    _check("oasis_pipeline_check", lib().oasis_pipeline_check(handle))


PREDICT_AUTO = 0              # OASIS_PREDICT_AUTO
PREDICT_BESIDE_ATTENTION = 1  # OASIS_PREDICT_BESIDE_ATTENTION
PREDICT_AFTER_ATTENTION = 2   # OASIS_PREDICT_AFTER_ATTENTION


def oasis_pipeline_set_prediction_order(handle: int, order: int) -> None:
    """Start each step's prediction beside or after its attention (PREDICT_AUTO: by the pair count)."""
    _check("oasis_pipeline_set_prediction_order", lib().oasis_pipeline_set_prediction_order(handle, int(order)))


def oasis_pipeline_set_wait_limit(handle: int, polls: int) -> None:
    """Bound (in polls, about 1 us each) of the staging kernel's wait for its prediction."""
    _check("oasis_pipeline_set_wait_limit", lib().oasis_pipeline_set_wait_limit(handle, int(polls)))


def oasis_pipeline_destroy(handle: int | None) -> None:
    if handle:
        _PIPE_SIZES.pop(handle, None)
        lib().oasis_pipeline_destroy(handle)


PROFILE_KINDS = ("attn", "score", "topk", "stage")


_PROF_CAP: dict[int, int] = {}


def oasis_pipeline_profile_begin(handle: int, max_steps: int) -> None:
    _check("oasis_pipeline_profile_begin", lib().oasis_pipeline_profile_begin(handle, int(max_steps)))
    _PROF_CAP[handle] = int(max_steps)


def oasis_pipeline_profile_end(handle: int, per_step: bool = False):
    """Mean kernel durations (us) over the profiled steps and the number of steps; with
    ``per_step`` also a [steps, 4] array of each step's durations (columns: PROFILE_KINDS)."""
    avg = (ctypes.c_float * 4)()
    n = _I32()
    cap = _PROF_CAP.pop(handle, 0)
    steps = (ctypes.c_float * (4 * max(cap, 1)))() if per_step else None
    _check("oasis_pipeline_profile_end", lib().oasis_pipeline_profile_end(handle, avg, steps, ctypes.byref(n)))
    means = {k: float(avg[i]) for i, k in enumerate(PROFILE_KINDS)}
    if not per_step:
        return means, int(n.value)
    import numpy as np
    return means, int(n.value), np.ctypeslib.as_array(steps)[: 4 * int(n.value)].reshape(-1, 4).copy()
