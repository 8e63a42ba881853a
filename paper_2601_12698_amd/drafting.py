"""ctypes binding of the operators of a step that checks drafted tokens -- argument marshalling only.

``include/treeattn.h`` (attention of trees of drafted tokens over a paged cache), ``include/logits.h`` (penalties, biases and masks
on logits, and the best tokens), ``include/treeaccept.h`` (the path of nodes that agree with the model) and ``include/kvmove.h``
(tokens that move in the cache).  Every function has the name of the C entry point it calls; the checks, errors and streams are
those of :mod:`paper_2601_12698_amd.serving`, whose caches these operators share.

A step in order (``examples/tree_decode.py`` runs it), all of whose sizes are the host's and all of whose lengths the device's::

    rotary_run(q, k, q, k, ...)                 # positions go by a node's depth
    kvcache_write(k, v, slots, ...)             # the nodes' keys behind their sequence's
    treeattn_run(q, ..., masks, out, lse, ...)
    logits_run(logits, None, best, ...)         # what the model gives after each node
    treeaccept_run(best, tokens, masks, ...)    # the path that agrees, and the slots of its keys
    kvmove_run(*cache, from_slots, to_slots)    # in every layer: the path's keys side by side
"""
from __future__ import annotations

import ctypes
from ctypes import POINTER, Structure, byref, c_float, c_int, c_int32, c_int64, c_void_p

from . import binding as B
from . import serving as S
from .binding import AddrmsError, AddrmsLibraryMissing  # noqa: F401  (what the calls raise)
from .serving import PrefixAttnShape, _cache, _dtype, _heads, _on_device, _tables, _whole

MAX_NODES, MAX_MOVED, MAX_BIASES, MAX_HISTORY = 64, 256, 1023, 1048575


class LogitsLists(Structure):
    _fields_ = [(n, c_void_p) for n in ("history", "history_lens", "prompt_lens", "penalties", "bias_tokens", "bias_values", "allowed", "tree_tokens",
                                        "tree_masks")] + \
               [("history_stride", c_int64), ("allowed_stride", c_int64), ("history_width", c_int32), ("biases", c_int32)]


SIGNATURES = {
    "treeattn_workspace_bytes": (c_int64, [POINTER(PrefixAttnShape)]),
    "treeattn_run": (c_int, [c_void_p, POINTER(c_int64), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                             c_float, POINTER(PrefixAttnShape), c_void_p, c_int64, c_void_p]),
    "treeattn_algorithmic_bytes": (c_int64, [POINTER(PrefixAttnShape), c_int64]),
    "treeaccept_run": (c_int, [c_void_p] * 10 + [c_int64, c_int32, c_int32, c_int64, c_int64, c_int32, c_void_p]),
    "kvmove_run": (c_int, [c_void_p] * 6 + [c_int64, c_int32, c_int32, c_int32, c_int64, c_int32, c_int, c_int, c_void_p]),
    "kvmove_algorithmic_bytes": (c_int64, [c_int64, c_int32, c_int64, c_int32, c_int32, c_int]),
    "logits_workspace_bytes": (c_int64, [c_int64, c_int32, c_int64, c_int]),
    "logits_run": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_int32, c_int64, c_int, POINTER(LogitsLists), c_void_p, c_int64, c_void_p]),
    "logits_algorithmic_bytes": (c_int64, [c_int64, c_int32, c_int64, c_int, c_int64, c_int32, c_int, c_int]),
}

_lib = None
_bound = None           # the module _native that these entry points were handed to


def _fast():
    """Module _native, which takes the usual calls as one native call (csrc/native_calls.cpp), or None."""
    global _bound
    native = B._native
    if native is not _bound:
        if native is not None:
            lib = load()
            native.bind_drafting(B.DTYPE_IDS, *(ctypes.cast(getattr(lib, f), c_void_p).value for f in
                                                ("treeattn_run", "logits_run", "treeaccept_run", "kvmove_run")))
        _bound = native
    return native


def load() -> ctypes.CDLL:
    """The library, with these entry points declared."""
    global _lib
    if _lib is None:
        lib = B.load()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _workspace(workspace, bytes_: int, stream, tensor):
    """The caller's workspace, or one from torch's allocator, on the current stream."""
    if workspace is None:
        import torch
        if stream is not None and B._stream_ptr(stream, tensor) != B._stream_ptr(None, tensor):
            raise ValueError("a call on a stream of its own brings its workspace")
        return torch.empty(max(16, bytes_), dtype=torch.uint8, device=tensor.device)
    _on_device("workspace", workspace, tensor.device)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace


# ---- attention of trees (include/treeattn.h) --------------------------------------------------------------------

def treeattn_workspace_bytes(shape: PrefixAttnShape) -> int:
    """For a shape of :func:`paper_2601_12698_amd.serving.prefixattn_shape`, whose q_len is the number of nodes."""
    return B._check(load().treeattn_workspace_bytes(byref(shape)))


def treeattn_algorithmic_bytes(shape: PrefixAttnShape, suffix_keys: int) -> int:
    return B._check(load().treeattn_algorithmic_bytes(byref(shape), suffix_keys))


def treeattn_run(q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len: int, suffix_pages, suffix_lens, masks, out, lse, scale: float, dtype,
                 workspace=None, stream=None) -> None:
    """Queries q [batch * nodes, q_heads, d] of trees, masks int64 [batch, nodes], against the ``prefix_len`` keys in ``prefix_pages`` (int32),
    which all share, the ``suffix_lens`` (int32 [batch]) keys in ``suffix_pages`` (int32 [batch, width]) of each sequence, and those of
    the nodes, which lie behind these, that each node's mask names; out as q, contiguous, lse fp32 [batch * nodes, q_heads] or None.
    ``workspace``: bytes on the device, as many as treeattn_workspace_bytes says; without one the call takes it from torch's
    allocator, on the current stream."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.treeattn_run(q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len, suffix_pages, suffix_lens, masks, out, lse, scale, dtype,
                                 workspace)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype)
    if q.dim() != 3 or masks.dim() != 2:
        raise ValueError("q must be [batch * nodes, heads, d] and masks [batch, nodes]")
    _tables(prefix_pages, prefix_len, suffix_pages, suffix_lens)
    rows, hq, _ = q.shape
    batch, nodes = masks.shape
    fmt, pages, hk, page, d, ptrs = _cache(k_pages, v_pages, k_scale, v_scale, dt, q.device)
    qs = _heads("q", q, dt, (batch * nodes, hq, d))
    seen = _whole("masks", masks, "int64", (batch, nodes), q.device)
    width = 0
    tables = [None, None, None]
    if prefix_len:
        first = prefix_pages.numel()
        tables[0] = _whole("prefix_pages", prefix_pages, "int32", (first,), q.device)
        if first * page < prefix_len:
            raise ValueError(f"{first} prefix_pages of {page} keys do not hold {prefix_len}")
    if suffix_pages is not None and suffix_pages.numel():
        width = suffix_pages.shape[-1]
        tables[1] = _whole("suffix_pages", suffix_pages, "int32", (batch, width), q.device)
        tables[2] = _whole("suffix_lens", suffix_lens, "int32", (batch,), q.device)
    o = _whole("out", out, B._X_ELEM[dt], (rows, hq, d), q.device)
    s = None if lse is None else _whole("lse", lse, "float32", (rows, hq), q.device)
    shape = PrefixAttnShape(batch, nodes, hq, hk, d, page, pages, prefix_len, width, dt, fmt)
    room = _workspace(workspace, treeattn_workspace_bytes(shape), stream, q)
    B._check(load().treeattn_run(q.data_ptr(), qs, *ptrs, *tables, seen, o, s, float(scale), byref(shape), room.data_ptr(),
                                 room.numel() * room.element_size(), B._stream_ptr(stream, q)))


# ---- logits (include/logits.h) ----------------------------------------------------------------------------------

def logits_workspace_bytes(batch: int, nodes: int, vocab: int, dtype) -> int:
    return B._check(load().logits_workspace_bytes(batch, nodes, vocab, B._dtype_id(dtype)))


def logits_algorithmic_bytes(batch: int, nodes: int, vocab: int, dtype, tokens: int = 0, biases: int = 0, masked: bool = False, write: bool = True) -> int:
    return B._check(load().logits_algorithmic_bytes(batch, nodes, vocab, B._dtype_id(dtype), tokens, biases, int(masked), int(write)))


def _rows(name: str, t, elem: str, rows: int, width, device=None) -> int:
    """A [rows, width] tensor (width None: any) whose last axis is contiguous; the distance of its rows."""
    B._expect_elem(name, t, elem)
    if t.dim() != 2 or t.shape[0] != rows or (width is not None and t.shape[1] != width):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [{rows}, {'...' if width is None else width}]")
    _on_device(name, t, device)
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return t.stride(0)


def logits_run(logits, out, best, dtype, nodes: int = 1, history=None, history_lens=None, prompt_lens=None, penalties=None, bias_tokens=None,
               bias_values=None, allowed=None, tree_tokens=None, tree_masks=None, workspace=None, stream=None) -> None:
    """logits [batch * nodes, vocab] (rows any distance apart) -> out (as logits, or logits itself; None: not written) and best
    (int32 [batch * nodes], None: not looked for).  history int32 [batch, width], history_lens and prompt_lens int32 [batch]; penalties
    fp32 [batch, 3] (repetition, frequency, presence); bias_tokens int32 and bias_values fp32 [batch, n]; allowed int32 [batch * nodes,
    ceil(vocab / 32) or more], bit t % 32 of word t / 32; tree_tokens int32 and tree_masks int64 [batch, nodes], whose history ends before
    node 0's token.  ``workspace``: bytes on the device, as many as logits_workspace_bytes says; without one the call takes it from torch's
    allocator, on the current stream (with best on a stream of its own it brings one, of no bytes where none are needed)."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.logits_run(logits, out, best, dtype, nodes, history, history_lens, prompt_lens, penalties, bias_tokens, bias_values, allowed,
                               tree_tokens, tree_masks, workspace)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype, (B.BF16, B.FP16, B.FP32))
    elem = B._X_ELEM[dt]
    if logits.dim() != 2 or nodes < 1 or logits.shape[0] % nodes:
        raise ValueError(f"logits must be [batch * nodes, vocab], and nodes={nodes} at least 1")
    rows, vocab = logits.shape
    batch, dev = rows // nodes, logits.device
    stride = _rows("logits", logits, elem, rows, vocab)
    out_stride = 0 if out is None else _rows("out", out, elem, rows, vocab, dev)
    to = None if best is None else _whole("best", best, "int32", (rows,), dev)
    lists = LogitsLists()
    if history is not None:
        if history_lens is None:
            raise ValueError("history has history_lens")
        lists.history_stride = _rows("history", history, "int32", batch, None, dev)
        lists.history, lists.history_width = history.data_ptr(), history.shape[1]
        lists.history_lens = _whole("history_lens", history_lens, "int32", (batch,), dev)
        if prompt_lens is not None:
            lists.prompt_lens = _whole("prompt_lens", prompt_lens, "int32", (batch,), dev)
    if penalties is not None:
        lists.penalties = _whole("penalties", penalties, "float32", (batch, 3), dev)
    if (bias_tokens is None) != (bias_values is None):
        raise ValueError("bias_tokens and bias_values are given together")
    if bias_tokens is not None:
        lists.biases = bias_tokens.shape[-1]
        lists.bias_tokens = _whole("bias_tokens", bias_tokens, "int32", (batch, lists.biases), dev)
        lists.bias_values = _whole("bias_values", bias_values, "float32", (batch, lists.biases), dev)
    if allowed is not None:
        lists.allowed_stride = _rows("allowed", allowed, "int32", rows, None, dev)
        if allowed.shape[1] * 32 < vocab:
            raise ValueError(f"{allowed.shape[1]} words of allowed do not hold {vocab} tokens")
        lists.allowed = allowed.data_ptr()
    if (tree_tokens is None) != (tree_masks is None):
        raise ValueError("tree_tokens and tree_masks are given together")
    if tree_tokens is not None:
        lists.tree_tokens = _whole("tree_tokens", tree_tokens, "int32", (batch, nodes), dev)
        lists.tree_masks = _whole("tree_masks", tree_masks, "int64", (batch, nodes), dev)
    need = 0 if best is None else B._check(load().logits_workspace_bytes(batch, nodes, vocab, dt))
    room = None if best is None else _workspace(workspace, need, stream, logits)
    B._check(load().logits_run(logits.data_ptr(), stride, None if out is None else out.data_ptr(), out_stride, to, batch, nodes, vocab, dt, byref(lists),
                               None if room is None else room.data_ptr(), 0 if room is None else room.numel() * room.element_size(),
                               B._stream_ptr(stream, logits)))


# ---- the path that agrees (include/treeaccept.h) ----------------------------------------------------------------

def treeaccept_run(chosen, tokens, masks, suffix_pages, suffix_lens, page_size: int, pages: int, path, count, next_token, from_slots, to_slots,
                   stream=None) -> None:
    """chosen and tokens int32, masks int64 [batch, nodes] -> path int32 [batch, depth], count and next_token int32 [batch], from_slots and
    to_slots int64 [batch, depth] (None: without; then suffix_pages int32 [batch, width] and suffix_lens int32 [batch] may be None)."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.treeaccept_run(chosen, tokens, masks, suffix_pages, suffix_lens, page_size, pages, path, count, next_token, from_slots, to_slots)
        if st is not None:
            if st:
                B._check(st)
            return
    if masks.dim() != 2 or path.dim() != 2:
        raise ValueError("masks must be [batch, nodes] and path [batch, depth]")
    if (from_slots is None) != (to_slots is None):
        raise ValueError("from_slots and to_slots are given together")
    if from_slots is not None and (suffix_pages is None or suffix_lens is None):
        raise ValueError("from_slots have suffix_pages and suffix_lens")
    (batch, nodes), depth, dev = masks.shape, path.shape[1], masks.device
    ptrs = [_whole("chosen", chosen, "int32", (batch, nodes), dev), _whole("tokens", tokens, "int32", (batch, nodes), dev),
            _whole("masks", masks, "int64", (batch, nodes))]
    width = 0
    if from_slots is None:
        ptrs += [None, None]
    else:
        if suffix_pages.dim() != 2:
            raise ValueError("suffix_pages must be [batch, width]")
        width = suffix_pages.shape[1]
        ptrs += [_whole("suffix_pages", suffix_pages, "int32", (batch, width), dev), _whole("suffix_lens", suffix_lens, "int32", (batch,), dev)]
    ptrs += [_whole("path", path, "int32", (batch, depth), dev), _whole("count", count, "int32", (batch,), dev),
             _whole("next_token", next_token, "int32", (batch,), dev)]
    ptrs += [None, None] if from_slots is None else [_whole("from_slots", from_slots, "int64", (batch, depth), dev),
                                                     _whole("to_slots", to_slots, "int64", (batch, depth), dev)]
    B._check(load().treeaccept_run(*ptrs, batch, nodes, depth, width, pages, page_size, B._stream_ptr(stream, masks)))


# ---- tokens that move (include/kvmove.h) ------------------------------------------------------------------------

def kvmove_algorithmic_bytes(groups: int, tokens: int, moved: int, heads: int, d: int, quantised: bool = True) -> int:
    return B._check(load().kvmove_algorithmic_bytes(groups, tokens, moved, heads, d, S.KVCACHE_E4M3 if quantised else S.KVCACHE_SAME))


def kvmove_run(k_pages, v_pages, k_scale, v_scale, from_slots, to_slots, dtype, stream=None) -> None:
    """Tokens of a cache, as kvcache_write takes it, go from from_slots to to_slots (int64 [groups, tokens], up to MAX_MOVED tokens): those of
    a group as if all were read before one is written.  Where one of a token's slots is not in the cache, it stays."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.kvmove_run(k_pages, v_pages, k_scale, v_scale, from_slots, to_slots, dtype)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype)
    fmt, pages, heads, page, d, ptrs = _cache(k_pages, v_pages, k_scale, v_scale, dt, k_pages.device)
    if from_slots.dim() != 2:
        raise ValueError("from_slots must be [groups, tokens]")
    groups, tokens = from_slots.shape
    B._check(load().kvmove_run(*ptrs, _whole("from_slots", from_slots, "int64", (groups, tokens), k_pages.device),
                               _whole("to_slots", to_slots, "int64", (groups, tokens), k_pages.device), groups, tokens, heads, d, pages, page, dt, fmt,
                               B._stream_ptr(stream, k_pages)))
