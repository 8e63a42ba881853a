"""ctypes binding of the operators around a decode step's attention -- argument marshalling only.

``include/rotary.h`` (rotary positions with several axes), ``include/kvcache.h`` (a paged cache, quantised as it is
written, and read back) and ``include/prefixattn.h`` (attention of a batch that shares a long prefix, over that cache).
Every function has the name of the C entry point it calls; the checks, errors and streams are those of
:mod:`paper_2601_12698_amd.binding`.  Sizes and strides come from the tensors' shapes: their last axis is contiguous,
the others may have any stride where the header says so.

A decode step in order (``examples/shared_prefix_decode.py`` runs it)::

    addrms_run(...)                       # add + norm, then the projection to q, k, v
    rotary_run(q, k, q, k, ...)           # in place
    kvcache_write(k, v, slots, ...)       # the new tokens into the pages
    prefixattn_run(q, ..., out, lse, ...) # prefix once for all, suffixes each
"""
from __future__ import annotations

import ctypes
from ctypes import POINTER, Structure, byref, c_float, c_int, c_int32, c_int64, c_void_p
from typing import Sequence

from . import binding as B
from .binding import AddrmsError, AddrmsLibraryMissing  # noqa: F401  (what the calls raise)

ROTARY_INTERLEAVED, ROTARY_INVERSE = 1, 2
KVCACHE_SAME, KVCACHE_E4M3 = 0, 1
MAX_HEAD = 256


class PrefixAttnShape(Structure):
    _fields_ = [("batch", c_int32), ("q_len", c_int32), ("q_heads", c_int32), ("kv_heads", c_int32), ("d", c_int32), ("page_size", c_int32),
                ("pages", c_int64), ("prefix_len", c_int64), ("suffix_width", c_int64), ("dtype", c_int32), ("format", c_int32)]


_S = POINTER(c_int64)
SIGNATURES = {
    "rotary_run": (c_int, [c_void_p, _S, c_void_p, _S, c_void_p, _S, c_void_p, _S, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32,
                           c_int32, c_int32, c_int32, c_int, c_int, c_void_p]),
    "rotary_algorithmic_bytes": (c_int64, [c_int64, c_int32, c_int32, c_int32, c_int]),
    "kvcache_write": (c_int, [c_void_p, _S, c_void_p, _S, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32, c_int64,
                              c_int32, c_int, c_int, c_void_p]),
    "kvcache_read": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32, c_int64, c_int32,
                             c_int, c_int, c_void_p]),
    "kvcache_algorithmic_bytes": (c_int64, [c_int64, c_int32, c_int32, c_int, c_int]),
    "prefixattn_workspace_bytes": (c_int64, [POINTER(PrefixAttnShape)]),
    "prefixattn_run": (c_int, [c_void_p, _S, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_float,
                               POINTER(PrefixAttnShape), c_void_p, c_int64, c_void_p]),
    "prefixattn_algorithmic_bytes": (c_int64, [POINTER(PrefixAttnShape), c_int64]),
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
            native.bind_serving(B.DTYPE_IDS, *(ctypes.cast(getattr(lib, f), c_void_p).value for f in
                                               ("rotary_run", "kvcache_write", "kvcache_read", "prefixattn_run")))
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


# ---- checks -----------------------------------------------------------------------------------------------------

def _dtype(dtype, known=(B.BF16, B.FP16)) -> int:
    dt = B.DTYPE_IDS.get(dtype, -1) if isinstance(dtype, str) else int(dtype)
    if dt not in known:
        raise ValueError(f"unknown dtype {dtype!r}")
    return dt


def _on_device(name: str, t, device=None) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the others are on {device}")


def _heads(name: str, t, dt: int, shape, device=None):
    """A [tokens, heads, d] tensor's strides, as the C entry points take them."""
    B._expect_elem(name, t, B._X_ELEM[dt])
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    _on_device(name, t, device)
    token, head, last = t.stride()
    if last != 1 and t.shape[2] > 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return (c_int64 * 2)(token, head)


def _whole(name: str, t, elem: str, shape, device=None) -> int:
    B._expect_elem(name, t, elem)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    _on_device(name, t, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _cache(k_pages, v_pages, k_scale, v_scale, dt: int, device):
    """(format, pages, heads, page size, d, pointers) of a cache."""
    if k_pages.dim() != 4:
        raise ValueError(f"k_pages must be [pages, heads, page_size, d], not {tuple(k_pages.shape)}")
    pages, heads, page, d = k_pages.shape
    got = str(k_pages.dtype).replace("torch.", "")
    quantised = got in ("float8_e4m3fn", "uint8")
    elem = got if quantised else B._X_ELEM[dt]
    ptrs = [_whole("k_pages", k_pages, elem, k_pages.shape, device), _whole("v_pages", v_pages, elem, k_pages.shape, device)]
    if quantised:
        if k_scale is None or v_scale is None:
            raise ValueError("a cache of e4m3 codes has scales")
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            kind = str(t.dtype).replace("torch.", "")
            ptrs.append(_whole(name, t, kind if kind in ("uint8", "float8_e8m0fnu") else "uint8", (pages, heads, page), device))
    else:
        if k_scale is not None or v_scale is not None:
            raise ValueError("a cache of 16-bit elements has no scales")
        ptrs += [None, None]
    return (KVCACHE_E4M3 if quantised else KVCACHE_SAME), pages, heads, page, d, ptrs


# ---- rotary positions (include/rotary.h) ------------------------------------------------------------------------

def rotary_algorithmic_bytes(tokens: int, heads: int, d: int, axes: int, dtype) -> int:
    return B._check(load().rotary_algorithmic_bytes(tokens, heads, d, axes, B._dtype_id(dtype)))


def rotary_plan(rotary_dim: int, base: float, sections: Sequence[int], device, cyclic: bool = False):
    """(inv_freq, pair_axis) of ``base ** (-2 i / rotary_dim)``: the first ``sections[0]`` pairs belong to the first axis and
    so on, or with ``cyclic`` pair i to axis i % axes as long as that axis has pairs left.  Made once, kept by the program."""
    import torch
    pairs, axes = rotary_dim // 2, len(sections)
    if rotary_dim <= 0 or rotary_dim % 2 or axes == 0 or min(sections) < 0 or sum(sections) != pairs:
        raise ValueError(f"sections {tuple(sections)} do not add up to the {pairs} pairs of {rotary_dim} elements")
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    if cyclic:
        left, axis, a = list(sections), [], 0
        for _ in range(pairs):
            while left[a] == 0:
                a = (a + 1) % axes
            axis.append(a)
            left[a] -= 1
            a = (a + 1) % axes
    freq = [float(base) ** (-2.0 * i / rotary_dim) for i in range(pairs)]
    return torch.tensor(freq, dtype=torch.float64, device=device), torch.tensor(axis, dtype=torch.uint8, device=device)


def rotary_run(q, k, q_out, k_out, positions, inv_freq, pair_axis, dtype, interleaved: bool = False, inverse: bool = False,
               stream=None) -> None:
    """Turns q [tokens, q_heads, d] and k [tokens, k_heads, d] (None: queries alone) by their positions [axes, tokens] (int64);
    ``inverse`` turns back, which is the gradient.  q_out and k_out may be q and k themselves."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.rotary_run(q, k, q_out, k_out, positions, inv_freq, pair_axis, dtype, interleaved, inverse)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype, (B.BF16, B.FP16, B.FP32))
    if (k is None) != (k_out is None):
        raise ValueError("k and k_out are given together")
    if q.dim() != 3 or (k is not None and k.dim() != 3):
        raise ValueError("q and k must be [tokens, heads, d]")
    tokens, hq, d = q.shape
    hk = 0 if k is None else k.shape[1]
    qs, qos = _heads("q", q, dt, q.shape), _heads("q_out", q_out, dt, q.shape, q.device)
    ks = kos = None
    if k is not None:
        ks, kos = _heads("k", k, dt, (tokens, hk, d), q.device), _heads("k_out", k_out, dt, (tokens, hk, d), q.device)
    if positions.dim() != 2 or inv_freq.dim() != 1:
        raise ValueError("positions must be [axes, tokens] and inv_freq [pairs]")
    axes, pairs = positions.shape[0], inv_freq.shape[0]
    pos = _whole("positions", positions, "int64", (axes, tokens), q.device)
    freq = _whole("inv_freq", inv_freq, "float64", (pairs,), q.device)
    axis = _whole("pair_axis", pair_axis, "uint8", (pairs,), q.device)
    flags = (ROTARY_INTERLEAVED if interleaved else 0) | (ROTARY_INVERSE if inverse else 0)
    B._check(load().rotary_run(q.data_ptr(), qs, None if k is None else k.data_ptr(), ks, q_out.data_ptr(), qos,
                               None if k is None else k_out.data_ptr(), kos, pos, freq, axis, tokens, hq, hk, d, 2 * pairs, axes, dt, flags,
                               B._stream_ptr(stream, q)))


# ---- the cache (include/kvcache.h) ------------------------------------------------------------------------------

def kvcache_algorithmic_bytes(tokens: int, heads: int, d: int, dtype, quantised: bool = True) -> int:
    return B._check(load().kvcache_algorithmic_bytes(tokens, heads, d, _dtype(dtype), KVCACHE_E4M3 if quantised else KVCACHE_SAME))


def kvcache_write(k, v, slots, k_pages, v_pages, k_scale, v_scale, dtype, stream=None) -> None:
    """Tokens k, v [tokens, heads, d] go to their slots (int64 [tokens], each named once) of the pages [pages, heads, page_size, d]: quantised
    where the pages are ``float8_e4m3fn`` (or bytes) with scale bytes [pages, heads, page_size], else copied (scales None)."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.kvcache_write(k, v, slots, k_pages, v_pages, k_scale, v_scale, dtype)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype)
    fmt, pages, heads, page, d, ptrs = _cache(k_pages, v_pages, k_scale, v_scale, dt, k.device)
    if k.dim() != 3:
        raise ValueError("k and v must be [tokens, heads, d]")
    tokens = k.shape[0]
    ks, vs = _heads("k", k, dt, (tokens, heads, d)), _heads("v", v, dt, (tokens, heads, d), k.device)
    B._check(load().kvcache_write(k.data_ptr(), ks, v.data_ptr(), vs, _whole("slots", slots, "int64", (tokens,), k.device), *ptrs, tokens, heads, d,
                                  pages, page, dt, fmt, B._stream_ptr(stream, k)))


def kvcache_read(k_pages, v_pages, k_scale, v_scale, slots, k_out, v_out, dtype, stream=None) -> None:
    """Tokens at the slots, back in 16 bits: k_out, v_out [tokens, heads, d], contiguous; zeros for slots outside the cache."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.kvcache_read(k_pages, v_pages, k_scale, v_scale, slots, k_out, v_out, dtype)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype)
    fmt, pages, heads, page, d, ptrs = _cache(k_pages, v_pages, k_scale, v_scale, dt, slots.device)
    tokens = slots.shape[0]
    B._check(load().kvcache_read(*ptrs, _whole("slots", slots, "int64", (tokens,)),
                                 _whole("k_out", k_out, B._X_ELEM[dt], (tokens, heads, d), slots.device),
                                 _whole("v_out", v_out, B._X_ELEM[dt], (tokens, heads, d), slots.device), tokens, heads, d, pages, page, dt, fmt,
                                 B._stream_ptr(stream, slots)))


# ---- attention over a shared prefix (include/prefixattn.h) ------------------------------------------------------

def prefixattn_shape(batch: int, q_len: int, q_heads: int, kv_heads: int, d: int, page_size: int, pages: int, prefix_len: int,
                     suffix_width: int, dtype, quantised: bool) -> PrefixAttnShape:
    return PrefixAttnShape(batch, q_len, q_heads, kv_heads, d, page_size, pages, prefix_len, suffix_width, _dtype(dtype),
                           KVCACHE_E4M3 if quantised else KVCACHE_SAME)


def prefixattn_workspace_bytes(shape: PrefixAttnShape) -> int:
    return B._check(load().prefixattn_workspace_bytes(byref(shape)))


def prefixattn_algorithmic_bytes(shape: PrefixAttnShape, suffix_keys: int) -> int:
    return B._check(load().prefixattn_algorithmic_bytes(byref(shape), suffix_keys))


def prefixattn_run(q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len: int, suffix_pages, suffix_lens, out, lse, scale: float,
                   dtype, q_len: int = 1, workspace=None, stream=None) -> None:
    """Queries q [batch * q_len, q_heads, d] against the ``prefix_len`` keys in ``prefix_pages`` (int32), which all share, and the
    ``suffix_lens`` (int32 [batch]) keys in ``suffix_pages`` (int32 [batch, width]) of each sequence; out as q, contiguous, lse
    fp32 [batch * q_len, q_heads] or None.  ``workspace``: bytes on the device, as many as prefixattn_workspace_bytes says; without
    one the call takes it from torch's allocator, on the current stream."""
    if stream is None and (B._torch_facts or B._torch()) and (native := _fast()) is not None:
        st = native.prefixattn_run(q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len, suffix_pages, suffix_lens, out, lse, scale,
                                   dtype, q_len, workspace)
        if st is not None:
            if st:
                B._check(st)
            return
    dt = _dtype(dtype)
    if q.dim() != 3 or q_len < 1 or q.shape[0] % q_len:
        raise ValueError(f"q must be [batch * q_len, heads, d], and q_len={q_len} at least 1")
    rows, hq, d = q.shape
    batch = rows // q_len
    fmt, pages, hk, page, _, ptrs = _cache(k_pages, v_pages, k_scale, v_scale, dt, q.device)
    qs = _heads("q", q, dt, (rows, hq, k_pages.shape[3]))
    if prefix_len < 0:
        raise ValueError("prefix_len must be >= 0")
    first = width = 0
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
    shape = PrefixAttnShape(batch, q_len, hq, hk, d, page, pages, prefix_len, width, dt, fmt)
    lib = load()
    if workspace is None:
        import torch
        if stream is not None and B._stream_ptr(stream, q) != B._stream_ptr(None, q):
            raise ValueError("a call on a stream of its own brings its workspace")
        workspace = torch.empty(max(16, prefixattn_workspace_bytes(shape)), dtype=torch.uint8, device=q.device)
    else:
        _on_device("workspace", workspace, q.device)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
    B._check(lib.prefixattn_run(q.data_ptr(), qs, *ptrs, *tables, o, s, float(scale), byref(shape), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), B._stream_ptr(stream, q)))
