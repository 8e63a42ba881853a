"""What the operators around a decode step's attention refuse, and what is decided without a GPU: every entry point checks its
arguments before anything is launched, so wrong ones can be passed here (the pointers are numbers that nothing reads)."""
import ctypes
import os
import re
from ctypes import byref, c_int64

import pytest
import torch

import serving_ref as R
from paper_2601_12698_amd import binding as B
from paper_2601_12698_amd import serving as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                                   # an address that is aligned to everything
ST = (c_int64 * 2)(64 * 8, 64)
E = S.AddrmsError


def test_headers_library_and_binding_name_the_same_entry_points():
    names = set()
    for header in ("rotary.h", "kvcache.h", "prefixattn.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names |= set(re.findall(r"\b((?:rotary|kvcache|prefixattn)_[a-z_0-9]+)\s*\(", text))
    assert names == set(S.SIGNATURES) and len(names) == 8
    lib = ctypes.CDLL(B.LIB_PATH)
    for n in names:
        assert hasattr(lib, n) and callable(getattr(S, n))
    assert ctypes.sizeof(S.PrefixAttnShape) == 6 * 4 + 3 * 8 + 2 * 4


def rotary(q=P, qs=ST, k=P, ks=ST, qo=P, qos=ST, ko=P, kos=ST, pos=P, freq=P, axis=P, tokens=4, hq=8, hk=8, d=64, rot=64, axes=3, dtype=0, flags=0):
    return S.load().rotary_run(q, qs, k, ks, qo, qos, ko, kos, pos, freq, axis, tokens, hq, hk, d, rot, axes, dtype, flags, None)


@pytest.mark.parametrize("what,status", [
    (dict(dtype=2), B.ERR_UNSUPPORTED_DTYPE), (dict(dtype=9), B.ERR_UNSUPPORTED_DTYPE), (dict(flags=4), B.ERR_INVALID_ARG),
    (dict(tokens=-1), B.ERR_INVALID_ARG), (dict(hq=-1), B.ERR_INVALID_ARG), (dict(rot=63), B.ERR_INVALID_ARG), (dict(rot=66), B.ERR_INVALID_ARG),
    (dict(rot=0), B.ERR_INVALID_ARG), (dict(axes=0), B.ERR_INVALID_ARG), (dict(axes=256), B.ERR_INVALID_ARG), (dict(d=0), B.ERR_INVALID_ARG),
    (dict(d=258, rot=64), B.ERR_UNSUPPORTED_SHAPE), (dict(tokens=1 << 31), B.ERR_UNSUPPORTED_SHAPE), (dict(hq=65536), B.ERR_UNSUPPORTED_SHAPE),
    (dict(q=None), B.ERR_INVALID_ARG), (dict(ko=None), B.ERR_INVALID_ARG), (dict(pos=None), B.ERR_INVALID_ARG), (dict(axis=None), B.ERR_INVALID_ARG),
    (dict(qs=None), B.ERR_INVALID_ARG), (dict(q=P + 1), B.ERR_MISALIGNED), (dict(pos=P + 4), B.ERR_MISALIGNED), (dict(freq=P + 4), B.ERR_MISALIGNED),
    (dict(qos=(c_int64 * 2)(64, 64)), B.ERR_INVALID_ARG), (dict(kos=(c_int64 * 2)(512, 32)), B.ERR_INVALID_ARG), (dict(qos=(c_int64 * 2)(0, 64)), B.ERR_INVALID_ARG),
    (dict(tokens=0), B.OK), (dict(hq=0, hk=0), B.OK), (dict(tokens=0, q=None, pos=None), B.OK),
])
def test_rotary_refusals(what, status):
    assert rotary(**what) == status
    if status != B.OK:
        assert B.addrms_last_error()


def cache_write(k=P, ks=ST, v=P, vs=ST, slots=P, kp=P, vp=P, kc=P, vc=P, tokens=4, heads=8, d=64, pages=10, page=16, dtype=0, fmt=1):
    return S.load().kvcache_write(k, ks, v, vs, slots, kp, vp, kc, vc, tokens, heads, d, pages, page, dtype, fmt, None)


def cache_read(k=P, ks=None, v=P, vs=None, slots=P, kp=P, vp=P, kc=P, vc=P, tokens=4, heads=8, d=64, pages=10, page=16, dtype=0, fmt=1):
    return S.load().kvcache_read(kp, vp, kc, vc, slots, k, v, tokens, heads, d, pages, page, dtype, fmt, None)


@pytest.mark.parametrize("call", [cache_write, cache_read])
@pytest.mark.parametrize("what,status", [
    (dict(dtype=3), B.ERR_UNSUPPORTED_DTYPE), (dict(dtype=2), B.ERR_UNSUPPORTED_DTYPE), (dict(fmt=2), B.ERR_INVALID_ARG), (dict(tokens=-1), B.ERR_INVALID_ARG),
    (dict(heads=0), B.ERR_INVALID_ARG), (dict(pages=-1), B.ERR_INVALID_ARG), (dict(page=24), B.ERR_INVALID_ARG), (dict(page=0), B.ERR_INVALID_ARG),
    (dict(page=131072), B.ERR_INVALID_ARG), (dict(d=40), B.ERR_UNSUPPORTED_SHAPE), (dict(d=272), B.ERR_UNSUPPORTED_SHAPE),
    (dict(pages=1 << 31), B.ERR_UNSUPPORTED_SHAPE), (dict(tokens=1 << 29), B.ERR_UNSUPPORTED_SHAPE), (dict(k=None), B.ERR_INVALID_ARG),
    (dict(slots=None), B.ERR_INVALID_ARG), (dict(kp=None), B.ERR_INVALID_ARG), (dict(kc=None), B.ERR_INVALID_ARG), (dict(vc=None), B.ERR_INVALID_ARG),
    (dict(v=P + 1), B.ERR_MISALIGNED), (dict(slots=P + 4), B.ERR_MISALIGNED), (dict(vp=P + 8), B.ERR_MISALIGNED), (dict(tokens=0), B.OK),
])
def test_cache_refusals(call, what, status):
    assert call(**what) == status


def shape(**more):
    s = dict(batch=4, q_len=1, q_heads=8, kv_heads=2, d=128, page_size=16, pages=100, prefix_len=3000, suffix_width=4, dtype="bf16", quantised=True)
    s.update(more)
    return S.prefixattn_shape(**s)


def attend(s=None, q=P, qs=ST, kp=P, vp=P, kc=P, vc=P, pre=P, suf=P, lens=P, out=P, lse=P, scale=0.1, room=P, bytes_=1 << 40):
    return S.load().prefixattn_run(q, qs, kp, vp, kc, vc, pre, suf, lens, out, lse, scale, None if s is None else byref(s), room, bytes_, None)


@pytest.mark.parametrize("what,status", [
    (dict(batch=-1), B.ERR_INVALID_ARG), (dict(q_len=-1), B.ERR_INVALID_ARG), (dict(q_heads=9), B.ERR_INVALID_ARG), (dict(kv_heads=0), B.ERR_INVALID_ARG),
    (dict(page_size=48), B.ERR_INVALID_ARG), (dict(prefix_len=-1), B.ERR_INVALID_ARG), (dict(suffix_width=-1), B.ERR_INVALID_ARG),
    (dict(d=72), B.ERR_UNSUPPORTED_SHAPE), (dict(d=512), B.ERR_UNSUPPORTED_SHAPE), (dict(pages=1 << 31), B.ERR_UNSUPPORTED_SHAPE),
    (dict(prefix_len=1 << 30), B.ERR_UNSUPPORTED_SHAPE), (dict(suffix_width=1 << 26), B.ERR_UNSUPPORTED_SHAPE), (dict(suffix_width=1 << 62), B.ERR_UNSUPPORTED_SHAPE),
    (dict(batch=1 << 22), B.ERR_UNSUPPORTED_SHAPE), (dict(batch=1 << 30, q_len=1 << 30), B.ERR_UNSUPPORTED_SHAPE),
    (dict(q_heads=65544, kv_heads=1), B.ERR_UNSUPPORTED_SHAPE),
])
def test_attention_shapes_refused(what, status):
    s = shape(**what)
    assert S.load().prefixattn_workspace_bytes(byref(s)) == status
    assert attend(s) == status


@pytest.mark.parametrize("what,status", [
    (dict(q=None), B.ERR_INVALID_ARG), (dict(qs=None), B.ERR_INVALID_ARG), (dict(out=None), B.ERR_INVALID_ARG), (dict(kp=None), B.ERR_INVALID_ARG),
    (dict(vc=None), B.ERR_INVALID_ARG), (dict(pre=None), B.ERR_INVALID_ARG), (dict(suf=None), B.ERR_INVALID_ARG), (dict(lens=None), B.ERR_INVALID_ARG),
    (dict(room=None), B.ERR_INVALID_ARG), (dict(bytes_=100), B.ERR_INVALID_ARG), (dict(bytes_=-1), B.ERR_INVALID_ARG), (dict(scale=0.0), B.ERR_INVALID_ARG),
    (dict(scale=-1.0), B.ERR_INVALID_ARG), (dict(scale=float("nan")), B.ERR_INVALID_ARG), (dict(scale=float("inf")), B.ERR_INVALID_ARG),
    (dict(q=P + 1), B.ERR_MISALIGNED), (dict(out=P + 8), B.ERR_MISALIGNED), (dict(room=P + 4), B.ERR_MISALIGNED), (dict(lens=P + 2), B.ERR_MISALIGNED),
    (dict(lse=P + 2), B.ERR_MISALIGNED), (dict(kp=P + 8), B.ERR_MISALIGNED),
])
def test_attention_arguments_refused(what, status):
    assert attend(shape(), **what) == status


def test_attention_without_work_and_unknown_shapes():
    assert attend(None) == B.ERR_INVALID_ARG
    assert attend(shape(batch=0), q=None, out=None) == B.OK and attend(shape(q_len=0), q=None) == B.OK
    s = shape()
    s.dtype = 3
    assert attend(s) == B.ERR_UNSUPPORTED_DTYPE
    s = shape()
    s.format = 7
    assert attend(s) == B.ERR_INVALID_ARG
    assert S.prefixattn_workspace_bytes(shape(prefix_len=0, suffix_width=0)) == 0


def test_workspace_holds_a_part_for_each_split():
    """4 d + 8 bytes for each row and part; the parts of a range never hold less than 128 keys but for the last.  Suffixes that fill
    the chip by themselves join the prefix's parts to their own and have none, and where they also see a short prefix there is no part."""
    for prefix, width in ((0, 4), (1, 0), (256, 0), (257, 4), (100000, 100), (1 << 20, 1 << 10)):
        for batch, q_len, heads in ((1, 1, (1, 1)), (64, 1, (64, 8)), (3, 40, (8, 2))):
            s = shape(batch=batch, q_len=q_len, q_heads=heads[0], kv_heads=heads[1], prefix_len=prefix, suffix_width=width, pages=1 << 20)
            rows, n = batch * q_len * heads[0], S.prefixattn_workspace_bytes(s)
            if n == 0:
                assert prefix <= 1024 and q_len * heads[0] // heads[1] <= 16
                continue
            assert n % (rows * (4 * 128 + 8)) == 0
            parts = n // (rows * (4 * 128 + 8))
            assert (prefix > 0) + (width > 0 and batch * heads[1] < 256) <= parts <= -(-prefix // 128) + -(-width * 16 // 128)


def test_bytes_formulas():
    assert S.rotary_algorithmic_bytes(10, 5, 64, 3, "bf16") == 10 * (2 * 5 * 64 * 2 + 24)
    assert S.kvcache_algorithmic_bytes(10, 2, 64, "fp16") == 40 * 64 * 2 + 40 * 65 + 80
    assert S.kvcache_algorithmic_bytes(10, 2, 64, "fp16", quantised=False) == 40 * 64 * 4 + 80
    assert S.prefixattn_algorithmic_bytes(shape(), 50) == 3050 * 2 * 2 * 129 + 32 * (4 * 128 + 4)
    with pytest.raises(E):
        S.rotary_algorithmic_bytes(10, 5, 64, 3, "fp16_res32")


class Dev:
    """Looks like a device tensor of this shape; a call that went on to the library would ask for its address."""

    def __init__(self, *shape, dtype=torch.bfloat16, stride=None, device="cuda:0"):
        self.shape, self.dtype, self.is_cuda, self.device = torch.Size(shape), dtype, True, device
        self._stride = stride or torch.empty(shape, device="meta").stride()

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(self._stride)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def is_contiguous(self):
        return tuple(self._stride) == torch.empty(self.shape, device="meta").stride()

    def data_ptr(self):
        return P


def rot_args(**more):
    a = dict(q=Dev(4, 8, 64), k=Dev(4, 2, 64), q_out=Dev(4, 8, 64), k_out=Dev(4, 2, 64), positions=Dev(3, 4, dtype=torch.int64),
             inv_freq=Dev(32, dtype=torch.float64), pair_axis=Dev(32, dtype=torch.uint8), dtype="bf16")
    a.update(more)
    return a


@pytest.mark.parametrize("what,words", [
    (dict(dtype="fp16"), "dtype asks for"), (dict(dtype="fp16_res32"), "unknown dtype"), (dict(q=Dev(4, 8, 64, stride=(512, 64, 2))), "contiguous"),
    (dict(q=Dev(4, 512)), "must be"), (dict(k_out=None), "given together"), (dict(q_out=Dev(4, 8, 32)), "has shape"), (dict(k=Dev(3, 2, 64)), "has shape"),
    (dict(positions=Dev(3, 5, dtype=torch.int64)), "has shape"), (dict(positions=Dev(3, 4, dtype=torch.int32)), "dtype asks for"),
    (dict(positions=Dev(4, dtype=torch.int64)), "must be"), (dict(pair_axis=Dev(31, dtype=torch.uint8)), "has shape"),
    (dict(inv_freq=Dev(32, dtype=torch.float32)), "dtype asks for"), (dict(q=torch.zeros(4, 8, 64, dtype=torch.bfloat16)), "device tensor"),
    (dict(k_out=Dev(4, 2, 64, device="cuda:1")), "is on cuda:1"),
])
def test_rotary_binding_refuses(what, words):
    with pytest.raises(ValueError, match=words):
        S.rotary_run(**rot_args(**what))


def cache(quantised=True, **more):
    a = dict(k_pages=Dev(9, 2, 16, 64, dtype=torch.float8_e4m3fn if quantised else torch.bfloat16), v_pages=Dev(9, 2, 16, 64, dtype=torch.float8_e4m3fn if quantised else torch.bfloat16),
             k_scale=Dev(9, 2, 16, dtype=torch.uint8) if quantised else None, v_scale=Dev(9, 2, 16, dtype=torch.uint8) if quantised else None)
    a.update(more)
    return a


@pytest.mark.parametrize("what,words", [
    (dict(k_scale=None), "has scales"), (dict(v_scale=Dev(9, 2, 8, dtype=torch.uint8)), "has shape"), (dict(v_scale=Dev(9, 2, 16, dtype=torch.float32)), "dtype asks for"),
    (dict(v_pages=Dev(9, 2, 16, 64)), "dtype asks for"), (dict(v_pages=Dev(9, 2, 16, 32, dtype=torch.float8_e4m3fn)), "has shape"), (dict(k_pages=Dev(9, 32, 64)), "must be"),
    (dict(k_pages=Dev(9, 2, 16, 64), v_pages=Dev(9, 2, 16, 64)), "has no scales"), (dict(k_pages=Dev(9, 2, 16, 64, dtype=torch.float16)), "dtype asks for"),
])
def test_cache_binding_refuses(what, words):
    c = cache(**what)
    slots = Dev(4, dtype=torch.int64)
    with pytest.raises(ValueError, match=words):
        S.kvcache_write(Dev(4, 2, 64), Dev(4, 2, 64), slots, *c.values(), "bf16")
    with pytest.raises(ValueError, match=words):
        S.kvcache_read(*c.values(), slots, Dev(4, 2, 64), Dev(4, 2, 64), "bf16")
    with pytest.raises(ValueError, match=words):
        S.prefixattn_run(Dev(4, 8, 64), *c.values(), Dev(5, dtype=torch.int32), 70, Dev(4, 1, dtype=torch.int32), Dev(4, dtype=torch.int32), Dev(4, 8, 64), None, 0.1, "bf16")


@pytest.mark.parametrize("what,words", [
    (dict(q=Dev(4, 8, 32)), "has shape"), (dict(q_len=3), "q_len=3"), (dict(q_len=0), "q_len=0"), (dict(prefix_len=81), "do not hold"), (dict(prefix_len=-1), "prefix_len"),
    (dict(suffix_pages=Dev(5, 1, dtype=torch.int32)), "has shape"), (dict(suffix_lens=Dev(4, dtype=torch.int64)), "dtype asks for"),
    (dict(out=Dev(4, 8, 64, stride=(1024, 64, 1))), "contiguous"), (dict(lse=Dev(4, 8, dtype=torch.bfloat16)), "dtype asks for"),
    (dict(workspace=Dev(100, dtype=torch.uint8, stride=(2,))), "contiguous"), (dict(prefix_pages=Dev(5, dtype=torch.int64)), "dtype asks for"),
])
def test_attention_binding_refuses(what, words):
    a = dict(q=Dev(4, 8, 64), **cache(), prefix_pages=Dev(5, dtype=torch.int32), prefix_len=80, suffix_pages=Dev(4, 1, dtype=torch.int32),
             suffix_lens=Dev(4, dtype=torch.int32), out=Dev(4, 8, 64), lse=None, scale=0.1, dtype="bf16", workspace=Dev(1 << 24, dtype=torch.uint8))
    a.update(what)
    with pytest.raises(ValueError, match=words):
        S.prefixattn_run(**a)


def test_rotary_plan():
    freq, axis = S.rotary_plan(16, 100.0, (1, 3, 4), "cpu")
    assert axis.tolist() == [0, 1, 1, 1, 2, 2, 2, 2] and freq.dtype == torch.float64
    assert [float(f) for f in freq] == [100.0 ** (-2.0 * i / 16) for i in range(8)]
    assert S.rotary_plan(16, 100.0, (1, 3, 4), "cpu", cyclic=True)[1].tolist() == [0, 1, 2, 1, 2, 1, 2, 2]
    for bad in ((16, 100.0, (1, 3)), (15, 100.0, (7,)), (16, 100.0, ()), (16, 100.0, (9, -1))):
        with pytest.raises(ValueError):
            S.rotary_plan(*bad, "cpu")


def test_the_64_bit_quantiser_against_torchs_own_rounding():
    """The oracle of the cache: its rounding is that of torch's conversion to e4m3 for every 16-bit value within range, and its scale
    is the least power of two."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[x.abs() <= 448]
    rows = torch.stack((torch.full_like(x, 448.0), x), -1)
    codes, s = R.quantise(rows, "bf16")
    assert (s == 127).all() and torch.equal(codes[:, 1], x.to(torch.float8_e4m3fn).double())
    for a, e in ((448.0, 0), (450.0, 1), (1.0, -8), (0.875, -9), (0.0, 0), (2.0 ** -130, -126), (3e38, 120)):
        assert R.quantise(torch.tensor([[a, -a]], dtype=torch.bfloat16), "bf16")[1].tolist() == [e + 127]
