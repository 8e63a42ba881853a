"""The largest sizes that the operators around a decode step's attention take: a call beyond them is refused for its shape before anything is
launched, not by the launch.  (On the CPU; what is within them is asked of functions that launch nothing.)"""
from ctypes import byref, c_int64

import pytest

from paper_2601_12698_amd import binding as B
from paper_2601_12698_amd import serving as S
from test_serving_checks import attend, cache_read, cache_write, rotary, shape


@pytest.mark.parametrize("call", [cache_write, cache_read])
@pytest.mark.parametrize("heads,d,lanes", [(8, 256, 32), (1, 144, 32), (3, 128, 16), (7, 96, 16), (8, 64, 8), (16, 16, 2)])
def test_a_cache_call_has_fewer_than_2_to_32_threads(call, heads, d, lanes):
    """A row of d elements takes `lanes` threads; a write rounds the tokens up to eight."""
    most = min((1 << 32) // (heads * lanes), (1 << 31) // heads)
    st = (c_int64 * 2)(heads * d, d)
    for tokens in (most, most + 1, most + 1000, (1 << 31) // heads - 9):
        if tokens >= most:
            assert call(tokens=tokens, heads=heads, d=d, ks=st, vs=st) == B.ERR_UNSUPPORTED_SHAPE, tokens
    fits = most - 300                                          # of whole workgroups of 256 threads
    assert S.load().kvcache_algorithmic_bytes(fits, heads, d, 0, 1) == 2 * fits * heads * (3 * d + 1) + 8 * fits


def test_rotary_calls_beyond_a_launch():
    """Heads of 256 elements that are not aligned, two of them turned: 255 threads a head, two tokens a workgroup."""
    st = (c_int64 * 2)(257, 257)
    one = dict(qs=st, qos=st, hq=1, hk=0, d=256, rot=2, axes=1, dtype=0)
    for tokens in (2 * ((1 << 32) // 255) + 2, (1 << 30) + 1, (1 << 31) - 1):
        assert rotary(tokens=tokens, **one) == B.ERR_UNSUPPORTED_SHAPE, tokens


def test_attention_calls_beyond_a_launch():
    """2^24 sequences of one head: a workgroup of 256 threads each, 2^32 together, one too many.  One sequence fewer is planned."""
    few = dict(q_heads=1, kv_heads=1, d=64, prefix_len=0, suffix_width=1)
    assert S.prefixattn_workspace_bytes(shape(batch=(1 << 24) - 1, **few)) == 0
    s = shape(batch=1 << 24, **few)
    assert S.load().prefixattn_workspace_bytes(byref(s)) == B.ERR_UNSUPPORTED_SHAPE and attend(s) == B.ERR_UNSUPPORTED_SHAPE
    for more in (dict(batch=(1 << 24) + 1), dict(batch=1 << 20, q_len=17)):
        assert attend(shape(**{**few, **more})) == B.ERR_UNSUPPORTED_SHAPE
    # as many rows in workgroups that have 64 and more
    assert S.prefixattn_workspace_bytes(shape(batch=1, q_len=1 << 24, **few)) >= 0
    assert S.prefixattn_workspace_bytes(shape(batch=1 << 17, q_len=128, **few)) >= 0


def test_a_scale_whose_product_with_log2_e_is_no_number_is_refused():
    """Scores are formed as powers of two; beyond this scale every weight would be NaN, also where scores are small."""
    for scale in (2.36e38, 3e38, 3.4e38):
        assert attend(shape(), scale=scale) == B.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 20])
def test_a_huge_scale(q_len):
    """Tiny queries and a scale to match: as their product would be."""
    import torch

    from test_gpu_prefixattn import build, call, check
    c, dtype = build((1, q_len, 4, 1, 64, 30, [q_len], 2, 16, "bf16", False), seed=1)
    c["q"], c["scale"] = (c["q"].double() * 2.0 ** -115).to(torch.bfloat16), 2.0 ** 112
    check(c, dtype, call(c, dtype))


@pytest.mark.gpu
def test_rotary_with_as_many_heads_as_a_call_takes():
    """65536 heads, one a workgroup: as many workgroups along an axis."""
    import torch

    import serving_ref as R
    x = torch.randn(1, 65536, 257, generator=torch.Generator().manual_seed(1)).to(torch.float16)[:, :, :256]
    out = torch.zeros(1, 65536, 257, dtype=torch.float16, device="cuda")[:, :, :256]
    dev = torch.zeros(1, 65536, 257, dtype=torch.float16, device="cuda")[:, :, :256].copy_(x)
    pos, freq, axis = torch.tensor([[5]]), torch.ones(1, dtype=torch.float64), torch.zeros(1, dtype=torch.uint8)
    S.rotary_run(dev[:, :65535], dev[:, 65535:], out[:, :65535], out[:, 65535:], pos.cuda(), freq.cuda(), axis.cuda(), "fp16")
    want = R.rotary(x, pos, freq, axis)
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -20 * (1 + x.double().abs().amax())).all()
