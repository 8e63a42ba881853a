"""Rotary positions, cache writes and reads of 4 MB and more, whose results are stored past the caches, and the gradient of rotary
positions in every type, against the 64-bit forms (needs an MI355X).  Bars as in test_gpu_rotary.py and test_gpu_kvcache.py."""
import math

import pytest
import torch

import serving_ref as R
from paper_2601_12698_amd import serving as S
from test_gpu_kvcache import check_written, empty, nan_equal, slots_of, tokens
from test_gpu_rotary import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,hq,hk,d,sections", [
    (3, 5, 2, 64, (8, 24)),                                   # small: stored through the caches
    (2050, 8, 1, 128, (16, 24, 24)), (1031, 13, 4, 128, (10, 30)), (4099, 3, 2, 256, (64, 32)), (9001, 2, 2, 64, (32,)), (701, 40, 8, 96, (16, 16)),
])
def test_rotary_and_its_gradient(T, hq, hk, d, sections, dtype, interleaved, inverse):
    x, pos, freq, axis = make(T, hq, hk, d, sections, dtype, T + d)
    big = torch.zeros(T, hq + 2 * hk, d, dtype=x.dtype, device="cuda")          # a fused projection: the values stand behind
    dev = big[:, :hq + hk].copy_(x)
    out = torch.full((T, hq + hk, d), math.nan, dtype=x.dtype, device="cuda")
    p, f, a = pos.cuda(), freq.cuda(), axis.cuda()
    S.rotary_run(dev[:, :hq], dev[:, hq:], out[:, :hq], out[:, hq:], p, f, a, dtype, interleaved=interleaved, inverse=inverse)
    check(out.cpu(), x, pos, freq, axis, dtype, inverse, interleaved)
    S.rotary_run(dev[:, :hq], dev[:, hq:], dev[:, :hq], dev[:, hq:], p, f, a, dtype, interleaved=interleaved, inverse=inverse)      # in place
    assert torch.equal(dev, out) and (big[:, hq + hk:] == 0).all()


@pytest.mark.parametrize("quantised", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,h,d,page", [(1101, 8, 128, 16), (4201, 1, 256, 64), (3001, 5, 80, 32)])
def test_write_and_read(T, h, d, page, dtype, quantised):
    pages = T // page + 3
    x, slots = tokens(T, h, d, dtype, T + d), slots_of(T, pages, page, 5)
    slots[2], slots[3], slots[T - 1] = -1, pages * page, -7     # left out: padding, and a slot beyond the cache
    cache = empty(pages, h, page, d, dtype, quantised)
    before = [None if c is None else c.clone() for c in cache]
    dev, at = x.cuda(), slots.cuda()
    S.kvcache_write(dev[:, :h], dev[:, h:], at, *cache, dtype)
    check_written(cache, x[:, :h], x[:, h:], slots, dtype, page)
    untouched = torch.ones(pages * page, dtype=torch.bool)
    untouched[slots[(slots >= 0) & (slots < pages * page)]] = False
    for new, old in zip(cache, before):
        if new is not None:
            a, b = (c.view(torch.uint8).view(pages, h, page, -1).transpose(1, 2).flatten(0, 1).cpu() for c in (new, old))
            assert torch.equal(a[untouched], b[untouched])
    ko, vo = (torch.full((T, h, d), math.nan, dtype=R.TYPES[dtype], device="cuda") for _ in range(2))
    S.kvcache_read(*cache, at, ko, vo, dtype)
    inside = (slots >= 0) & (slots < pages * page)
    for out, codes, scales in ((ko, cache[0], cache[2]), (vo, cache[1], cache[3])):
        all_ = R.values(codes.cpu(), None if scales is None else scales.cpu()).transpose(1, 2).flatten(0, 1)
        want = torch.zeros(T, h, d, dtype=torch.float64)
        want[inside] = all_[slots[inside]]
        assert nan_equal(out.cpu(), want.to(R.TYPES[dtype]))       # rows that overflow the type before they are written hold NaN codes
