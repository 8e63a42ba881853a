"""The quantised cache on the device against its 64-bit form: codes, scale bytes and 16-bit copies are the same bits; what is read back
is the code's value rounded once (needs an MI355X)."""
import math

import pytest
import torch

import serving_ref as R
from paper_2601_12698_amd import serving as S

pytestmark = pytest.mark.gpu


def empty(pages, h, page, d, dtype, quantised):
    """A cache of bytes that no write gives: places that are to stay are seen to stay."""
    if quantised:
        return [torch.full((pages, h, page, d), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)] + \
               [torch.full((pages, h, page), 77, dtype=torch.uint8, device="cuda") for _ in range(2)]
    return [torch.full((pages, h, page, d), 3.0, dtype=R.TYPES[dtype], device="cuda") for _ in range(2)] + [None, None]


def tokens(T, h, d, dtype, seed, fused=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, 2 * h, d), generator=g) * torch.exp(3 * torch.randn((T, 2 * h, 1), generator=g))
    x[T // 2, 0] = 0.0                                        # a row of zeros
    x[0, -1, 0] = 448.0 * 2.0 ** -3                           # largest magnitudes on and next to the border of two scales
    x[0, -1, 1:] *= 1e-3
    return x.to(R.TYPES[dtype])


def slots_of(T, pages, page, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(pages * page, generator=g)[:T]


def nan_equal(a, b):
    return torch.equal(torch.nan_to_num(a, nan=1e30), torch.nan_to_num(b, nan=1e30)) and torch.equal(a.isnan(), b.isnan())


def check_written(cache, k, v, slots, dtype, page):
    for x, codes, scales in ((k, cache[0].cpu(), cache[2]), (v, cache[1].cpu(), cache[3])):
        n, s = R.quantise(x, dtype) if scales is not None else (x.double(), None)
        for t, slot in enumerate(slots.tolist()):
            if 0 <= slot < codes.shape[0] * page:
                p, o = divmod(slot, page)
                assert nan_equal(codes[p, :, o].double(), n[t]), (t, slot)
                if s is not None:
                    assert torch.equal(scales[p, :, o].cpu(), s[t]), (t, slot)


@pytest.mark.parametrize("quantised", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,h,d,page", [(1, 1, 16, 1), (1, 8, 128, 16), (33, 3, 96, 4), (70, 2, 256, 16), (129, 5, 80, 32), (40, 1, 48, 256), (17, 4, 112, 8)])
def test_write_and_read(T, h, d, page, dtype, quantised):
    pages = T // page + 3
    x, slots = tokens(T, h, d, dtype, T + d), slots_of(T, pages, page, 5)
    if T > 4:
        slots[2], slots[3] = -1, pages * page                 # left out: padding, and a slot beyond the cache
    cache = empty(pages, h, page, d, dtype, quantised)
    before = [None if c is None else c.clone() for c in cache]
    dev, at = x.cuda(), slots.cuda()
    S.kvcache_write(dev[:, :h], dev[:, h:], at, *cache, dtype)
    check_written(cache, x[:, :h], x[:, h:], slots, dtype, page)
    kept = torch.ones(pages * page, dtype=torch.bool)
    kept[slots[(slots >= 0) & (slots < pages * page)]] = False
    for new, old in zip(cache, before):
        if new is not None:
            a, b = (c.view(torch.uint8).view(pages, h, page, -1).transpose(1, 2).flatten(0, 1).cpu() for c in (new, old))
            assert torch.equal(a[kept], b[kept])
    ko, vo = (torch.full((T, h, d), math.nan, dtype=R.TYPES[dtype], device="cuda") for _ in range(2))
    S.kvcache_read(*cache, at, ko, vo, dtype)
    for out, codes, scales in ((ko, cache[0], cache[2]), (vo, cache[1], cache[3])):
        all_ = R.values(codes.cpu(), None if scales is None else scales.cpu())
        want = torch.zeros(T, h, d, dtype=torch.float64)
        for t, slot in enumerate(slots.tolist()):
            if 0 <= slot < pages * page:
                want[t] = all_[slot // page, :, slot % page]
        assert torch.equal(out.cpu(), want.to(R.TYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_extreme_rows(dtype):
    t = torch.finfo(R.TYPES[dtype])
    rows = [[t.max] * 16, [-t.max, t.tiny] + [1.0] * 14, [t.smallest_normal * t.eps] * 16, [t.smallest_normal] + [0.0] * 15, [-0.0] * 16,
            [math.nan] + [2.0] * 15, [math.inf, -math.inf] + [3.0] * 14, [math.nan] * 16, [math.inf] * 16, [448.0] + [1.0] * 15, [449.0] + [1.0] * 15,
            [1.75 * 2 ** 10] + [2.0 ** -9] * 15, [448.0, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.5 * 2.0 ** -9, 17.0, 19.0, 25.0, 2.0 ** -6, 0.0146] + [0.0] * 7]
    x = torch.tensor(rows, dtype=torch.float64).to(R.TYPES[dtype])[:, None]       # [T, 1, 16]
    T = x.shape[0]
    cache, slots = empty(2, 1, 16, 16, dtype, True), torch.arange(T)
    S.kvcache_write(x.cuda(), x.flip(0).cuda(), slots.cuda(), *cache, dtype)
    check_written(cache, x, x.flip(0), slots, dtype, 16)
    ko, vo = (torch.empty((T, 1, 16), dtype=R.TYPES[dtype], device="cuda") for _ in range(2))
    S.kvcache_read(*cache, slots.cuda(), ko, vo, dtype)
    assert not ko.isinf().any() and torch.equal(ko.cpu().isnan(), ~torch.isfinite(x))
    fine = torch.isfinite(x)
    # half of 2^-3 relative wherever the code is a normal one
    big = fine & (x.double().abs() >= x.double().abs().amax(-1, keepdim=True).nan_to_num(0, 0, 0) * 2.0 ** -13) & (x.double().abs() > 2.0 ** -100)
    error = (ko.cpu().double() - x.double()).abs()
    if dtype == "bf16":
        assert (error[big] <= x.double().abs()[big] / 16).all()


@pytest.mark.parametrize("how", ["odd stride", "offset", "heads apart"])
def test_strides_and_alignment(how):
    T, h, d, page = 21, 3, 64, 8
    x = tokens(T, h, d, "bf16", 4)
    k, v = x[:, :h], x[:, h:]
    if how == "odd stride":
        dev = torch.zeros(T, 2 * h * d + 5, dtype=x.dtype, device="cuda")[:, :2 * h * d].view(T, 2 * h, d)
    elif how == "offset":
        dev = torch.zeros(T * 2 * h * d + 1, dtype=x.dtype, device="cuda")[1:].view(T, 2 * h, d)
    else:
        dev = torch.zeros(2 * h, T, d, dtype=x.dtype, device="cuda").transpose(0, 1)
    dev.copy_(x)
    for quantised in (True, False):
        cache, slots = empty(4, h, page, d, "bf16", quantised), slots_of(T, 4, page, 1)
        S.kvcache_write(dev[:, :h], dev[:, h:], slots.cuda(), *cache, "bf16")
        check_written(cache, k, v, slots, "bf16", page)


def test_slots_beyond_32_bits_and_broadcast_values():
    """A cache of more than 2^32 bytes; v is one row for all tokens (stride 0)."""
    h, d, page = 1, 256, 65536
    pages = 257                                               # 4.3e9 bytes of codes
    cache = [torch.zeros((pages, h, page, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros((pages, h, page), dtype=torch.uint8, device="cuda") for _ in range(2)]
    x = tokens(4, h, d, "bf16", 2)
    k, v = x[:, :h], x[:1, h:].expand(4, h, d)
    slots = torch.tensor([pages * page - 1, 0, 2 ** 24 + 1, 255 * page + 3])
    S.kvcache_write(k.cuda(), x.cuda()[:1, h:].expand(4, h, d), slots.cuda(), *cache, *scales, "bf16")
    ko, vo = (torch.empty((4, h, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    S.kvcache_read(*cache, *scales, slots.cuda(), ko, vo, "bf16")
    for got, want in ((ko, k), (vo, v)):
        n, s = R.quantise(want, "bf16")
        assert torch.equal(got.cpu(), R.values(n, s).to(torch.bfloat16))


def test_on_another_stream_and_in_a_graph():
    T, h, d, page = 24, 4, 128, 16
    x, slots = tokens(T, h, d, "fp16", 3).cuda(), slots_of(T, 4, page, 2).cuda()
    want, cache = empty(4, h, page, d, "fp16", True), empty(4, h, page, d, "fp16", True)
    s = torch.cuda.Stream()
    S.kvcache_write(x[:, :h], x[:, h:], slots, *want, "fp16")
    torch.cuda.synchronize()
    S.kvcache_write(x[:, :h], x[:, h:], slots, *cache, "fp16", stream=s)
    s.synchronize()
    same = lambda a, b: all(torch.equal(p.view(torch.uint8), r.view(torch.uint8)) for p, r in zip(a, b))  # noqa: E731
    assert same(cache, want)
    ko, vo = (torch.empty((T, h, d), dtype=torch.float16, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.kvcache_write(x[:, :h], x[:, h:], slots, *cache, "fp16")
        S.kvcache_read(*cache, slots, ko, vo, "fp16")
    for n in range(4):
        x.mul_(1.25)
        S.kvcache_write(x[:, :h], x[:, h:], slots, *want, "fp16")
        graph.replay()
        torch.cuda.synchronize()
        assert same(cache, want), n
        assert torch.equal(ko.cpu(), R.values(cache[0].cpu(), cache[2].cpu()).transpose(1, 2).flatten(0, 1)[slots.cpu()].to(torch.float16)), n
