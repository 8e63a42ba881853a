"""Rotary positions on the device against the 64-bit form (needs an MI355X).

Bar: an output is u c - v s with c, s within 2^-22 absolute (2 units in the last place of fp32), a product rounded to fp32 and a
fused multiply-add: 2^-21 (|u| + |v|) covers them; the rounding into the type adds half a step of the result."""
import math

import pytest
import torch

import serving_ref as R
from paper_2601_12698_amd import serving as S

pytestmark = pytest.mark.gpu


def bound(x, want, dtype, pairs, interleaved):
    x = x.double().abs()
    near = torch.zeros_like(x)
    a, b = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])
    both = torch.stack((a + b, a + b), -1).flatten(-2) if interleaved else torch.cat((a + b, a + b), -1)
    near[..., :2 * pairs] = both
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0           # half a step of fp16 below its normal range
    return 2.0 ** -21 * near + (R.HALF_STEP[dtype] * (want.abs() + 2.0 ** -21 * near)) * (dtype != "fp32") + tiny


def make(T, hq, hk, d, sections, dtype, seed, far=100000, rot=None):
    g = torch.Generator().manual_seed(seed)
    rot = rot or 2 * sum(sections)
    x = torch.randn((T, hq + hk, d), generator=g).to(R.TYPES[dtype])
    pos = torch.randint(0, far, (len(sections), T), generator=g)
    freq, axis = S.rotary_plan(rot, 10000.0, sections, "cpu")
    return x, pos, freq, axis


def check(got, x, pos, freq, axis, dtype, inverse, interleaved):
    want = R.rotary(x, pos, freq, axis, inverse, interleaved)
    assert ((got.double() - want).abs() <= bound(x, want, dtype, freq.numel(), interleaved)).all(), float((got.double() - want).abs().max())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,hq,hk,d,sections", [
    (1, 32, 8, 128, (16, 24, 24)), (1, 1, 1, 64, (32,)), (5, 5, 1, 80, (5, 7, 8)), (37, 3, 3, 96, (11, 21)), (2, 4, 2, 6, (1, 1)),
    (700, 8, 1, 64, (8, 12, 12)), (33, 40, 8, 256, (128,)), (3, 7, 0, 128, (60, 4)), (1030, 2, 1, 16, (3, 1)), (9, 1, 1, 256, (1,)), (4, 2, 1, 250, (124,)),
])
def test_against_the_formula(T, hq, hk, d, sections, dtype, interleaved):
    x, pos, freq, axis = make(T, hq, hk, d, sections, dtype, T + d)
    dev = x.cuda()
    q, k = dev[:, :hq], dev[:, hq:] if hk else None
    qo, ko = torch.full_like(q, math.nan).contiguous(), torch.full_like(k, math.nan).contiguous() if hk else None
    p, f, a = pos.cuda(), freq.cuda(), axis.cuda()
    S.rotary_run(q, k, qo, ko, p, f, a, dtype, interleaved=interleaved)
    check(qo.cpu(), x[:, :hq], pos, freq, axis, dtype, False, interleaved)
    if hk:
        check(ko.cpu(), x[:, hq:], pos, freq, axis, dtype, False, interleaved)
    assert torch.equal(dev.cpu(), x)
    S.rotary_run(q, k, q, k, p, f, a, dtype, interleaved=interleaved)           # in place, the same bits
    assert torch.equal(q, qo) and (not hk or torch.equal(k, ko))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("how", ["token", "head", "offset", "transposed"])
def test_strides_and_alignment(how, dtype):
    T, h, d = 13, 6, 64
    x, pos, freq, axis = make(T, h, 0, d, (10, 22), dtype, 3)
    if how == "token":
        dev = torch.zeros(T, h * d + 3, dtype=x.dtype, device="cuda")[:, :h * d].view(T, h, d)
    elif how == "head":
        dev = torch.zeros(T, h, d + 4, dtype=x.dtype, device="cuda")[:, :, 2:d + 2]
    elif how == "offset":
        dev = torch.zeros(T * h * d + 1, dtype=x.dtype, device="cuda")[1:].view(T, h, d)
    else:
        dev = torch.zeros(h, T, d, dtype=x.dtype, device="cuda").transpose(0, 1)
    dev.copy_(x)
    out = torch.zeros(T, h, d, dtype=x.dtype, device="cuda")
    S.rotary_run(dev, None, out, None, pos.cuda(), freq.cuda(), axis.cuda(), dtype)
    check(out.cpu(), x, pos, freq, axis, dtype, False, False)
    S.rotary_run(dev, None, dev, None, pos.cuda(), freq.cuda(), axis.cuda(), dtype)
    assert torch.equal(dev, out)


def test_far_and_negative_positions_turn_by_the_right_angle():
    x, _, freq, axis = make(6, 2, 0, 128, (32, 32), "fp32", 9)
    pos = torch.tensor([[0, 1, -1, 2 ** 20 + 1, 2 ** 31 + 7, -(2 ** 31)], [3, 2 ** 24 + 1, -77777777, 5, 0, 2 ** 31 - 1]])
    out = torch.empty_like(x, device="cuda")
    S.rotary_run(x.cuda(), None, out, None, pos.cuda(), freq.cuda(), axis.cuda(), "fp32")
    check(out.cpu(), x, pos, freq, axis, "fp32", False, False)
    assert torch.equal(out[0, :, 0].cpu(), x[0, :, 0])                          # position 0 on the first axis: pair 0 does not turn


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_gradient_is_the_inverse(interleaved):
    """<g, turn(x)> = <inverse(g), x>, and the directional difference of turn: turn is linear, so its difference quotient is exact."""
    x, pos, freq, axis = make(11, 4, 2, 96, (8, 20, 4), "fp32", 5)
    g = torch.randn(x.shape, generator=torch.Generator().manual_seed(6))
    p, f, a = pos.cuda(), freq.cuda(), axis.cuda()

    def turn(t, inverse):
        out = torch.empty_like(t, device="cuda")
        S.rotary_run(t[:, :4].cuda(), t[:, 4:].cuda(), out[:, :4], out[:, 4:], p, f, a, "fp32", interleaved=interleaved, inverse=inverse)
        return out.cpu()

    back = turn(g, True)
    check(back, g, pos, freq, axis, "fp32", True, interleaved)
    # 6336 products, each off by at most 2^-21 (|u| + |v|) |g|: far below 2^-18 of the sums of magnitudes
    left, right = (g.double() * turn(x, False).double()).sum(), (back.double() * x.double()).sum()
    assert abs(left - right) <= 2.0 ** -18 * (g.abs().sum() + x.abs().sum())
    step = torch.zeros_like(x)
    step[3, 1, 7] = 0.5
    difference = (R.rotary(x + step, pos, freq, axis, False, interleaved) - R.rotary(x - step, pos, freq, axis, False, interleaved)) / 1.0
    assert abs((difference * g.double()).sum() - back[3, 1, 7].double()) <= 2.0 ** -19 * 8


def test_an_axis_beyond_the_last_counts_as_the_last_and_cyclic_sections():
    x, pos, freq, _ = make(4, 2, 0, 64, (16, 16), "fp32", 7)
    out = torch.empty_like(x, device="cuda")
    axis = torch.full((32,), 9, dtype=torch.uint8)
    S.rotary_run(x.cuda(), None, out, None, pos.cuda(), freq.cuda(), axis.cuda(), "fp32")
    check(out.cpu(), x, pos, freq, torch.ones(32, dtype=torch.uint8), "fp32", False, False)


def test_on_another_stream_and_in_a_graph():
    x, pos, freq, axis = make(64, 8, 2, 128, (16, 24, 24), "bf16", 8)
    dev, p, f, a = x.cuda(), pos.cuda(), freq.cuda(), axis.cuda()
    want, out = torch.empty_like(dev), torch.zeros_like(dev)
    S.rotary_run(dev[:, :8], dev[:, 8:], want[:, :8], want[:, 8:], p, f, a, "bf16")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    S.rotary_run(dev[:, :8], dev[:, 8:], out[:, :8], out[:, 8:], p, f, a, "bf16", stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.rotary_run(dev[:, :8], dev[:, 8:], out[:, :8], out[:, 8:], p, f, a, "bf16")
    for n in range(4):
        p.add_(n)
        S.rotary_run(dev[:, :8], dev[:, 8:], want[:, :8], want[:, 8:], p, f, a, "bf16")
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), n
