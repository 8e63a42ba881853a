"""Attention over a shared prefix on the device against its 64-bit form (needs an MI355X).

Bar.  A weight is 2^(fp32 argument), rounded to 16 bits for the second product: half a step of the type, relative.  Its argument is off by
what an fp32 sum of d products is off by, taken as 2^-21 of the sum of their magnitudes (x), in numerator and denominator, and by 2^-19
for the exponential, the running maximum and the sum of weights.  So an output is off by at most
(half a step + 2 x + 2^-18) * sum of weight |v|, and half a step of itself for its own rounding; fp16 weights below 2^-21 of the largest
lose bits, at most 2^-31 of the largest each.  lse is off by x + 2^-18 + 2^-22 |lse|."""
import math

import pytest
import torch

import serving_ref as R
from paper_2601_12698_amd import serving as S

pytestmark = pytest.mark.gpu


def build(case, seed=0, junk=True):
    """A cache whose unused places hold NaN, and a call's other inputs, on the CPU."""
    batch, q_len, hq, hk, d, prefix, lens, width, page, dtype, quantised = case
    g = torch.Generator().manual_seed(seed)
    first = -(-prefix // page)
    pages = first + batch * width + 2
    k, v = (torch.randn((pages, hk, page, d), generator=g) for _ in range(2))
    k *= 1 + 5 * (torch.arange(d) % 13 == 3)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table, own = order[:first].clone(), order[first:first + batch * width].view(batch, width).clone()
    used = torch.zeros(pages, page, dtype=torch.bool)
    for j in range(prefix):
        used[int(table[j // page]), j % page] = True
    for b in range(batch if width else 0):
        for j in range(min(max(lens[b], 0), width * page)):
            used[int(own[b, j // page]), j % page] = True
    ks = vs = None
    k, v = k.to(R.TYPES[dtype]), v.to(R.TYPES[dtype])
    if quantised:
        (k, ks), (v, vs) = R.quantise(k, dtype), R.quantise(v, dtype)
        k, v = k.to(torch.float8_e4m3fn), v.to(torch.float8_e4m3fn)
    if junk:
        free = ~used[:, None].expand(pages, hk, page)
        for x, s in ((k, ks), (v, vs)):
            if quantised:
                x.view(torch.uint8)[free] = 0x7f
                s[free] = 255
            else:
                x[free] = math.nan
    q = torch.randn((batch * q_len, hq + 3, d), generator=g).to(R.TYPES[dtype])[:, 2:2 + hq]
    return dict(q=q, k_pages=k, v_pages=v, k_scale=ks, v_scale=vs, prefix_pages=table, prefix_len=prefix, suffix_pages=own if width else None,
                suffix_lens=torch.tensor(lens, dtype=torch.int32) if width else None, scale=d ** -0.5, q_len=q_len), dtype


def call(c, dtype, lse=True, **more):
    dev = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in c.items()}
    if c["q"].stride() != dev["q"].stride():
        big = torch.zeros(c["q"].shape[0], c["q"].shape[1] + 3, c["q"].shape[2], dtype=c["q"].dtype, device="cuda")
        dev["q"] = big[:, 2:2 + c["q"].shape[1]].copy_(c["q"])
    out = torch.full(c["q"].shape, math.nan, dtype=c["q"].dtype, device="cuda")
    s = torch.full(c["q"].shape[:2], math.nan, device="cuda") if lse else None
    S.prefixattn_run(dev["q"], dev["k_pages"], dev["v_pages"], dev["k_scale"], dev["v_scale"], dev["prefix_pages"], c["prefix_len"],
                     dev["suffix_pages"], dev["suffix_lens"], out, s, c["scale"], dtype, q_len=c["q_len"], **more)
    torch.cuda.synchronize()
    return out.cpu(), None if s is None else s.cpu()


def check(c, dtype, got):
    want, lse, size = R.attention(**c)
    top = lambda x, s: float(R.values(x, s).nan_to_num(0, 0, 0).abs().max())  # noqa: E731
    x = 2.0 ** -21 * c["scale"] * c["q"].double().abs().sum(-1) * top(c["k_pages"], c["k_scale"])
    keys = c["prefix_len"] + (0 if c["suffix_pages"] is None else c["suffix_pages"].shape[1] * c["k_pages"].shape[2])
    low = keys * 2.0 ** -31 * top(c["v_pages"], c["v_scale"]) if dtype == "fp16" else 0.0
    half = R.HALF_STEP[dtype]
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0
    limit = (half + 2 * x[..., None] + 2.0 ** -18) * size * (1 + half) + half * want.abs() + low + tiny
    off = (got[0].double() - want).abs()
    assert (off <= limit).all(), (float(off.max()), float((off / limit).max()))
    if got[1] is not None:
        seen = torch.isfinite(lse)
        assert torch.equal(torch.isneginf(got[1]), ~seen)
        assert ((got[1].double() - lse).abs()[seen] <= (x + 2.0 ** -18 + 2.0 ** -22 * lse.abs())[seen]).all()


CASES = [
    # batch, q_len, q heads, kv heads, d, prefix, suffix lengths, pages of a suffix, page, type, quantised
    (1, 1, 1, 1, 16, 1, [1], 1, 1, "bf16", False),
    (1, 1, 4, 1, 128, 0, [1], 1, 16, "bf16", True),
    (2, 1, 8, 2, 128, 37, [5, 16], 1, 16, "bf16", True),
    (2, 1, 8, 2, 64, 300, [0, 31], 2, 16, "fp16", True),
    (3, 1, 5, 5, 96, 129, [0, 1, 40], 3, 16, "fp16", False),
    (1, 1, 16, 1, 256, 700, [130], 3, 64, "bf16", False),
    (1, 1, 16, 1, 256, 515, [], 0, 64, "fp16", True),
    (7, 1, 8, 2, 128, 331, [0, 1, 17, 64, 63, 65, -4], 8, 8, "bf16", True),
    (40, 1, 4, 1, 128, 200, [i % 9 for i in range(40)], 2, 8, "bf16", False),
    (9, 4, 4, 1, 64, 100, [0, 1, 2, 3, 4, 5, 33, 20, 7], 3, 16, "bf16", True),
    (3, 7, 8, 2, 80, 65, [3, 7, 100], 7, 16, "fp16", True),
    (2, 40, 8, 2, 128, 130, [40, 75], 5, 16, "bf16", False),
    (1, 150, 2, 1, 256, 64, [260], 5, 64, "bf16", True),
    (2, 3, 8, 8, 112, 0, [2, 300], 19, 16, "bf16", True),
    (5, 2, 6, 3, 48, 1000, [1000, 0, 512, 513, 3], 250, 4, "fp16", False),
    (4, 1, 32, 8, 128, 2049, [1, 300, 0, 257], 10, 32, "bf16", True),
    (33, 1, 16, 4, 256, 260, [3] * 33, 1, 16, "fp16", False),
    # longer prefixes, seen by workgroups of their own: 16, 64, 128 and 256 rows
    (40, 1, 4, 1, 128, 600, [i % 9 for i in range(40)], 2, 8, "bf16", False),
    (9, 4, 4, 1, 64, 700, [0, 1, 2, 3, 4, 5, 33, 20, 7], 3, 16, "bf16", True),
    (20, 1, 8, 2, 256, 900, [i % 11 for i in range(20)], 1, 16, "bf16", True),
    (13, 1, 4, 1, 256, 577, [2] * 13, 1, 32, "fp16", False),
    (70, 1, 4, 1, 128, 1100, [i % 40 for i in range(70)], 3, 16, "fp16", True),
    (70, 1, 4, 1, 96, 1100, [i % 40 for i in range(70)], 3, 16, "bf16", False),
    (24, 1, 5, 1, 112, 777, [i % 5 for i in range(24)], 1, 64, "bf16", False),
    (30, 1, 5, 1, 48, 3000, [i % 5 for i in range(30)], 1, 64, "fp16", True),
    (3, 1, 5, 1, 128, 5000, [100, 0, 1700], 30, 64, "bf16", True),
    # batches that fill the chip with their suffixes: their workgroups join the prefix's parts
    (130, 1, 8, 2, 128, 700, [(7 * i) % 41 - 1 for i in range(130)], 3, 16, "bf16", True),
    (257, 1, 2, 1, 64, 0, [i % 5 for i in range(257)], 1, 4, "fp16", False),
    (129, 2, 6, 2, 256, 33, [(5 * i) % 9 for i in range(129)], 2, 8, "bf16", False),
    (64, 5, 16, 4, 128, 300, [(11 * i) % 50 for i in range(64)], 4, 16, "bf16", True),
    (32, 5, 32, 8, 80, 0, [i for i in range(32)], 2, 16, "fp16", True),
    (43, 13, 12, 2, 256, 130, [(3 * i) % 33 for i in range(43)], 3, 16, "fp16", False),
    (65, 18, 16, 4, 96, 257, [(9 * i) % 40 for i in range(65)], 3, 16, "bf16", False),
    (64, 25, 24, 4, 128, 65, [(13 * i) % 90 for i in range(64)], 6, 16, "bf16", True),
    (86, 20, 21, 3, 64, 200, [(7 * i) % 60 for i in range(86)], 4, 16, "fp16", True),
    # the same with few rows, with four waves and with eight
    (130, 1, 8, 2, 128, 2100, [(7 * i) % 41 - 1 for i in range(130)], 3, 16, "bf16", True),
    (64, 1, 16, 4, 64, 2150, [(7 * i) % 41 - 1 for i in range(64)], 3, 16, "bf16", True),
    (64, 2, 12, 4, 112, 1100, [(5 * i) % 35 for i in range(64)], 2, 16, "fp16", False),
    (129, 1, 6, 2, 256, 600, [(3 * i) % 17 for i in range(129)], 1, 16, "fp16", False),
    # longer prefixes that the suffixes' workgroups see: by four waves and by eight
    (130, 1, 8, 2, 64, 1999, [(7 * i) % 41 - 1 for i in range(130)], 3, 16, "bf16", True),
    (64, 1, 16, 4, 64, 2047, [(7 * i) % 41 - 1 for i in range(64)], 3, 16, "fp16", False),
    (36, 3, 8, 4, 128, 701, [(7 * i) % 33 - 1 for i in range(36)], 2, 16, "bf16", False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:6]) + f"_{c[8]}_{c[9]}_{'e4m3' if c[10] else 'same'}")
def test_against_64_bits(case):
    c, dtype = build(case, seed=case[0] + case[5])
    got = call(c, dtype)
    check(c, dtype, got)
    again = call(c, dtype, lse=False)                          # the same bits each time, with and without lse
    assert torch.equal(again[0], got[0])


def test_pages_outside_the_cache_are_masked():
    for case in (CASES[3], CASES[7], CASES[10], CASES[17], CASES[18], CASES[19], CASES[20], CASES[21]):
        c, dtype = build(case, seed=3)
        c["prefix_pages"][1] = -1
        c["prefix_pages"][-1] = c["k_pages"].shape[0]
        if c["suffix_pages"] is not None:
            c["suffix_pages"][-1, 0] = 2 ** 31 - 1
        check(c, dtype, call(c, dtype))


def test_lengths_beyond_the_row_of_pages_end_with_it():
    c, dtype = build((3, 1, 4, 2, 64, 20, [32, 32, 32], 2, 16, "bf16", True), seed=4)
    c["suffix_lens"] = torch.tensor([33, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    got = call(c, dtype)
    c["suffix_lens"] = torch.tensor([32, 32, 0], dtype=torch.int32)
    check(c, dtype, got)


def test_no_keys_at_all_and_no_tokens():
    c, dtype = build((2, 3, 4, 2, 64, 0, [2, 0], 1, 16, "bf16", True), seed=5)
    out, lse = call(c, dtype)
    check(c, dtype, (out, lse))
    assert (out[3:] == 0).all() and torch.isneginf(lse[3:]).all() and torch.isneginf(lse[0]).all()
    c, dtype = build((2, 1, 4, 2, 64, 0, [], 0, 16, "bf16", True), seed=5)
    out, lse = call(c, dtype)
    assert (out == 0).all() and torch.isneginf(lse).all()
    c["q"] = c["q"][:0]
    call(c, dtype)


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("batch,prefix", [(1, 400), (1, 640), (40, 640), (70, 640)])
def test_large_scores_and_a_late_maximum(quantised, batch, prefix):
    """Scores that grow from key to key by far more than an exponent holds, and one key that has nearly all the weight at the end."""
    c, dtype = build((batch, 1, 4, 1, 128, prefix, [3] * batch, 1, 16, "bf16", quantised), seed=6, junk=False)
    c["scale"] = 3.0
    check(c, dtype, call(c, dtype))
    c["scale"] = 40.0
    q = c["q"].double()
    got = call(c, dtype)
    assert torch.isfinite(got[0].double()).all() and torch.isfinite(got[1]).all() and torch.isfinite(q).all()
    check(c, dtype, got)


@pytest.mark.parametrize("scale", [1e-39, 1e-37])
def test_a_scale_that_makes_all_scores_alike(scale):
    c, dtype = build((20, 1, 4, 1, 64, 800, [5] * 20, 1, 16, "bf16", True), seed=11)
    c["scale"] = scale
    check(c, dtype, call(c, dtype))


@pytest.mark.parametrize("prefix", [100, 800])
def test_nan_in_a_seen_key_reaches_its_row_alone(prefix):
    c, dtype = build((20, 1, 4, 2, 64, prefix, [5] * 20, 1, 16, "bf16", False), seed=7)
    p = int(c["suffix_pages"][3, 0])
    c["v_pages"][p, 1, 2, 5] = math.nan
    out, lse = call(c, dtype)
    nan = torch.zeros(20, 4, 64, dtype=torch.bool)
    nan[3, 2:, 5] = True
    assert torch.equal(out.isnan(), nan) and torch.isfinite(lse).all()
    c["k_pages"][p, 0, 1, 0] = math.nan
    out, lse = call(c, dtype)
    nan[3, :2] = True
    assert torch.equal(out.isnan(), nan) and torch.equal(lse.isnan(), nan[:, :, 0])


def test_split_states_merge_to_the_same_result():
    """out and lse are what mergestates_run takes: prefix alone and suffixes alone, merged, are the whole."""
    from paper_2601_12698_amd import binding as B
    c, dtype = build((6, 1, 8, 2, 128, 1333, [9, 1, 30, 4, 16, 17], 2, 16, "bf16", True), seed=8)
    whole = call(c, dtype)
    a = call(dict(c, suffix_pages=None, suffix_lens=None), dtype)
    b = call(dict(c, prefix_len=0), dtype)
    va, vb, sa, sb = a[0].cuda(), b[0].cuda(), a[1].cuda(), b[1].cuda()
    vo, so = torch.empty_like(va), torch.empty_like(sa)
    B.mergestates_run(va, sa, vb, sb, vo, so, 48, 128, "bf16")
    check(c, dtype, whole)
    # two more roundings of parts whose magnitudes are at most |v|'s, 4 x 2^-9 with the merge's own
    assert (vo.cpu().double() - whole[0].double()).abs().max() <= 4 * 2.0 ** -9 * float(R.values(c["v_pages"], c["v_scale"]).nan_to_num(0, 0, 0).abs().max())
    assert (so.cpu() - whole[1]).abs().max() <= 2.0 ** -16


def test_a_cache_beyond_32_bits():
    """Pages whose places are past 2^32 bytes and 2^32 / 2 elements."""
    h, d, page = 1, 256, 1024
    pages = 9000                                               # 4.7e9 bytes of bf16 keys
    k, v = (torch.zeros((pages, h, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(1)
    table = torch.tensor([8999, 0, 8500], dtype=torch.int32)
    small = {n: torch.randn((3, h, page, d), generator=g).to(torch.bfloat16) for n in "kv"}
    for i, p in enumerate(table.tolist()):
        k[p], v[p] = small["k"][i].cuda(), small["v"][i].cuda()
    q = torch.randn((2, 4, d), generator=g).to(torch.bfloat16)
    c = dict(q=q, k_pages=small["k"], v_pages=small["v"], k_scale=None, v_scale=None, prefix_pages=torch.arange(3, dtype=torch.int32), prefix_len=2500,
             suffix_pages=None, suffix_lens=None, scale=1 / 16, q_len=1)
    out, lse = torch.empty((2, 4, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 4), device="cuda")
    S.prefixattn_run(q.cuda(), k, v, None, None, table.cuda(), 2500, None, None, out, lse, 1 / 16, "bf16")
    check(c, "bf16", (out.cpu(), lse.cpu()))


@pytest.mark.parametrize("short", [True, False])
def test_on_another_stream_and_in_a_graph_with_growing_suffixes(short):
    prefix = 150 if short else 1150
    c, dtype = build((5, 1, 8, 2, 128, prefix, [64] * 5, 4, 16, "bf16", True), seed=9)
    dev = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in c.items()}
    shape = S.prefixattn_shape(5, 1, 8, 2, 128, 16, c["k_pages"].shape[0], prefix, 4, dtype, True)
    room = torch.empty(S.prefixattn_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros((5, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((5, 8), device="cuda")

    def step(o, s, **more):
        S.prefixattn_run(dev["q"], dev["k_pages"], dev["v_pages"], dev["k_scale"], dev["v_scale"], dev["prefix_pages"], prefix, dev["suffix_pages"],
                         dev["suffix_lens"], o, s, c["scale"], dtype, workspace=room, **more)

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(out, lse, stream=stream)
    stream.synchronize()
    check(c, dtype, (out.cpu(), lse.cpu()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, lse)
    for n in (1, 0, 17, 64, 33):
        dev["suffix_lens"].fill_(n)
        want, ws = torch.empty_like(out), torch.empty_like(lse)
        step(want, ws)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, ws), n


def test_one_workspace_after_the_other_and_refused_where_small():
    c, dtype = build((2, 1, 8, 2, 128, 1600, [5, 16], 1, 16, "bf16", True), seed=1)
    shape = S.prefixattn_shape(2, 1, 8, 2, 128, 16, c["k_pages"].shape[0], 1600, 1, dtype, True)
    n = S.prefixattn_workspace_bytes(shape)
    with pytest.raises(S.AddrmsError, match="workspace has"):
        call(c, dtype, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    room = torch.full((n + 64,), 0xff, dtype=torch.uint8, device="cuda")
    check(c, dtype, call(c, dtype, workspace=room[:n]))
    assert (room[n:] == 0xff).all()
