"""Attention of trees of drafted tokens on the device against its 64-bit form (needs an MI355X).

Bar.  A weight is 2^(fp32 argument), rounded to 16 bits for the second product: half a step of the type, relative.  Its argument is off by
what an fp32 sum of d products is off by, taken as 2^-21 of the sum of their magnitudes (x), in numerator and denominator, and by 2^-19
for the exponential, the running maximum and the sum of weights.  So an output is off by at most
(half a step + 2 x + 2^-18) * sum of weight |v|, and half a step of itself for its own rounding; fp16 weights below 2^-21 of the largest
lose bits, at most 2^-31 of the largest each.  lse is off by x + 2^-18 + 2^-22 |lse|."""
import math

import pytest
import torch

import drafting_ref as D
import serving_ref as R
from paper_2601_12698_amd import drafting
from paper_2601_12698_amd import serving as S

pytestmark = pytest.mark.gpu


def build(case, seed=0, odd=False):
    """A cache whose unused places hold NaN, and a call's other inputs, on the CPU."""
    batch, nodes, hq, hk, d, prefix, lens, width, page, dtype, quantised = case
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
        for j in range(min(max(lens[b], 0) + nodes, width * page)):
            used[int(own[b, j // page]), j % page] = True
    ks = vs = None
    k, v = k.to(R.TYPES[dtype]), v.to(R.TYPES[dtype])
    if quantised:
        (k, ks), (v, vs) = R.quantise(k, dtype), R.quantise(v, dtype)
        k, v = k.to(torch.float8_e4m3fn), v.to(torch.float8_e4m3fn)
    free = ~used[:, None].expand(pages, hk, page)
    for x, s in ((k, ks), (v, vs)):
        if quantised:
            x.view(torch.uint8)[free] = 0x7f
            s[free] = 255
        else:
            x[free] = math.nan
    q = torch.randn((batch * nodes, hq + 3, d), generator=g).to(R.TYPES[dtype])[:, 2:2 + hq]
    masks = D.int64_masks(D.tree_masks(D.rng(seed), batch, nodes, odd))
    return dict(q=q, k_pages=k, v_pages=v, k_scale=ks, v_scale=vs, prefix_pages=table, prefix_len=prefix, suffix_pages=own if width else None,
                suffix_lens=torch.tensor(lens, dtype=torch.int32) if width else None, masks=masks, scale=d ** -0.5), dtype


def device(c):
    dev = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in c.items()}
    if c["q"].stride() != dev["q"].stride():
        big = torch.zeros(c["q"].shape[0], c["q"].shape[1] + 3, c["q"].shape[2], dtype=c["q"].dtype, device="cuda")
        dev["q"] = big[:, 2:2 + c["q"].shape[1]].copy_(c["q"])
    return dev


def run(dev, dtype, out, lse, **more):
    drafting.treeattn_run(dev["q"], dev["k_pages"], dev["v_pages"], dev["k_scale"], dev["v_scale"], dev["prefix_pages"], dev["prefix_len"],
                          dev["suffix_pages"], dev["suffix_lens"], dev["masks"], out, lse, dev["scale"], dtype, **more)


def call(c, dtype, lse=True, **more):
    out = torch.full(c["q"].shape, math.nan, dtype=c["q"].dtype, device="cuda")
    s = torch.full(c["q"].shape[:2], math.nan, device="cuda") if lse else None
    run(device(c), dtype, out, s, **more)
    torch.cuda.synchronize()
    return out.cpu(), None if s is None else s.cpu()


def check(c, dtype, got, want=None):
    want, lse, size = want or D.tree_attention(**c)
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
    # batch, nodes, q heads, kv heads, d, prefix, own keys, pages of a sequence, page, type, quantised
    (1, 1, 1, 1, 16, 0, [0], 1, 1, "bf16", False),
    (1, 1, 4, 1, 128, 0, [40], 3, 16, "bf16", True),
    (2, 4, 8, 2, 128, 37, [5, 12], 1, 16, "bf16", True),
    (2, 3, 8, 2, 64, 300, [0, 27], 2, 16, "fp16", True),
    (3, 2, 5, 5, 96, 129, [0, 1, 40], 3, 16, "fp16", False),
    (1, 2, 8, 1, 256, 700, [130], 3, 64, "bf16", False),
    (7, 4, 8, 2, 128, 331, [0, 1, 17, 60, 61, 65, -4], 8, 8, "bf16", True),
    (9, 4, 4, 1, 64, 100, [0, 1, 2, 3, 4, 5, 33, 20, 7], 3, 16, "bf16", True),
    (3, 7, 8, 2, 80, 65, [3, 7, 100], 7, 16, "fp16", True),
    (2, 40, 8, 2, 128, 130, [30, 35], 5, 16, "bf16", False),
    (1, 64, 2, 1, 256, 64, [260], 6, 64, "bf16", True),
    (2, 64, 16, 2, 128, 0, [190, 0], 16, 16, "bf16", False),
    (2, 63, 5, 1, 64, 0, [1000, 77], 67, 16, "fp16", False),
    (2, 64, 24, 2, 112, 70, [129, 5], 4, 64, "fp16", True),
    (5, 2, 6, 3, 48, 1000, [998, 0, 510, 511, 3], 250, 4, "fp16", False),
    (4, 13, 32, 8, 128, 0, [3000, 301, 0, 1257], 100, 32, "bf16", True),
    (3, 16, 5, 1, 128, 5000, [100, 0, 1700], 30, 64, "bf16", True),
    (2, 12, 16, 2, 256, 900, [1200, 40], 20, 64, "fp16", False),
    (2, 9, 8, 1, 256, 0, [2500, 40], 40, 64, "bf16", True),
    # long shared prefixes, and sequences that are pages short for their nodes
    (20, 2, 8, 2, 256, 900, [i % 11 for i in range(20)], 1, 16, "bf16", True),
    (24, 3, 5, 1, 112, 777, [i % 5 for i in range(24)], 1, 4, "bf16", False),
    (13, 1, 4, 1, 256, 577, [2] * 13, 1, 32, "fp16", False),
    # batches that fill the chip
    (130, 2, 8, 2, 128, 700, [(7 * i) % 41 - 1 for i in range(130)], 3, 16, "bf16", True),
    (257, 1, 2, 1, 64, 0, [i % 5 for i in range(257)], 2, 4, "fp16", False),
    (129, 2, 6, 2, 256, 33, [(5 * i) % 9 for i in range(129)], 2, 8, "bf16", False),
    (64, 5, 16, 4, 128, 300, [(11 * i) % 50 for i in range(64)], 4, 16, "bf16", True),
    (32, 5, 32, 8, 80, 0, [i for i in range(32)], 3, 16, "fp16", True),
    (43, 13, 12, 2, 256, 130, [(3 * i) % 33 for i in range(43)], 3, 16, "fp16", False),
    (65, 18, 16, 4, 96, 257, [(9 * i) % 40 for i in range(65)], 4, 16, "bf16", False),
    (64, 25, 24, 4, 128, 65, [(13 * i) % 90 for i in range(64)], 8, 16, "bf16", True),
    (86, 20, 21, 3, 64, 200, [(7 * i) % 60 for i in range(86)], 6, 16, "fp16", True),
    (64, 64, 20, 4, 128, 0, [(29 * i) % 200 for i in range(64)], 5, 64, "bf16", False),
    # the same with a prefix that the sequences' workgroups see before their own keys, in tiles of its own
    (64, 16, 16, 4, 128, 130, [(7 * i) % 50 for i in range(64)], 5, 16, "bf16", False),
    (64, 16, 16, 4, 64, 64, [(7 * i) % 50 for i in range(64)], 5, 16, "fp16", True),
    (64, 30, 16, 4, 112, 63, [(5 * i) % 70 for i in range(64)], 7, 16, "fp16", False),
    (130, 10, 16, 2, 256, 70, [(3 * i) % 30 for i in range(130)], 3, 16, "bf16", True),
    (130, 10, 16, 2, 256, 200, [(3 * i) % 30 for i in range(130)], 5, 8, "fp16", False),
    (64, 40, 20, 4, 128, 700, [(9 * i) % 100 for i in range(64)], 5, 32, "bf16", True),
    # many sequences beside a prefix in more parts than a sequence's workgroup joins
    (300, 1, 1, 1, 64, 9000, [(5 * i) % 14 for i in range(300)], 2, 8, "bf16", False),
    # a prefix and nothing else
    (64, 40, 20, 4, 128, 300, [], 0, 32, "bf16", True),
    (64, 3, 8, 4, 128, 100, [], 0, 32, "fp16", False),
    (2, 10, 8, 2, 256, 40, [], 0, 8, "bf16", False),
]
SHARED_OUT = [
    # many sequences, a few of them long: cut although their workgroups nearly fill the chip, alone and beside a prefix
    (33, 17, 8, 8, 64, 0, [2200 if i % 16 == 3 else (37 * i) % 90 for i in range(33)], 70, 32, "bf16", False),
    (33, 17, 8, 8, 64, 1500, [2200 if i % 16 == 3 else (37 * i) % 90 for i in range(33)], 70, 32, "fp16", True),
    (36, 9, 16, 8, 128, 130, [2210 if i == 7 else (31 * i) % 60 for i in range(36)], 35, 64, "bf16", True),
    # sequences of few keys, of few rows, beside a prefix seen by many rows
    (3, 15, 1, 1, 256, 2500, [6, 0, 40], 1, 64, "bf16", True),
    (12, 4, 8, 4, 128, 1300, [(17 * i) % 100 for i in range(12)], 7, 16, "bf16", False),
    (7, 7, 8, 2, 256, 1000, [(29 * i) % 90 for i in range(7)], 4, 32, "fp16", False),
    # few keys in all, of many rows; rows joined by several workgroups each; heads beyond 128 of few rows
    (20, 36, 32, 4, 128, 0, [(19 * i) % 200 for i in range(20)], 4, 64, "bf16", False),
    (20, 30, 16, 2, 64, 90, [(23 * i) % 300 for i in range(20)], 6, 64, "fp16", True),
    (2, 15, 1, 1, 256, 80, [3000, 1700], 95, 32, "bf16", True),
    (2, 3, 4, 1, 96, 0, [2500, 60], 80, 32, "fp16", False),
    (1, 2, 4, 1, 80, 40, [4000], 64, 64, "bf16", True),
    (3, 4, 8, 2, 256, 20, [1300, 900, 2], 42, 32, "fp16", False),
    (1, 1, 260, 260, 256, 1100, [20], 1, 32, "bf16", True),
    (2, 4, 4, 1, 256, 700, [], 0, 32, "bf16", False),
    # rows in tiles of 128 where tiles of 256 would leave a half empty; a longer prefix before sequences that nearly fill the chip
    (6, 52, 10, 2, 128, 0, [(211 * i) % 1400 for i in range(6)], 46, 32, "bf16", True),
    (2, 28, 10, 1, 128, 1300, [40, 600], 20, 32, "fp16", False),
    (30, 14, 16, 8, 128, 900, [(11 * i) % 70 for i in range(30)], 10, 32, "bf16", False),
    # a prefix in as many splits as rounds of workgroups hold, and in the share of the places that its keys are of all
    (20, 40, 8, 2, 128, 1100, [(41 * i) % 130 for i in range(20)], 3, 64, "bf16", False),
    (44, 16, 32, 8, 64, 900, [(13 * i) % 60 for i in range(44)], 3, 32, "bf16", True),
    (5, 30, 16, 4, 96, 2100, [1400, 3, 0, 77, 600], 30, 64, "fp16", False),
]
name = lambda c: "x".join(str(x) for x in c[:6]) + f"_{c[8]}_{c[9]}_{'e4m3' if c[10] else 'same'}"  # noqa: E731


@pytest.mark.parametrize("case", SHARED_OUT, ids=name)
def test_work_that_is_shared_out_against_64_bits(case):
    c, dtype = build(case, seed=case[0] + case[5], odd=case[0] % 2 == 0)
    got = call(c, dtype)
    check(c, dtype, got)
    again = call(c, dtype)
    assert torch.equal(again[0].view(torch.uint8), got[0].view(torch.uint8)) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("case", CASES, ids=name)
def test_against_64_bits(case):
    c, dtype = build(case, seed=case[0] + case[5], odd=case[0] % 2 == 0)
    got = call(c, dtype)
    check(c, dtype, got)
    again = call(c, dtype, lse=False)                          # the same bits each time, with and without lse
    assert torch.equal(again[0], got[0])


def test_pages_outside_the_cache_are_masked():
    for case in (CASES[2], CASES[6], CASES[8], CASES[9], CASES[11], CASES[15], CASES[17], CASES[19]):
        c, dtype = build(case, seed=3)
        if case[5]:
            c["prefix_pages"][1] = -1
            c["prefix_pages"][-1] = c["k_pages"].shape[0]
        c["suffix_pages"][-1, 0] = 2 ** 31 - 1
        check(c, dtype, call(c, dtype))


def test_lengths_beyond_the_row_of_pages():
    """Keys that the row of pages does not hold are not there, whoever sees them."""
    c, dtype = build((4, 3, 4, 2, 64, 20, [32, 32, 32, 30], 2, 16, "bf16", True), seed=4)
    c["suffix_lens"] = torch.tensor([33, 2 ** 31 - 1, -2 ** 31, 30], dtype=torch.int32)
    check(c, dtype, call(c, dtype))
    c, dtype = build((2, 40, 8, 2, 128, 0, [40, 40], 2, 16, "fp16", False), seed=4)
    c["suffix_lens"] = torch.tensor([2 ** 31 - 1, 20], dtype=torch.int32)
    check(c, dtype, call(c, dtype))


def test_no_keys_at_all_and_no_sequences():
    c, dtype = build((2, 3, 4, 2, 64, 0, [0, 0], 1, 16, "bf16", True), seed=5)
    c["masks"][:, 1] = 0
    out, lse = call(c, dtype)
    check(c, dtype, (out, lse))
    assert (out.view(2, 3, 4, 64)[:, 1] == 0).all() and torch.isneginf(lse.view(2, 3, 4)[:, 1]).all()
    c, dtype = build((2, 1, 4, 2, 64, 0, [], 0, 16, "bf16", True), seed=5)
    out, lse = call(c, dtype)
    assert (out == 0).all() and torch.isneginf(lse).all()
    c["q"], c["masks"] = c["q"][:0], c["masks"][:0]
    call(c, dtype)


@pytest.mark.parametrize("case", [CASES[2], CASES[8], CASES[9], CASES[14], CASES[15], CASES[27]], ids=name)
def test_a_chain_is_the_order_of_prefixattn(case):
    """Lower triangles: what prefixattn_run gives where the last queries of a sequence are its nodes, within both operators' bars."""
    case = case[:6] + ([max(n, 0) for n in case[6]],) + case[7:]
    c, dtype = build(case, seed=8)
    nodes, room = case[1], case[7] * case[8]
    c["masks"][:] = torch.tensor([D.signed((2 << i) - 1) for i in range(nodes)])
    c["suffix_lens"].clamp_(max=room - nodes)
    want = D.tree_attention(**c)
    check(c, dtype, call(c, dtype), want)
    dev = device(c)
    out, lse = torch.empty(c["q"].shape, dtype=c["q"].dtype, device="cuda"), torch.empty(c["q"].shape[:2], device="cuda")
    S.prefixattn_run(dev["q"], dev["k_pages"], dev["v_pages"], dev["k_scale"], dev["v_scale"], dev["prefix_pages"], c["prefix_len"], dev["suffix_pages"],
                     dev["suffix_lens"] + nodes, out, lse, c["scale"], dtype, q_len=nodes)
    check(c, dtype, (out.cpu(), lse.cpu()), want)


STRAYS = [(2, 4, 8, 2, 128, 37, [5, 12], 1, 16, "bf16", False), (3, 4, 4, 1, 64, 0, [4, 9, 2], 2, 8, "fp16", True), (2, 2, 8, 1, 256, 0, [31, 33], 3, 16, "bf16", False),
          (2, 2, 8, 1, 256, 20, [1, 33], 3, 16, "fp16", True), (130, 2, 8, 2, 128, 60, [(7 * i) % 41 for i in range(130)], 3, 16, "bf16", False),
          (129, 2, 6, 2, 256, 600, [(3 * i) % 17 for i in range(129)], 2, 16, "fp16", False), (3, 7, 8, 2, 80, 65, [3, 7, 100], 7, 16, "fp16", True),
          (2, 14, 8, 2, 128, 700, [14, 70], 6, 16, "bf16", False), (2, 40, 8, 2, 128, 130, [25, 35], 5, 16, "bf16", False),
          (2, 30, 8, 2, 64, 1000, [20, 140], 11, 16, "fp16", True), (2, 60, 8, 2, 128, 0, [60, 100], 11, 16, "bf16", True),
          (1, 64, 4, 1, 256, 64, [130], 13, 16, "bf16", True), (2, 20, 2, 1, 192, 300, [12, 40], 4, 16, "fp16", False),
          (64, 25, 24, 4, 128, 65, [(13 * i) % 60 for i in range(64)], 6, 16, "fp16", False), (2, 64, 20, 2, 96, 0, [700, 30], 50, 16, "bf16", False)]


@pytest.mark.parametrize("case", STRAYS, ids=name)
def test_values_of_nodes_that_are_not_seen_do_not_arrive(case):
    """Values of some nodes are NaN or infinite: nodes that do not see them get what they would without, the others what the formula gives."""
    c, dtype = build(case, seed=case[0] + case[4])
    batch, nodes, d, page = case[0], case[1], case[4], case[8]
    clean = {n: x.clone() if n == "v_pages" else x for n, x in c.items()}
    for b in range(batch):
        if b % 3 == 2:
            continue
        for node, head, e, value in ((nodes - 1, 0, 3, math.nan), (nodes // 2, 1, d - 1, math.inf), (nodes // 2, 0, d // 2, -math.inf), (nodes // 3, 0, 9, math.inf),
                                     (nodes - 1, 0, 9, -math.inf), (0, 3, 0, math.nan)):
            j = case[6][b] + node
            if j >= case[7] * page:
                continue
            p, o, head = int(c["suffix_pages"][b, j // page]), j % page, head % case[3]
            if case[10]:
                c["v_pages"].view(torch.uint8)[p, head, o, e] = 0x7f if value > 0 or math.isnan(value) else 0xff
                clean["v_pages"].view(torch.uint8)[p, head, o, e] = 0
            else:
                c["v_pages"][p, head, o, e] = value
                clean["v_pages"][p, head, o, e] = 0
    got = call(c, dtype)
    want, _, _ = D.tree_attention(**c)
    odd = ~torch.isfinite(want)
    assert odd.any() and not odd.all()
    assert torch.equal(got[0].isnan(), want.isnan())
    assert torch.equal(got[0].double()[odd & ~want.isnan()], want[odd & ~want.isnan()])
    plain = D.tree_attention(**clean)
    assert torch.equal(plain[0][~odd], want[~odd])
    check(clean, dtype, (torch.where(odd, plain[0], got[0].double()).to(got[0].dtype), got[1]), plain)
    # the workspace of a call with strays serves one without
    fine = call(clean, dtype)
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    call(c, dtype, workspace=room)
    again = call(clean, dtype, workspace=room)
    assert torch.equal(again[0], fine[0]) and torch.equal(again[1], fine[1])


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("nodes,heads", [(3, 4), (40, 8), (64, 12)])
def test_nan_in_keys_that_are_not_seen(nodes, heads, quantised):
    """All keys and values of the nodes are NaN: a node that sees none of them is as without a tree, one that sees one is NaN."""
    c, dtype = build((2, nodes, heads, 2, 128, 0, [70, 33], 9, 16, "bf16", quantised), seed=nodes)
    for b in range(2):
        for i in range(nodes):
            j = int(c["suffix_lens"][b]) + i
            for n in ("k_pages", "v_pages"):
                c[n].view(torch.uint8)[int(c["suffix_pages"][b, j // 16]), :, j % 16] = 0x7f if quantised else 0xff
    c["masks"][:, ::2] = 0
    out, lse = (x.view(2, nodes, heads, -1) for x in call(c, dtype))
    assert out[:, 1::2].isnan().logical_or(c["masks"][:, 1::2, None, None] == 0).all() and torch.isfinite(out[:, ::2]).all()
    c["masks"][:] = 0
    check(c, dtype, call(c, dtype))


def test_a_cache_beyond_32_bits():
    """Pages whose places are past 2^32 bytes and 2^32 / 2 elements."""
    h, d, page, pages = 1, 256, 1024, 9000                     # 4.7e9 bytes of bf16 keys
    k, v = (torch.zeros((pages, h, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(1)
    table = torch.tensor([[8999, 0, 8500]], dtype=torch.int32)
    small = {n: torch.randn((3, h, page, d), generator=g).to(torch.bfloat16) for n in "kv"}
    for i, p in enumerate(table[0].tolist()):
        k[p], v[p] = small["k"][i].cuda(), small["v"][i].cuda()
    q = torch.randn((6, 4, d), generator=g).to(torch.bfloat16)
    c = dict(q=q, k_pages=small["k"], v_pages=small["v"], k_scale=None, v_scale=None, prefix_pages=None, prefix_len=0,
             suffix_pages=torch.arange(3, dtype=torch.int32)[None], suffix_lens=torch.tensor([2500], dtype=torch.int32),
             masks=D.int64_masks(D.tree_masks(D.rng(1), 1, 6)), scale=1 / 16)
    out, lse = torch.empty((6, 4, d), dtype=torch.bfloat16, device="cuda"), torch.empty((6, 4), device="cuda")
    drafting.treeattn_run(q.cuda(), k, v, None, None, None, 0, table.cuda(), c["suffix_lens"].cuda(), c["masks"].cuda(), out, lse, 1 / 16, "bf16")
    check(c, "bf16", (out.cpu(), lse.cpu()))


@pytest.mark.parametrize("case", [(5, 3, 8, 2, 128, 150, [64] * 5, 5, 16, "bf16", True), (5, 20, 8, 2, 128, 1150, [64] * 5, 6, 16, "bf16", True),
                                  (3, 20, 8, 2, 64, 0, [500] * 3, 40, 16, "fp16", False)], ids=name)
def test_on_another_stream_and_in_a_graph_with_other_lengths_and_masks(case):
    c, dtype = build(case, seed=9)
    batch, nodes, hq, hk, d, prefix, lens, width, page, _, quantised = case
    dev = device(c)
    shape = S.prefixattn_shape(batch, nodes, hq, hk, d, page, c["k_pages"].shape[0], prefix, width, dtype, quantised)
    room = torch.empty(max(16, drafting.treeattn_workspace_bytes(shape)), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(c["q"].shape, dtype=c["q"].dtype, device="cuda"), torch.zeros(c["q"].shape[:2], device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(dev, dtype, out, lse, workspace=room, stream=stream)
    stream.synchronize()
    check(c, dtype, (out.cpu(), lse.cpu()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(dev, dtype, out, lse, workspace=room)
    for i, n in enumerate((1, 0, 17, lens[0], 33)):
        dev["suffix_lens"].fill_(n)
        dev["masks"].copy_(D.int64_masks(D.tree_masks(D.rng(i), batch, nodes)))
        want, ws = torch.empty_like(out), torch.empty_like(lse)
        run(dev, dtype, want, ws, workspace=room)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, ws), n


def test_the_workspace_is_as_long_as_it_says():
    case = (2, 12, 8, 2, 128, 1600, [5, 700], 50, 16, "bf16", True)
    c, dtype = build(case, seed=1)
    shape = S.prefixattn_shape(2, 12, 8, 2, 128, 16, c["k_pages"].shape[0], 1600, 50, dtype, True)
    n = drafting.treeattn_workspace_bytes(shape)
    with pytest.raises(S.AddrmsError, match="workspace has"):
        call(c, dtype, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    room = torch.full((n + 64,), 0xff, dtype=torch.uint8, device="cuda")
    check(c, dtype, call(c, dtype, workspace=room[:n]))
    assert (room[n:] == 0xff).all()


def test_queries_at_any_elements_address():
    case = (2, 7, 4, 2, 64, 0, [50, 3], 4, 16, "bf16", False)
    c, dtype = build(case, seed=2)
    dev = device(c)
    whole = torch.zeros(14 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")
    dev["q"] = whole[1:].view(14, 4, 64).copy_(c["q"])
    out, lse = torch.empty(14, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(14, 4, device="cuda")
    run(dev, dtype, out, lse)
    check(c, dtype, (out.cpu(), lse.cpu()))
