"""Attention of trees on every way that its plan may go (tree_paths.py), against 64 bits: as the values are, and with keys and values of some
nodes that are no finite numbers, which only the rows that see them may notice (needs an MI355X).

The bar is that of test_gpu_treeattn.py: an output is off by at most (half a step + 2 x + 2^-18) * sum of weight |v| and half a step of itself,
with x = 2^-21 times the sum of a score's magnitudes; fp16 weights below 2^-21 of the largest lose at most 2^-31 of the largest each.  lse is
off by x + 2^-18 + 2^-22 |lse|."""
import math
import random

import pytest
import torch

import drafting_ref as D
import serving_ref as R
import tree_paths as P
from paper_2601_12698_amd import drafting

pytestmark = pytest.mark.gpu


def lengths(batch, nodes, room):
    """Keys before the trees: a sequence that fills its pages, one whose nodes have no place, an empty one, and others."""
    n = [(i * 7919 + 13) % (room + 1) for i in range(batch)]
    n[0] = max(0, room - nodes)
    if batch > 2:
        n[1], n[-1] = room, 0
    return n


def stored(x, dtype, quantised):
    """(codes or elements, scale bytes): rows with the least power of two that brings them within 448."""
    if not quantised:
        return x.to(R.TYPES[dtype]), None
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def values(x, s):
    return x.double() if s is None else torch.ldexp(x.double(), s.int()[..., None] - 127)


def build(case):
    """A call's inputs on the device; places of the cache that no sequence has hold NaN."""
    batch, nodes, hq, hk, d, prefix, width, page, dtype, quantised = case
    seed = sum(case[:8])
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages, first = P.pages_of(case), -(-prefix // page)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table, own = order[:first].contiguous(), order[first:first + batch * width].view(batch, width).contiguous()
    lens = torch.tensor(lengths(batch, nodes, width * page), dtype=torch.int32, device="cuda")
    used = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    used[table.long()] = (torch.arange(first * page, device="cuda") < prefix).view(first, page)
    used[own.long()] = (torch.arange(width * page, device="cuda") < (lens + nodes)[:, None]).view(batch, width, page)
    cache = []
    for name in "kv":
        x = torch.randn((pages, hk, page, d), generator=g, device="cuda")
        x = x * (1 + 5 * (torch.arange(d, device="cuda") % 13 == 3)) if name == "k" else x
        x, s = stored(x, dtype, quantised)
        raw = x.view(torch.uint8) if quantised else x
        raw.masked_fill_(~used[:, None, :, None], 0x7f if quantised else math.nan)
        cache.append((x, s if s is None else s.masked_fill_(~used[:, None], 255)))
    q = torch.randn((batch * nodes, hq + 3, d), generator=g, device="cuda").to(R.TYPES[dtype])[:, 2:2 + hq]
    masks = D.int64_masks(D.tree_masks(random.Random(seed), batch, nodes, odd=seed % 2 == 0)).cuda()
    return dict(q=q, k_pages=cache[0][0], v_pages=cache[1][0], k_scale=cache[0][1], v_scale=cache[1][1], prefix_pages=table, prefix_len=prefix,
                suffix_pages=own if width else None, suffix_lens=lens if width else None, masks=masks, scale=d ** -0.5)


def exact(c):
    """(out, lse, size, x) in 64 bits, sequence by sequence; values that are no finite numbers count where a row sees them."""
    batch, nodes = c["masks"].shape
    rows, hq, d = c["q"].shape
    _, hk, page, _ = c["k_pages"].shape
    group, prefix = hq // hk, c["prefix_len"]
    width = 0 if c["suffix_pages"] is None else c["suffix_pages"].shape[1] * page

    def gather(n, table, count):
        x, s = c[n + "_pages"], c[n + "_scale"]
        at = table.long()
        x = values(x.view(torch.uint8)[at].view(x.dtype) if s is not None else x[at], None if s is None else s[at])
        return x.transpose(0, 1).flatten(1, 2)[:, :count]                                # [kv heads, keys, d]

    out, size = (torch.zeros((batch, nodes, hk, group, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse, x = (torch.zeros((batch, nodes, hk, group), dtype=torch.float64, device="cuda") for _ in range(2))
    q = c["q"].double().view(batch, nodes, hk, group, d)
    pre = {n: gather(n, c["prefix_pages"], prefix) for n in "kv"}
    lens = c["suffix_lens"].tolist() if width else [0] * batch
    for b in range(batch):
        count = min(lens[b] + nodes, width)
        k, v = (torch.cat((pre[n], gather(n, c["suffix_pages"][b], count)), 1) if width else pre[n] for n in "kv")
        node = torch.arange(k.shape[1], device="cuda") - prefix - lens[b]
        if k.shape[1] == 0:
            lse[b] = -math.inf
            continue
        seen = (node < 0) | ((c["masks"][b, :, None] >> node.clamp(0, 63) & 1) != 0)     # [nodes, keys]
        fine = torch.isfinite(k).all(-1)                                                 # [kv heads, keys]
        z = (q[b].permute(1, 0, 2, 3).reshape(hk, nodes * group, d) @ torch.where(fine[..., None], k, 0.0).transpose(1, 2).contiguous()) * c["scale"]
        z = z.view(hk, nodes, group, -1).masked_fill(~seen[:, None], -math.inf)
        top = z.amax(-1, keepdim=True)
        w = torch.where(top == -math.inf, 0.0, (z - top).exp())
        total = w.sum(-1)
        w = (w / torch.where(total > 0, total, 1.0)[..., None]).view(hk, nodes * group, -1)
        whole = torch.where(torch.isfinite(v), v, 0.0)
        o, t = ((w @ y).view(hk, nodes, group, d) for y in (whole, whole.abs()))
        eye = seen.double()                                                              # of each row: how many such values it sees
        nan, up, down = (torch.matmul(eye, m.double())[:, :, None] > 0 for m in (v.isnan(), v == math.inf, v == -math.inf))
        o = torch.where(up, math.inf, torch.where(down, -math.inf, o))
        bad = torch.matmul(eye, (~fine).double()[..., None])[:, :, None] > 0             # [kv heads, nodes, 1, 1]: a key that is seen is none
        o = torch.where(nan | (up & down) | bad, math.nan, o)
        size[b], out[b] = t.permute(1, 0, 2, 3), o.permute(1, 0, 2, 3)
        lse[b] = torch.where(bad[..., 0], math.nan, top[..., 0] + total.log()).permute(1, 0, 2)
        x[b] = 2.0 ** -21 * c["scale"] * q[b].abs().sum(-1) * torch.where(fine[..., None], k, 0.0).abs().max()
    return out.view(rows, hq, d), lse.view(rows, hq), size.view(rows, hq, d), x.view(rows, hq)


def call(c, dtype, room=None):
    out = torch.full(c["q"].shape, math.nan, dtype=c["q"].dtype, device="cuda")
    lse = torch.full(c["q"].shape[:2], 7.0, device="cuda")
    drafting.treeattn_run(c["q"], c["k_pages"], c["v_pages"], c["k_scale"], c["v_scale"], c["prefix_pages"], c["prefix_len"], c["suffix_pages"], c["suffix_lens"],
                          c["masks"], out, lse, c["scale"], dtype, workspace=room)
    return out, lse


def check(c, dtype, got, want):
    out, lse, size, x = want
    fine, half = torch.isfinite(out), R.HALF_STEP[dtype]
    assert torch.equal(got[0].isnan(), out.isnan())
    assert torch.equal(got[0].double()[~fine].nan_to_num(nan=0.0), out[~fine].nan_to_num(nan=0.0))
    keys = c["prefix_len"] + (0 if c["suffix_pages"] is None else c["suffix_pages"].shape[1] * c["k_pages"].shape[2])
    most = values(c["v_pages"], c["v_scale"])
    low = keys * 2.0 ** -31 * float(torch.where(torch.isfinite(most), most, 0.0).abs().max()) + 2.0 ** -25 if dtype == "fp16" else 0.0
    limit = (half + 2 * x[..., None] + 2.0 ** -18) * size * (1 + half) + half * out.abs() + low
    off = (got[0].double() - out).abs()[fine] / limit[fine].clamp(min=1e-300)
    assert off.numel() == 0 or float(off.max()) <= 1, float(off.max())
    assert torch.equal(got[1].isnan(), lse.isnan()) and torch.equal(torch.isneginf(got[1]), torch.isneginf(lse))
    fine = torch.isfinite(lse)
    assert ((got[1].double() - lse).abs()[fine] <= (x + 2.0 ** -18 + 2.0 ** -22 * lse.abs())[fine]).all()


@pytest.mark.parametrize("case", P.WITHOUT_OWN, ids=P.name)
def test_a_prefix_alone_seen_by_many_workgroups(case):
    c = build(case)
    check(c, case[8], call(c, case[8]), exact(c))


@pytest.mark.parametrize("case", P.CASES, ids=P.name)
def test_every_way_against_64_bits(case):
    batch, nodes, hq, hk, d, prefix, width, page, dtype, quantised = case
    print("case", case, flush=True)
    c = build(case)
    want = exact(c)
    room = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    plain = call(c, dtype, room)
    check(c, dtype, plain, want)
    if not width:
        return
    # values of some nodes, and the keys of one, are no finite numbers
    strange = {n: x.clone() if n in ("k_pages", "v_pages") else x for n, x in c.items()}
    lens = c["suffix_lens"].tolist()
    for b in range(0, batch, 2):
        for n, node, head, e, value in (("v", nodes - 1, 0, 3, math.nan), ("v", nodes // 2, 1, d - 1, math.inf), ("v", nodes // 2, 0, d // 2, -math.inf),
                                        ("v", nodes // 3, 0, 9, math.inf), ("v", nodes - 1, 0, 9, -math.inf), ("v", nodes * 2 // 3, hk - 1, 17, math.nan),
                                        ("k", nodes * 3 // 4, hk - 1, 5, math.nan)):
            j = lens[b] + node
            if j >= width * page or (n == "k" and b % 4):
                continue
            x = strange[n + "_pages"]
            place = int(c["suffix_pages"][b, j // page]), head % hk, j % page, e % d
            if quantised:
                x.view(torch.uint8)[place] = 0x7f
            else:
                x[place] = value
    want = exact(strange)
    check(strange, dtype, call(strange, dtype, room), want)
    # and nothing of them is left in the workspace
    again = call(c, dtype, room)
    assert torch.equal(again[0].view(torch.int16), plain[0].view(torch.int16)) and torch.equal(again[1].view(torch.int32), plain[1].view(torch.int32))
