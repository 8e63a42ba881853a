"""Attention over a shared prefix where a later token's values are no finite numbers: a query that does not see the token gets what it
would get without it, a query that sees it gets what the formula gives (needs an MI355X).  Bars as in test_gpu_prefixattn.py."""
import math

import pytest
import torch

import serving_ref as R
from test_gpu_prefixattn import build, call, check

pytestmark = pytest.mark.gpu

# batch, q_len, q heads, kv heads, d, prefix, suffix lengths, pages of a suffix, page, type, quantised: every form of a suffix's workgroup,
# alone, seeing a short prefix itself, beside a long one, and joining its parts
CASES = [
    (3, 4, 4, 1, 64, 0, [4, 9, 2], 2, 8, "bf16", False),
    (3, 4, 4, 1, 64, 0, [4, 9, 2], 2, 8, "fp16", True),
    (2, 4, 8, 2, 128, 37, [5, 16], 1, 16, "bf16", False),
    (2, 5, 6, 2, 128, 37, [3, 40], 3, 16, "fp16", True),
    (3, 3, 5, 5, 96, 0, [2, 70, 33], 5, 16, "fp16", False),
    (2, 2, 8, 1, 256, 0, [1, 33], 3, 16, "bf16", False),
    (2, 2, 8, 1, 256, 20, [1, 33], 3, 16, "fp16", True),
    (3, 4, 4, 1, 128, 5000, [100, 2, 300], 20, 16, "bf16", True),
    (5, 4, 4, 1, 256, 3000, [100, 2, 300, 0, 3], 20, 16, "fp16", False),
    (130, 2, 8, 2, 128, 60, [(7 * i) % 41 - 1 for i in range(130)], 3, 16, "bf16", False),
    (64, 2, 12, 4, 112, 1100, [(5 * i) % 35 for i in range(64)], 3, 16, "fp16", False),
    (129, 2, 6, 2, 256, 600, [(3 * i) % 17 for i in range(129)], 2, 16, "fp16", False),
    (3, 7, 8, 2, 80, 65, [3, 7, 100], 7, 16, "fp16", True),
    (2, 14, 8, 2, 128, 700, [14, 90], 6, 16, "bf16", False),
    (2, 40, 8, 2, 128, 130, [40, 75], 5, 16, "bf16", False),
    (2, 30, 8, 2, 64, 1000, [20, 175], 11, 16, "fp16", True),
    (2, 60, 8, 2, 128, 0, [60, 175], 11, 16, "bf16", True),
    (2, 80, 8, 2, 64, 40, [60, 175], 11, 16, "bf16", False),
    (1, 150, 2, 1, 256, 64, [260], 17, 16, "bf16", True),
    (2, 20, 2, 1, 192, 300, [12, 60], 4, 16, "fp16", False),
    (64, 5, 16, 4, 128, 300, [(11 * i) % 50 for i in range(64)], 4, 16, "bf16", True),
    (65, 18, 16, 4, 96, 257, [(9 * i) % 40 for i in range(65)], 3, 16, "bf16", False),
    (64, 25, 24, 4, 128, 65, [(13 * i) % 90 for i in range(64)], 6, 16, "fp16", False),
]


def spoil(c, dtype, bad):
    """Values of some of each sequence's last keys: `bad` lists (tokens from the end, key head, element, value)."""
    page = c["k_pages"].shape[2]
    for b, n in enumerate(c["suffix_lens"].tolist()):
        for back, head, e, value in bad:
            j = n - 1 - back
            if j < 0 or (b + back) % 3 == 2:                   # some sequences keep theirs
                continue
            p, o = int(c["suffix_pages"][b, j // page]), j % page
            head %= c["v_pages"].shape[1]
            if c["v_scale"] is None:
                c["v_pages"][p, head, o, e] = value
            else:
                c["v_pages"].view(torch.uint8)[p, head, o, e] = 0x7f if value > 0 or math.isnan(value) else 0xff      # either NaN


def check_strays(c, dtype, got):
    want, lse, _ = R.attention(**c)
    odd = ~torch.isfinite(want)
    assert odd.any()
    nan = want.isnan()
    assert torch.equal(got[0].isnan(), nan)
    assert torch.equal(got[0].double()[odd & ~nan], want[odd & ~nan])
    clean = dict(c)
    v = c["v_pages"].clone()
    x = R.values(v, c["v_scale"])
    if c["v_scale"] is None:
        v[~torch.isfinite(x)] = 0
    else:
        v.view(torch.uint8)[~torch.isfinite(x)] = 0
    clean["v_pages"] = v
    # elsewhere a stray value has no part, so that zeros in its place change nothing there
    plain, _, _ = R.attention(**clean)
    assert torch.equal(plain[~odd], want[~odd])
    check(clean, dtype, (torch.where(odd, plain, got[0].double()).to(got[0].dtype), got[1]))


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:6]) + f"_{c[8]}_{c[9]}_{'e4m3' if c[10] else 'same'}")
def test_a_later_tokens_values_do_not_reach_earlier_queries(case):
    c, dtype = build(case, seed=case[0] + case[4])
    d = case[4]
    spoil(c, dtype, [(0, 0, 3, math.nan), (0, 1, d - 1, math.inf), (1, 0, d // 2, -math.inf), (1, 0, 9, math.inf), (0, 0, 9, -math.inf), (2, 3, 0, math.nan)])
    check_strays(c, dtype, call(c, dtype))


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("q_len", [3, 12, 40, 70])
def test_queries_before_the_first_key_get_zeros(q_len, quantised):
    """One key, all of whose values are NaN: the last query is NaN, the others, which see no key at all, are zeros."""
    c, dtype = build((2, q_len, 4, 1, 128, 0, [1, 1], 1, 16, "bf16", quantised), seed=q_len)
    for b in range(2):
        c["v_pages"].view(torch.uint8)[int(c["suffix_pages"][b, 0]), :, 0] = 0x7f if quantised else 0xff
    out, lse = call(c, dtype)
    out, lse = out.view(2, q_len, 4, 128), lse.view(2, q_len, 4)
    assert (out[:, :-1] == 0).all() and torch.isneginf(lse[:, :-1]).all()
    assert out[:, -1].isnan().all() and torch.isfinite(lse[:, -1]).all()


def test_the_workspace_is_not_left_spoiled():
    """A call with strays and one without, through one workspace."""
    case = (3, 40, 4, 1, 128, 700, [100, 2, 300], 20, 16, "bf16", False)
    c, dtype = build(case, seed=2)
    fine = call(c, dtype)
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    bad, _ = build(case, seed=2)
    spoil(bad, dtype, [(0, 0, 3, math.nan)])
    check_strays(bad, dtype, call(bad, dtype, workspace=room))
    again = call(c, dtype, workspace=room)
    assert torch.equal(again[0], fine[0]) and torch.equal(again[1], fine[1])
