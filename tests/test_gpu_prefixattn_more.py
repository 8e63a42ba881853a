"""Attention over a shared prefix where the first tests do not go: queries that are not aligned to 16 bytes, heads between 128 and 256 in
every form, scores of one sign, one token a page (needs an MI355X).  Bars as in test_gpu_prefixattn.py."""
import math

import pytest
import torch

from paper_2601_12698_amd import serving as S
from test_gpu_prefixattn import build, check

pytestmark = pytest.mark.gpu

# batch, q_len, q heads, kv heads, d, prefix, suffix lengths, pages of a suffix, page, type, quantised
UNALIGNED = [
    (2, 1, 8, 2, 128, 37, [5, 16], 1, 16, "bf16", True),        # few rows, a short prefix
    (3, 1, 16, 1, 256, 900, [2, 0, 70], 5, 16, "fp16", False),  # a long one
    (32, 1, 4, 1, 256, 20, [i for i in range(32)], 2, 16, "bf16", False),
    (9, 4, 4, 1, 64, 700, [0, 1, 2, 3, 4, 5, 33, 20, 7], 3, 16, "fp16", False),
    (2, 40, 8, 2, 128, 130, [40, 75], 5, 16, "bf16", True),
    (70, 1, 4, 1, 112, 1100, [i % 40 for i in range(70)], 3, 16, "bf16", False),
    (2, 35, 8, 2, 240, 300, [35, 100], 7, 16, "bf16", False),
]


def run(c, dtype, q):
    out = torch.full(c["q"].shape, math.nan, dtype=c["q"].dtype, device="cuda")
    lse = torch.full(c["q"].shape[:2], math.nan, device="cuda")
    dev = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in c.items() if n != "q"}
    S.prefixattn_run(q, dev["k_pages"], dev["v_pages"], dev["k_scale"], dev["v_scale"], dev["prefix_pages"], c["prefix_len"], dev["suffix_pages"],
                     dev["suffix_lens"], out, lse, c["scale"], dtype, q_len=c["q_len"])
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("how", ["offset", "token stride", "head stride"])
@pytest.mark.parametrize("case", UNALIGNED, ids=lambda c: "x".join(str(x) for x in c[:6]))
def test_queries_that_are_not_aligned(case, how):
    c, dtype = build(case, seed=5)
    rows, heads, d = c["q"].shape
    if how == "offset":
        q = torch.zeros(rows * heads * d + 3, dtype=c["q"].dtype, device="cuda")[3:].view(rows, heads, d)
    elif how == "token stride":
        q = torch.zeros(rows, heads * d + 5, dtype=c["q"].dtype, device="cuda")[:, :heads * d].view(rows, heads, d)
    else:
        q = torch.zeros(rows, heads, d + 6, dtype=c["q"].dtype, device="cuda")[:, :, :d]
    q.copy_(c["q"])
    got = run(c, dtype, q)
    check(c, dtype, got)
    again = run(c, dtype, c["q"].contiguous().cuda())
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("d", [144, 160, 176, 192, 208, 224, 240])
def test_heads_between_128_and_256(d, quantised):
    dtype = "fp16" if d % 32 else "bf16"
    for batch, q_len, hq, hk, prefix, lens, width in (
            (3, 1, 8, 2, 40, [1, 0, 37], 3),                    # one launch, eight waves
            (4, 1, 16, 1, 1500, [100, 2, 0, 77], 7),            # few rows over a long prefix
            (130, 1, 4, 2, 700, [(7 * i) % 41 - 1 for i in range(130)], 3),     # suffixes that join the prefix's parts, four waves
            (64, 1, 8, 4, 700, [(7 * i) % 41 - 1 for i in range(64)], 3),       # and eight
            (20, 1, 8, 2, 900, [i % 11 for i in range(20)], 1),  # 128 rows of a prefix, few of a suffix
            (2, 45, 8, 2, 333, [45, 100], 7)):                  # many of both
        c, _ = build((batch, q_len, hq, hk, d, prefix, lens, width, 16, dtype, quantised), seed=d + batch)
        check(c, dtype, run(c, dtype, c["q"].cuda()))


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("q_len", [1, 12, 40])
def test_a_page_of_one_token_and_a_page_of_many(q_len, quantised):
    for page, width in ((1, 50), (1024 if quantised else 65536, 1)):
        c, dtype = build((2, q_len, 4, 2, 64, 129, [50, 33], width, page, "bf16", quantised), seed=q_len, junk=page == 1)
        check(c, dtype, run(c, dtype, c["q"].cuda()))


@pytest.mark.parametrize("q_len", [1, 12, 40, 80])
def test_scores_far_below_zero(q_len):
    """All of a row's scores are large and negative: weights are relative to the largest of them."""
    c, dtype = build((2, q_len, 4, 1, 128, 70, [q_len, q_len + 30], 8, 16, "bf16", False), seed=3, junk=False)
    c["k_pages"] = (c["k_pages"].float() * 0.05 + 4.0).to(torch.bfloat16)
    c["q"] = (c["q"].float() * 0.05 - 4.0).to(torch.bfloat16)
    got = run(c, dtype, c["q"].cuda())
    assert (got[1] < -100).all()
    check(c, dtype, got)
