"""Slots that several tokens of one call name: what include/kvcache.h says of them, and that the call's other places are as they should be
(needs an MI355X)."""
import os

import pytest
import torch

import serving_ref as R
from paper_2601_12698_amd import serving as S
from test_gpu_kvcache import check_written, empty, tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_header_promises_no_whole_token_for_a_slot_named_twice():
    text = " ".join(open(os.path.join(ROOT, "include", "kvcache.h")).read().replace("*", " ").split())
    assert "either token may stay" not in text and "A slot is to be named once" in text


@pytest.mark.gpu
@pytest.mark.parametrize("quantised", [True, False])
@pytest.mark.parametrize("T,h,d,page", [(64, 8, 128, 16), (1200, 2, 256, 16)])
def test_a_slot_named_twice_holds_parts_of_the_two(T, h, d, page, quantised):
    pages = T // page + 2
    x = tokens(T, h, d, "bf16", 12)
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(pages * page, generator=g)[:T]
    pairs = [(1, 2), (3, T // 2), (4, T - 1)]                  # beside each other, and far apart
    for a, b in pairs:
        slots[b] = slots[a]
    cache = empty(pages, h, page, d, "bf16", quantised)
    before = [None if c is None else c.clone() for c in cache]
    S.kvcache_write(x[:, :h].cuda(), x[:, h:].cuda(), slots.cuda(), *cache, "bf16")
    twice = {int(slots[a]) for a, _ in pairs}
    once = torch.tensor([-1 if int(s) in twice else int(s) for s in slots])
    check_written(cache, x[:, :h], x[:, h:], once, "bf16", page)
    untouched = torch.ones(pages * page, dtype=torch.bool)
    untouched[slots] = False
    for new, old in zip(cache, before):
        if new is not None:
            p, q = (c.view(torch.uint8).view(pages, h, page, -1).transpose(1, 2).flatten(0, 1).cpu() for c in (new, old))
            assert torch.equal(p[untouched], q[untouched])
    for y, codes, scales in ((x[:, :h], cache[0].cpu(), cache[2]), (x[:, h:], cache[1].cpu(), cache[3])):
        for a, b in pairs:
            p, o = divmod(int(slots[a]), page)
            n, s = R.quantise(y[[a, b]], "bf16") if quantised else (y[[a, b]].double(), None)
            got = codes[p, :, o].double()
            assert ((got == n[0]) | (got == n[1])).all()
            if quantised:
                assert ((scales[p, :, o].cpu() == s[0]) | (scales[p, :, o].cpu() == s[1])).all()
