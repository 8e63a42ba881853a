"""Penalties, biases and masks on logits on the device (needs an MI355X).

Every step is rounded to fp32 by the definition, so that the same steps in fp32 on the CPU give the same bits.  Against 64 bits: a quotient
or product, a product f * made, two differences and a sum, half a step (2^-24) each of numbers no larger than the sum of magnitudes that a
value goes through, and as many again as a token has biases (up to 8 here); then half a step of the type, and of fp16 the half of its
smallest number (2^-25)."""
import math

import pytest
import torch

import drafting_ref as D
import serving_ref as R
from paper_2601_12698_amd import drafting

pytestmark = pytest.mark.gpu


def build(batch, nodes, vocab, dtype, width=0, biases=0, masked=False, tree=False, prompts=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    rows = batch * nodes
    c = {"logits": (torch.randn((rows, vocab), generator=g) * 4).to(R.TYPES[dtype])}
    if width:
        c["history"] = torch.randint(-2, vocab + 2, (batch, width), generator=g, dtype=torch.int32)
        c["history"][:, ::3] = c["history"][:, :1].clone()             # one token that comes often
        c["history_lens"] = torch.randint(0, width + 1, (batch,), generator=g, dtype=torch.int32)
        c["history_lens"][0] = width
        if prompts:
            c["prompt_lens"] = torch.randint(0, width // 2 + 1, (batch,), generator=g, dtype=torch.int32)
    if width or tree:
        c["penalties"] = torch.rand((batch, 3), generator=g) + torch.tensor([0.8, -0.5, -0.5])
    if biases:
        c["bias_tokens"] = torch.randint(-1, vocab + 1, (batch, biases), generator=g, dtype=torch.int32)
        c["bias_values"] = torch.randn((batch, biases), generator=g) * 3
        c["bias_tokens"][:, -1] = c["bias_tokens"][:, 0]       # a token named twice
        c["bias_values"][:, biases // 2] = -math.inf
    if masked:
        c["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (rows, -(-vocab // 32) + 1), generator=g).to(torch.int32)
        c["allowed"][rows // 2] = 0
    if tree:
        c["tree_tokens"] = torch.randint(-1, vocab + 1, (batch, nodes), generator=g, dtype=torch.int32)
        c["tree_tokens"][:, nodes // 2] = c["tree_tokens"][:, 0]
        if width:
            c["tree_tokens"][:, -1] = c["history"][:, 0]
        c["tree_masks"] = D.int64_masks(D.tree_masks(D.rng(seed), batch, nodes, odd=True))
    return c


def call(c, dtype, nodes, write=True, best=True, **more):
    dev = {n: x.cuda() for n, x in c.items()}
    x = dev.pop("logits")
    out = torch.full(x.shape, math.nan, dtype=x.dtype, device="cuda") if write else None
    top = torch.full((x.shape[0],), -7, dtype=torch.int32, device="cuda") if best else None
    drafting.logits_run(x, out, top, dtype, nodes=nodes, **dev, **more)
    torch.cuda.synchronize()
    assert torch.equal(x.cpu().view(torch.uint8), c["logits"].view(torch.uint8))
    return None if out is None else out.cpu(), None if top is None else top.cpu()


def check(c, dtype, nodes, got):
    z, _ = D.logits(c, nodes, wide=False)
    if got[1] is not None:
        assert torch.equal(got[1], D.best(z))
    if got[0] is None:
        return
    want = z.to(R.TYPES[dtype])
    assert torch.equal(got[0].isnan(), want.isnan())
    assert torch.equal(got[0].nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
    exact, size = D.logits(c, nodes, wide=True)
    fine = torch.isfinite(exact) & torch.isfinite(want)
    limit = 14 * 2.0 ** -24 * size + R.HALF_STEP[dtype] * exact.abs() * (1 + 2.0 ** -10) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    assert ((got[0].double() - exact).abs()[fine] <= limit[fine]).all()


CASES = [dict(batch=1, nodes=1, vocab=1, dtype="bf16", width=3), dict(batch=1, nodes=1, vocab=32000, dtype="bf16", width=500, biases=10),
         dict(batch=3, nodes=1, vocab=8192, dtype="fp16", width=40, masked=True), dict(batch=3, nodes=1, vocab=8193, dtype="fp32", width=40, masked=True, prompts=False),
         dict(batch=2, nodes=5, vocab=10007, dtype="bf16", width=2000, biases=300, masked=True, tree=True),
         dict(batch=2, nodes=64, vocab=997, dtype="fp16", width=33, biases=1, tree=True), dict(batch=1, nodes=7, vocab=50001, dtype="fp32", tree=True),
         dict(batch=4, nodes=3, vocab=20000, dtype="fp32", width=100, biases=1023), dict(batch=5, nodes=1, vocab=31, dtype="bf16", masked=True),
         dict(batch=2, nodes=2, vocab=16385, dtype="bf16"), dict(batch=40, nodes=1, vocab=12345, dtype="fp16", biases=2, masked=True),
         dict(batch=1, nodes=1, vocab=152001, dtype="bf16", width=30000), dict(batch=3, nodes=24, vocab=40000, dtype="bf16", width=70, masked=True, tree=True)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "_".join(str(x) for x in c.values()))
def test_against_the_steps_in_fp32_and_64_bits(case):
    c = build(**case, seed=case["vocab"])
    nodes, dtype = case["nodes"], case["dtype"]
    got = call(c, dtype, nodes)
    check(c, dtype, nodes, got)
    alone = call(c, dtype, nodes, write=False)
    assert torch.equal(alone[1], got[1])
    alone = call(c, dtype, nodes, best=False)
    assert torch.equal(alone[0].view(torch.uint8), got[0].view(torch.uint8))


@pytest.mark.parametrize("case", [dict(batch=90, nodes=3, vocab=2901, dtype="bf16", width=40, biases=300, masked=True, tree=True),
                                  dict(batch=260, nodes=1, vocab=500, dtype="fp32", width=9, biases=5), dict(batch=44, nodes=6, vocab=9000, dtype="fp16", width=70, masked=True),
                                  dict(batch=2, nodes=5, vocab=8192, dtype="bf16", width=9000, biases=1, tree=True), dict(batch=1, nodes=1, vocab=16384, dtype="fp32", width=100),
                                  dict(batch=100, nodes=3, vocab=4097, dtype="bf16", masked=True)], ids=lambda c: "_".join(str(x) for x in c.values()))
def test_rows_of_one_workgroup_of_each_size(case):
    c = build(**case, seed=case["vocab"])
    check(c, case["dtype"], case["nodes"], call(c, case["dtype"], case["nodes"]))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_strides_unaligned_rows_and_in_place(dtype):
    c = build(3, 2, 9001, dtype, width=50, biases=4, masked=True, tree=True, seed=1)
    dev = {n: x.cuda() for n, x in c.items()}
    x = dev.pop("logits")
    want, top = call(c, dtype, 2)
    wide = torch.full((6, 9100), 77.0, dtype=x.dtype, device="cuda")
    for first in (0, 1, 8, 99):
        wide.fill_(77.0)
        at = wide[:, first:first + 9001].copy_(x)
        lists = dict(dev, history=torch.cat((dev["history"], dev["history"]), 1)[:, :50], allowed=torch.cat((dev["allowed"], dev["allowed"]), 1)[:, :283])
        best = torch.empty(6, dtype=torch.int32, device="cuda")
        drafting.logits_run(at, at, best, dtype, nodes=2, **lists)
        assert torch.equal(at.cpu().view(torch.uint8) if at.is_contiguous() else at.cpu().contiguous().view(torch.uint8), want.view(torch.uint8))
        assert torch.equal(best.cpu(), top)
        assert (wide[:, :first] == 77).all() and (wide[:, first + 9001:] == 77).all()


@pytest.mark.parametrize("vocab", [100, 8200, 70000])
def test_best_of_ties_nan_infinities_and_rows_without_a_token(vocab):
    x = torch.zeros((8, vocab))
    x[1, vocab - 1] = math.nan
    x[1, vocab // 2] = math.nan
    x[1, 3] = math.inf
    x[2] = -math.inf
    x[3, 5:] = math.inf
    x[4] = -1.0
    x[4, vocab // 3] = x[4, vocab - 2] = -0.5
    x[5, ::2] = -0.0
    x[6, 0], x[6, vocab - 1] = -math.inf, 1e-38
    allowed = torch.full((8, -(-vocab // 32)), -1, dtype=torch.int32)
    allowed[7] = 0
    for dtype in ("bf16", "fp16", "fp32"):
        c = {"logits": x.to(R.TYPES[dtype]), "allowed": allowed}
        got = call(c, dtype, 1)
        check(c, dtype, 1, got)
        assert int(got[1][7]) == 0 and int(got[1][2]) == 0 and int(got[1][1]) == vocab // 2
        lists = dict(c, penalties=torch.tensor([[1.5, 0.0, 0.0]] * 8), history=torch.arange(8, dtype=torch.int32)[:, None], history_lens=torch.ones(8, dtype=torch.int32))
        check(lists, dtype, 1, call(lists, dtype, 1))


@pytest.mark.parametrize("vocab", [31, 8200, 70000])
def test_best_where_all_that_is_allowed_is_minus_infinity(vocab):
    """What is ruled out is -infinity as well: the lowest token, not the lowest that is allowed."""
    x = torch.full((4, vocab), 2.0)
    x[0, 5] = x[0, vocab - 1] = x[1, vocab - 2] = -math.inf
    x[2, 7:] = -math.inf
    x[3, 11] = -1e30
    allowed = torch.zeros((4, -(-vocab // 32)), dtype=torch.int32)
    for row, t in ((0, 5), (0, vocab - 1), (1, vocab - 2), (2, 7), (2, 9), (2, 13), (3, 11)):
        allowed[row, t // 32] |= -2 ** 31 if t % 32 == 31 else 1 << t % 32
    for dtype in ("bf16", "fp32"):
        c = {"logits": x.to(R.TYPES[dtype]), "allowed": allowed}
        got = call(c, dtype, 1)
        check(c, dtype, 1, got)
        assert got[1].tolist() == [0, 0, 0, 11]
        lists = dict(c, penalties=torch.tensor([[1.5, 0.5, 0.5]] * 4), history=torch.tensor([[5], [3], [9], [0]], dtype=torch.int32), history_lens=torch.ones(4, dtype=torch.int32))
        got = call(lists, dtype, 1)
        check(lists, dtype, 1, got)
        assert got[1].tolist() == [0, 0, 0, 11]


def test_lengths_beyond_the_lists_and_tokens_that_are_none():
    c = build(4, 1, 300, "fp32", width=20, seed=2)
    c["history_lens"] = torch.tensor([2 ** 31 - 1, -5, 20, 3], dtype=torch.int32)
    c["prompt_lens"] = torch.tensor([5, 2 ** 31 - 1, -1, 10], dtype=torch.int32)
    c["history"][2, :4] = torch.tensor([-2 ** 31, 2 ** 31 - 1, 300, -1], dtype=torch.int32)
    check(c, "fp32", 1, call(c, "fp32", 1))


@pytest.mark.parametrize("vocab", [500, 40001])
def test_lists_that_say_nothing_and_rows_that_share_theirs(vocab):
    """Histories without penalties; penalties without histories; one history and one mask for all rows, by a stride of 0."""
    c = build(4, 1, vocab, "bf16", width=60, biases=5, masked=True, seed=6)
    for leave in (("penalties",), ("history", "history_lens", "prompt_lens"), ("bias_tokens", "bias_values"), ("allowed", "penalties")):
        some = {n: x for n, x in c.items() if n not in leave}
        check(some, "bf16", 1, call(some, "bf16", 1))
    dev = {n: x.cuda() for n, x in c.items()}
    x = dev.pop("logits")
    dev["history"], dev["allowed"] = dev["history"][:1].expand(4, -1), dev["allowed"][:1].expand(4, -1)
    out, best = torch.empty_like(x), torch.empty(4, dtype=torch.int32, device="cuda")
    drafting.logits_run(x, out, best, "bf16", **dev)
    check(dict(c, history=c["history"][:1].expand(4, -1), allowed=c["allowed"][:1].expand(4, -1)), "bf16", 1, (out.cpu(), best.cpu()))


def test_a_token_that_fills_its_history():
    """Counts of hundreds of thousands: as many as a history may hold."""
    n = drafting.MAX_HISTORY
    c = {"logits": torch.zeros(1, 50), "history": torch.full((1, n), 7, dtype=torch.int32), "history_lens": torch.tensor([n], dtype=torch.int32),
         "penalties": torch.tensor([[1.0, 0.5, 0.25]]), "bias_tokens": torch.tensor([[7]], dtype=torch.int32), "bias_values": torch.tensor([[2.0]])}
    out, best = call(c, "fp32", 1)
    assert float(out[0, 7]) == -0.5 * n - 0.25 + 2.0 and int(best[0]) == 0 and float(out.abs().sum()) == abs(float(out[0, 7]))


def test_rows_beyond_32_bits():
    """Logits of more than 2^32 bytes: the last rows lie past them."""
    rows, vocab = 70000, 32768
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    x[-1, 77], x[-2, vocab - 1], x[0, 5] = 3.0, 2.0, 1.0
    best = torch.empty(rows, dtype=torch.int32, device="cuda")
    bias = torch.tensor([[9]] * rows, dtype=torch.int32, device="cuda"), torch.full((rows, 1), -1.0, device="cuda")
    drafting.logits_run(x, x, best, "bf16", bias_tokens=bias[0], bias_values=bias[1])
    assert best[-1] == 77 and best[-2] == vocab - 1 and best[0] == 5 and int(best[1:-2].abs().sum()) == 0
    assert bool((x[:, 9] == -1).all()) and float(x[:, 10:].float().sum()) == 5.0


def test_the_workspace_is_as_long_as_it_says():
    c = build(3, 2, 100003, "bf16", biases=3, seed=4)
    n = drafting.logits_workspace_bytes(3, 2, 100003, "bf16")
    with pytest.raises(drafting.AddrmsError, match="workspace has"):
        call(c, "bf16", 2, workspace=torch.empty(n - 8, dtype=torch.uint8, device="cuda"))
    room = torch.full((n + 64,), 0xff, dtype=torch.uint8, device="cuda")
    check(c, "bf16", 2, call(c, "bf16", 2, workspace=room[:n]))
    assert (room[n:] == 0xff).all()


@pytest.mark.parametrize("width", [0, 70, 8191, 8192])
@pytest.mark.parametrize("vocab", [32769, 40000, 100003])
def test_the_workspace_is_long_enough_for_either_form_of_long_rows(vocab, width):
    """Histories from 8192 tokens on are gone over by workgroups of 512 threads, shorter ones by 256: other numbers of partial results."""
    c = build(2, 1, vocab, "bf16", width=width, biases=3, seed=vocab + width)
    n = drafting.logits_workspace_bytes(2, 1, vocab, "bf16")
    room = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    check(c, "bf16", 1, call(c, "bf16", 1, workspace=room[:n]))
    assert (room[n:] == 0xa5).all()


def test_on_another_stream_and_in_a_graph():
    c = build(3, 4, 20011, "bf16", width=100, biases=20, masked=True, tree=True, seed=5)
    dev = {n: x.cuda() for n, x in c.items()}
    x = dev.pop("logits")
    room = torch.empty(drafting.logits_workspace_bytes(3, 4, 20011, "bf16"), dtype=torch.uint8, device="cuda")
    out, best = torch.zeros_like(x), torch.zeros(12, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    drafting.logits_run(x, out, best, "bf16", nodes=4, **dev, workspace=room, stream=stream)
    stream.synchronize()
    check(c, "bf16", 4, (out.cpu(), best.cpu()))
    with pytest.raises(ValueError, match="workspace"):
        drafting.logits_run(x, out, best, "bf16", nodes=4, **dev, stream=stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        drafting.logits_run(x, out, best, "bf16", nodes=4, **dev, workspace=room)
    for i in range(4):
        dev["history_lens"].fill_(7 * i)
        dev["tree_tokens"].add_(3)
        x.copy_(torch.randn(x.shape, device="cuda") * 4)
        want, top = torch.empty_like(out), torch.empty_like(best)
        drafting.logits_run(x, want, top, "bf16", nodes=4, **dev, workspace=room)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(best, top)
