"""The operators of a step that checks drafted tokens together, as examples/tree_decode.py runs them, and their native calls against the
general ones (needs an MI355X)."""
import importlib.util
import os
import sys

import pytest
import torch

import drafting_ref as R
from paper_2601_12698_amd import binding as B
from paper_2601_12698_amd import drafting as D
from paper_2601_12698_amd import serving as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("tree_decode", os.path.join(ROOT, "examples", "tree_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_tree():
    e = example()
    masks, depths = e.tree()
    assert max(depths) + 1 == e.DEPTH and len(masks) == len(e.PARENTS) == len(e.GUESS)
    for i, p in enumerate(e.PARENTS):
        assert masks[i] == (0 if p < 0 else masks[p]) | 1 << i and p < i
    assert len({(p, g) for p, g in zip(e.PARENTS, e.GUESS)}) == len(masks)           # no two children have one guess


@pytest.mark.parametrize("args", [["--steps", "0"], ["--steps", "-3", "--check"], ["--batch", "0"], ["--prompt", "0"]])
def test_nothing_to_do_is_refused(args, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["tree_decode.py", *args])
    with pytest.raises(SystemExit) as e:
        example().main()
    assert e.value.code == 2 and "at least 1" in capsys.readouterr().err


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["e4m3", "same"])
@pytest.mark.parametrize("batch,prompt,steps", [(1, 40, 1), (2, 70, 2), (5, 700, 12), (40, 1500, 4)])
def test_a_step_against_plain_torch(batch, prompt, steps, cache):
    """Attention: one rounding of weights and one of the output, half a step each: together at most 2^-8 relative to a row's norm where values
    do not cancel; averages over many keys cancel to about a quarter of the values' size, hence 2^-6.  The rest is whole numbers and bytes:
    the best tokens of the step's own logits, the path they give, the tokens that are certain, and where their keys are."""
    e = example()
    layer, _, error, (q, k, v, logits), before = e.run(batch, prompt, steps, cache, check=True)
    assert error <= 2.0 ** -6
    if steps == 1:
        before = torch.zeros_like(before)
    count, path = layer.count.cpu(), layer.path.cpu()
    lens = layer.history_lens.cpu()
    case = {"logits": logits.cpu(), "history": layer.history.cpu(), "history_lens": lens - count, "prompt_lens": layer.prompt_lens.cpu(),
            "penalties": layer.penalties.cpu(), "tree_tokens": layer.tokens.cpu(), "tree_masks": layer.masks.cpu()}
    z, _ = R.logits(case, layer.nodes, wide=False)
    assert torch.equal(layer.best.cpu().view(-1), R.best(z))
    want = R.accept(layer.best.cpu(), layer.tokens.cpu(), layer.masks.cpu(), layer.suffix_pages.cpu(), before.cpu(), e.PAGE, layer.pages, e.DEPTH)
    for x, y in zip((path, count, layer.last.cpu(), layer.from_slots.cpu(), layer.to_slots.cpu()), want):
        assert torch.equal(x, y)
    assert torch.equal(layer.suffix_lens.cpu(), before.cpu() + count) and int(layer.suffix_lens.min()) >= steps
    # what the cache holds at the path's positions is what is written for its nodes
    for b in range(batch):
        for i in range(int(count[b])):
            node, at = int(path[b, i]), int(before[b]) + i
            assert int(layer.history[b, int(lens[b] - count[b]) + i]) == int(layer.tokens[b, node])
            row = b * layer.nodes + node
            fresh = [None if x is None else torch.zeros_like(x[:1]) for x in layer.cache]
            S.kvcache_write(k[row:row + 1], v[row:row + 1], torch.zeros(1, dtype=torch.int64, device="cuda"), *fresh, "bf16")
            page = int(layer.suffix_pages[b, at // e.PAGE])
            for x, y in zip(layer.cache, fresh):
                if x is not None:
                    assert torch.equal(x[page, :, at % e.PAGE].view(torch.uint8), y[0, :, 0].view(torch.uint8))
    eager = e.run(batch, prompt, steps, cache, graph=False)[0]       # the same without the graph
    assert torch.equal(eager.history, layer.history) and torch.equal(eager.suffix_lens, layer.suffix_lens) and torch.equal(eager.out, layer.out)


@pytest.mark.gpu
def test_native_and_general_calls_agree(monkeypatch):
    torch.manual_seed(0)
    dev = "cuda"
    q = torch.randn(6, 12, 64, device=dev).to(torch.bfloat16)[:, 2:10]
    base = [torch.randint(0, 120, (9, 2, 16, 64), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2)] + \
           [torch.randint(120, 130, (9, 2, 16), dtype=torch.uint8, device=dev) for _ in range(2)]
    prefix, own = torch.tensor([2, 0], dtype=torch.int32, device=dev), torch.tensor([[1, 4], [5, 7]], dtype=torch.int32, device=dev)
    lens, masks = torch.tensor([20, 3], dtype=torch.int32, device=dev), torch.tensor([[1, 3, 5], [1, 3, 7]], device=dev)
    logits = torch.randn(6, 40001, device=dev).to(torch.bfloat16)
    history = torch.randint(0, 40001, (2, 50), dtype=torch.int32, device=dev)
    tokens = torch.randint(0, 40001, (2, 3), dtype=torch.int32, device=dev)

    class Sub(torch.Tensor):
        pass

    def all_calls(wrap):
        cache = [x.clone() for x in base]
        out, lse = torch.empty(6, 8, 64, dtype=torch.bfloat16, device=dev), torch.empty(6, 8, device=dev)
        room = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
        D.treeattn_run(wrap(q), *cache, prefix, 20, own, lens, masks, out, lse, 0.125, "bf16", workspace=room)
        z, best = torch.empty_like(logits), torch.empty(6, dtype=torch.int32, device=dev)
        D.logits_run(wrap(logits), z, best, "bf16", nodes=3, history=history, history_lens=lens, prompt_lens=lens // 2, penalties=torch.tensor([[1.2, 0.1, 0.3]] * 2, device=dev),
                     bias_tokens=tokens, bias_values=torch.ones(2, 3, device=dev), allowed=torch.full((6, 1251), 0x7fff7ff7, dtype=torch.int32, device=dev),
                     tree_tokens=tokens, tree_masks=masks, workspace=room)
        chosen = tokens[:, [1, 2, 0]].contiguous()
        path, count, following = torch.empty(2, 4, dtype=torch.int32, device=dev), torch.empty(2, dtype=torch.int32, device=dev), torch.empty(2, dtype=torch.int32, device=dev)
        f, t = torch.empty(2, 4, dtype=torch.int64, device=dev), torch.empty(2, 4, dtype=torch.int64, device=dev)
        D.treeaccept_run(chosen, tokens, wrap(masks), own, lens, 16, 9, path, count, following, f, t)
        D.kvmove_run(wrap(cache[0]), *cache[1:], torch.tensor([[17, 3], [4, 100]], device=dev), torch.tensor([[3, 17], [90, 4]], device=dev), "bf16")
        torch.cuda.synchronize()
        return [x.contiguous().view(torch.uint8) for x in (out, lse, z, best, path, count, following, f, t, *cache)]

    want = all_calls(lambda t: t)
    for got, ref in zip(all_calls(lambda t: t.as_subclass(Sub)), want):                     # a subclass goes the general way
        assert torch.equal(got, ref)
    monkeypatch.setattr(B, "_native", None)
    for got, ref in zip(all_calls(lambda t: t), want):
        assert torch.equal(got, ref)
    monkeypatch.undo()
    # refused the general way, with words, whatever the native call was given
    out = torch.empty(6, 8, 64, dtype=torch.bfloat16, device=dev)
    with pytest.raises(ValueError, match="has shape"):
        D.treeattn_run(q, *base, prefix, 20, own, lens, masks[:1].contiguous(), out, None, 0.125, "bf16")
    with pytest.raises(ValueError, match="do not hold"):
        D.treeattn_run(q, *base, prefix, 33, own, lens, masks, out, None, 0.125, "bf16")
    with pytest.raises(ValueError, match="do not hold"):
        D.logits_run(logits, None, torch.empty(6, dtype=torch.int32, device=dev), "bf16", allowed=torch.zeros(6, 1250, dtype=torch.int32, device=dev))
    with pytest.raises(ValueError, match="together"):
        D.logits_run(logits, logits, None, "bf16", nodes=3, tree_tokens=tokens)
    with pytest.raises(ValueError, match="contiguous"):
        D.kvmove_run(*base, torch.zeros(2, 2, dtype=torch.int64, device=dev).T, torch.zeros(2, 2, dtype=torch.int64, device=dev), "bf16")
    with pytest.raises(D.AddrmsError, match="nodes is beyond"):
        many = torch.zeros(1, 65, dtype=torch.int64, device=dev)
        D.treeattn_run(torch.zeros(65, 8, 64, dtype=torch.bfloat16, device=dev), *base, None, 0, own[:1], lens[:1], many, torch.empty(65, 8, 64, dtype=torch.bfloat16, device=dev), None,
                       0.125, "bf16")
    D.treeattn_run(q, *base, prefix, 20, own, lens, masks, out, None, 0.125, "bf16")           # no workspace: torch's allocator
    assert torch.equal(out.view(torch.uint8), want[0])
    D.logits_run(logits[:0], None, torch.empty(0, dtype=torch.int32, device=dev), "bf16")


@pytest.mark.gpu
def test_two_graphs_with_one_workspace():
    """Two captured calls that take turns on one stream may share a workspace."""
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(3)
    cache = [torch.randn(80, 2, 16, 64, generator=g, device=dev).to(torch.bfloat16) for _ in range(2)] + [None, None]
    own = torch.randperm(80, generator=g, device=dev).to(torch.int32).view(2, 40)
    lens, masks = torch.tensor([600, 90], dtype=torch.int32, device=dev), torch.tensor([[1, 3, 5, 9]] * 2, device=dev)
    room = torch.empty(8 << 20, dtype=torch.uint8, device=dev)
    calls, graphs = [], []
    for i in range(2):
        q, out = torch.randn(8, 32, 64, generator=g, device=dev).to(torch.bfloat16), torch.empty(8, 32, 64, dtype=torch.bfloat16, device=dev)
        x, best = torch.randn(8, 60000, generator=g, device=dev), torch.empty(8, dtype=torch.int32, device=dev)

        def one(q=q, out=out, x=x, best=best):
            D.treeattn_run(q, *cache, None, 0, own, lens, masks, out, None, 0.125, "bf16", workspace=room)
            D.logits_run(x, None, best, "fp32", workspace=room)
        one()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one()
        calls.append((one, out, best))
        graphs.append(graph)
    for n in (5, 600, 0):
        lens.fill_(n)
        want = []
        for one, out, best in calls:
            one()
            want.append((out.clone(), best.clone()))
        for _ in range(2):
            for (_, out, best), graph in zip(calls, graphs):
                out.zero_()
                best.zero_()
                graph.replay()
        torch.cuda.synchronize()
        for (_, out, best), (o, b) in zip(calls, want):
            assert torch.equal(out, o) and torch.equal(best, b)
