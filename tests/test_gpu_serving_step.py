"""The operators of a decode step together, as examples/shared_prefix_decode.py runs them, and their native calls against the general
ones (needs an MI355X)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2601_12698_amd import binding as B
from paper_2601_12698_amd import serving as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("shared_prefix_decode", os.path.join(ROOT, "examples", "shared_prefix_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_prompt_positions():
    pos, following = example().prompt_positions(100, "cpu")
    assert pos.shape == (3, 100) and pos[:, 0].tolist() == [0, 0, 0] and following == int(pos.max()) + 1
    side = 7                                                  # 49 patches in the middle
    assert pos[:, 25].tolist() == [25, 25, 25] and pos[:, 25 + 8].tolist() == [25, 26, 26] and pos[:, 25 + 49].tolist() == [25 + side] * 3


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["e4m3", "same"])
@pytest.mark.parametrize("batch,prompt,steps", [(2, 70, 4), (5, 700, 18), (40, 1500, 6)])
def test_a_step_against_plain_torch(batch, prompt, steps, cache):
    """One rounding of weights and one of the output, half a step each: together at most 2^-8 relative to a row's norm where values
    do not cancel; averages over many keys cancel to about a quarter of the values' size, hence 2^-6."""
    layer, _, error = example().run(batch, prompt, steps, cache, check=True)
    assert int(layer.suffix_lens[0]) == steps and error <= 2.0 ** -6
    eager, _, _ = example().run(batch, prompt, steps, cache, graph=False)       # the same bits without the graph
    assert torch.equal(eager.out, layer.out) and torch.equal(eager.lse, layer.lse)


def test_native_calls_leave_what_is_not_usual_to_the_general_way():
    B._torch()
    n = S._fast()
    assert n is not None
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    pages, t = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    f, a = torch.zeros(32, dtype=torch.float64), torch.zeros(32, dtype=torch.uint8)
    assert n.rotary_run(x, x, x, x, i[None], f, a, "bf16", False, False) is None          # host tensors
    assert n.kvcache_write(x, x, i, pages, pages, None, None, "bf16") is None
    assert n.kvcache_read(pages, pages, None, None, i, x, x, "bf16") is None
    assert n.prefixattn_run(x, pages, pages, None, None, t, 4, None, None, x, None, 0.1, "bf16", 1, x) is None
    for call in (n.rotary_run, n.kvcache_write, n.kvcache_read, n.prefixattn_run):
        assert call() is None and call(1, 2, 3) is None
    assert n.prefixattn_run(x, torch.zeros(3, 2, 0, 64, dtype=torch.bfloat16), pages, None, None, t, 1 << 62, None, None, x, None, 0.1, "bf16", 0, x) is None
    with pytest.raises(TypeError):
        n.bind_serving(B.DTYPE_IDS)


@pytest.mark.gpu
def test_native_and_general_calls_agree(monkeypatch):
    torch.manual_seed(0)
    dev = "cuda"
    x = torch.randn(6, 12, 64, device=dev).to(torch.bfloat16)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    pos, (freq, axis) = torch.randint(0, 999, (2, 6), device=dev), S.rotary_plan(64, 1e4, (10, 22), dev)
    slots, table, own = torch.tensor([3, 40, 17, 0, 33, -1], device=dev), torch.tensor([2, 0], dtype=torch.int32, device=dev), torch.tensor([[1], [1], [0]], dtype=torch.int32, device=dev)
    lens = torch.tensor([2, 0, 16], dtype=torch.int32, device=dev)

    class Sub(torch.Tensor):
        pass

    def all_calls(wrap):
        cache = [torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn, device=dev) for _ in range(2)] + [torch.full((3, 2, 16), 127, dtype=torch.uint8, device=dev) for _ in range(2)]
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        S.rotary_run(wrap(q), k, qo, ko, pos, freq, axis, "bf16")
        S.kvcache_write(wrap(ko), v, slots, *cache, "bf16")
        kb, vb = torch.empty(6, 2, 64, dtype=torch.bfloat16, device=dev), torch.empty(6, 2, 64, dtype=torch.bfloat16, device=dev)
        S.kvcache_read(*cache, wrap(slots), kb, vb, "bf16")
        out, lse = torch.empty_like(qo).contiguous(), torch.empty(6, 8, device=dev)
        room = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
        S.prefixattn_run(wrap(qo), *cache, table, 20, own, lens, out, lse, 0.125, "bf16", q_len=2, workspace=room)
        torch.cuda.synchronize()
        return [t.view(torch.uint8) for t in (qo, ko, *cache, kb, vb, out)] + [lse]

    want = all_calls(lambda t: t)
    for got, ref in zip(all_calls(lambda t: t.as_subclass(Sub)), want):                     # a subclass goes the general way
        assert torch.equal(got, ref)
    monkeypatch.setattr(B, "_native", None)
    for got, ref in zip(all_calls(lambda t: t), want):
        assert torch.equal(got, ref)
    monkeypatch.undo()
    cache = [torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16, device=dev) for _ in range(2)] + [None, None]
    long = [torch.zeros(90, 2, 16, 64, dtype=torch.bfloat16, device=dev) for _ in range(2)] + [None, None]
    with pytest.raises(S.AddrmsError, match="workspace has"):
        S.prefixattn_run(q, *long, torch.zeros(90, dtype=torch.int32, device=dev), 1440, None, None, torch.empty(6, 8, 64, dtype=torch.bfloat16, device=dev),
                         None, 0.125, "bf16", workspace=torch.empty(4, dtype=torch.uint8, device=dev))
    with pytest.raises(ValueError, match="has shape"):
        S.rotary_run(q, k, torch.empty_like(k), torch.empty_like(k), pos, freq, axis, "bf16")
    out = torch.empty(6, 8, 64, dtype=torch.bfloat16, device=dev)
    S.prefixattn_run(q, *cache, table, int(np.int64(20)), own, lens, out, None, 0.125, "bf16", q_len=2)         # no workspace: torch's allocator
    assert torch.isfinite(out.float()).all()
