"""What the operators that check drafted tokens refuse, and what is decided without a GPU: every entry point checks its arguments before
anything is launched, so wrong ones can be passed here (the pointers are numbers that nothing reads)."""
import ctypes
import os
import re
from ctypes import byref, c_int64

import pytest
import torch

from paper_2601_12698_amd import binding as B
from paper_2601_12698_amd import build
from paper_2601_12698_amd import drafting as D
from paper_2601_12698_amd import serving as S
from test_host_sanitizers import BUILD

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                                   # an address that is aligned to everything
ST = (c_int64 * 2)(64 * 8, 64)
ARG, SHAPE, TYPE, ALIGN = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED_SHAPE, B.ERR_UNSUPPORTED_DTYPE, B.ERR_MISALIGNED


def test_headers_library_and_binding_name_the_same_entry_points():
    names = set()
    for header in ("treeattn.h", "treeaccept.h", "logits.h", "kvmove.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names |= set(re.findall(r"\b((?:treeattn|treeaccept|logits|kvmove)_[a-z_0-9]+)\s*\(", text))
    assert names == set(D.SIGNATURES) and len(names) == 9
    lib = ctypes.CDLL(B.LIB_PATH)
    for n in names:
        assert hasattr(lib, n) and callable(getattr(D, n))
    assert ctypes.sizeof(D.LogitsLists) == 9 * 8 + 2 * 8 + 2 * 4


def shape(**more):
    s = dict(batch=4, q_len=12, q_heads=8, kv_heads=2, d=128, page_size=16, pages=100, prefix_len=3000, suffix_width=40, dtype="bf16", quantised=True)
    s.update(more)
    return S.prefixattn_shape(**s)


def attend(s=None, q=P, qs=ST, kp=P, vp=P, kc=P, vc=P, pre=P, suf=P, lens=P, masks=P, out=P, lse=P, scale=0.1, room=P, bytes_=1 << 40):
    return D.load().treeattn_run(q, qs, kp, vp, kc, vc, pre, suf, lens, masks, out, lse, scale, None if s is None else byref(s), room, bytes_, None)


@pytest.mark.parametrize("what,status", [
    (dict(batch=-1), ARG), (dict(q_len=-1), ARG), (dict(q_heads=9), ARG), (dict(kv_heads=0), ARG), (dict(page_size=48), ARG), (dict(prefix_len=-1), ARG),
    (dict(suffix_width=-1), ARG), (dict(d=72), SHAPE), (dict(d=512), SHAPE), (dict(pages=1 << 31), SHAPE), (dict(prefix_len=1 << 30), SHAPE),
    (dict(suffix_width=1 << 26), SHAPE), (dict(suffix_width=1 << 62), SHAPE), (dict(batch=1 << 22), SHAPE), (dict(q_heads=65544, kv_heads=1), SHAPE), (dict(q_len=65), SHAPE),
])
def test_tree_shapes_refused(what, status):
    s = shape(**what)
    assert D.load().treeattn_workspace_bytes(byref(s)) == status
    assert attend(s) == status


@pytest.mark.parametrize("what,status", [
    (dict(q=None), ARG), (dict(qs=None), ARG), (dict(out=None), ARG), (dict(kp=None), ARG), (dict(vc=None), ARG), (dict(pre=None), ARG), (dict(suf=None), ARG),
    (dict(lens=None), ARG), (dict(masks=None), ARG), (dict(room=None), ARG), (dict(bytes_=100), ARG), (dict(bytes_=-1), ARG), (dict(scale=0.0), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(q=P + 1), ALIGN), (dict(out=P + 8), ALIGN), (dict(room=P + 4), ALIGN),
    (dict(lens=P + 2), ALIGN), (dict(lse=P + 2), ALIGN), (dict(kp=P + 8), ALIGN), (dict(masks=P + 4), ALIGN),
])
def test_tree_arguments_refused(what, status):
    assert attend(shape(), **what) == status
    assert B.addrms_last_error()


def test_trees_without_work_and_unknown_shapes():
    assert attend(None) == ARG
    assert attend(shape(batch=0), q=None, out=None, masks=None) == B.OK and attend(shape(q_len=0), q=None) == B.OK
    s = shape()
    s.dtype = 3
    assert attend(s) == TYPE
    s = shape()
    s.format = 7
    assert attend(s) == ARG
    assert D.treeattn_workspace_bytes(shape(prefix_len=0, suffix_width=0)) == 0
    a = shape()
    key, rows = 2 * 2 * 129, 4 * 12 * 8
    assert D.treeattn_algorithmic_bytes(a, 1000) == (3000 + 1000) * key + rows * (2 * 2 * 128 + 4) + 8 * 48
    with pytest.raises(D.AddrmsError):
        D.treeattn_algorithmic_bytes(a, -1)


def test_tree_workspace_holds_a_part_for_each_split():
    """4 d + 8 bytes for each row and part: of the prefix never more parts than pieces of 128 keys, of the sequences together no more than
    such pieces and one for the end of each."""
    for prefix, width in ((0, 4), (256, 0), (257, 40), (100000, 100), (0, 1 << 13)):
        for batch, nodes, heads in ((1, 1, (1, 1)), (64, 64, (64, 8)), (3, 40, (8, 2)), (1, 64, (32, 8))):
            s = shape(batch=batch, q_len=nodes, q_heads=heads[0], kv_heads=heads[1], prefix_len=prefix, suffix_width=width, pages=1 << 20)
            part, n = nodes * heads[0] * (4 * 128 + 8), D.treeattn_workspace_bytes(s)       # of one sequence
            assert n % part == 0
            assert n // part <= batch * -(-prefix // 128) + -(-batch * width * 16 // 128) + (batch if width else 0)


def accept(chosen=P, tokens=P, masks=P, table=P, lens=P, path=P, count=P, follows=P, f=P, t=P, batch=4, nodes=8, depth=5, width=10, pages=100, page=16):
    return D.load().treeaccept_run(chosen, tokens, masks, table, lens, path, count, follows, f, t, batch, nodes, depth, width, pages, page, None)


@pytest.mark.parametrize("what,status", [
    (dict(chosen=None), ARG), (dict(tokens=None), ARG), (dict(masks=None), ARG), (dict(table=None), ARG), (dict(lens=None), ARG), (dict(path=None), ARG),
    (dict(count=None), ARG), (dict(follows=None), ARG), (dict(f=None), ARG), (dict(t=None), ARG), (dict(batch=-1), ARG), (dict(nodes=0), ARG), (dict(nodes=65), SHAPE),
    (dict(depth=0), ARG), (dict(depth=65537), SHAPE), (dict(width=-1), ARG), (dict(width=1 << 26), SHAPE), (dict(pages=-1), ARG), (dict(pages=1 << 31), SHAPE),
    (dict(page=17), ARG), (dict(page=0), ARG), (dict(batch=1 << 24), SHAPE), (dict(masks=P + 4), ALIGN), (dict(f=P + 4), ALIGN), (dict(path=P + 2), ALIGN),
    (dict(chosen=P + 1), ALIGN), (dict(batch=0), B.OK), (dict(batch=0, chosen=None, f=None), B.OK),
])
def test_accept_refusals(what, status):
    assert accept(**what) == status


def move(kp=P, vp=P, kc=P, vc=P, f=P, t=P, groups=4, tokens=6, heads=8, d=64, pages=10, page=16, dtype=0, fmt=1):
    return D.load().kvmove_run(kp, vp, kc, vc, f, t, groups, tokens, heads, d, pages, page, dtype, fmt, None)


@pytest.mark.parametrize("what,status", [
    (dict(dtype=3), TYPE), (dict(dtype=2), TYPE), (dict(fmt=2), ARG), (dict(groups=-1), ARG), (dict(tokens=-1), ARG), (dict(tokens=257), SHAPE), (dict(heads=0), ARG),
    (dict(pages=-1), ARG), (dict(page=24), ARG), (dict(page=0), ARG), (dict(page=131072), ARG), (dict(d=40), SHAPE), (dict(d=272), SHAPE), (dict(pages=1 << 31), SHAPE),
    (dict(groups=1 << 18), SHAPE), (dict(groups=1 << 40), SHAPE), (dict(heads=65537), SHAPE), (dict(kp=None), ARG), (dict(kc=None), ARG), (dict(vc=None), ARG),
    (dict(f=None), ARG), (dict(t=None), ARG), (dict(f=P + 4), ALIGN), (dict(vp=P + 8), ALIGN), (dict(groups=0), B.OK), (dict(tokens=0, f=None), B.OK), (dict(pages=0), B.OK),
])
def test_move_refusals(what, status):
    assert move(**what) == status


def test_move_bytes():
    assert D.kvmove_algorithmic_bytes(3, 5, 10, 8, 128, True) == 4 * 10 * 8 * 129 + 16 * 15
    assert D.kvmove_algorithmic_bytes(3, 5, 10, 8, 128, False) == 4 * 10 * 8 * 256 + 16 * 15
    for moved in (-1, 16):
        with pytest.raises(D.AddrmsError):
            D.kvmove_algorithmic_bytes(3, 5, moved, 8, 128)


LISTS = dict(history=P, history_lens=P, prompt_lens=P, penalties=P, bias_tokens=P, bias_values=P, allowed=P, tree_tokens=P, tree_masks=P, history_stride=100,
             allowed_stride=1000, history_width=100, biases=10)


def logits(x=P, stride=32000, out=2 * P, out_stride=32000, best=P, batch=4, nodes=3, vocab=32000, dtype=0, lists=True, room=P, bytes_=1 << 30, **more):
    a = D.LogitsLists(**dict(LISTS, **more))
    return D.load().logits_run(x, stride, out, out_stride, best, batch, nodes, vocab, dtype, byref(a) if lists else None, room, bytes_, None)


@pytest.mark.parametrize("what,status", [
    (dict(dtype=2), TYPE), (dict(dtype=4), TYPE), (dict(batch=-1), ARG), (dict(nodes=-1), ARG), (dict(vocab=0), ARG), (dict(vocab=(1 << 24) + 1), SHAPE),
    (dict(batch=1 << 24), SHAPE), (dict(nodes=65), SHAPE), (dict(nodes=65537, tree_masks=None, tree_tokens=None), SHAPE), (dict(lists=False), ARG),
    (dict(history_width=-1), SHAPE), (dict(history_width=1 << 20), SHAPE), (dict(biases=1024), SHAPE), (dict(biases=-1), SHAPE), (dict(x=None), ARG),
    (dict(history_lens=None), ARG), (dict(bias_tokens=None), ARG), (dict(bias_values=None), ARG), (dict(tree_tokens=None), ARG), (dict(tree_masks=None), ARG),
    (dict(room=None, vocab=100000, out_stride=100000), ARG), (dict(bytes_=0, vocab=100000, out_stride=100000), ARG), (dict(x=P + 1), ALIGN), (dict(out=P + 1), ALIGN), (dict(best=P + 2), ALIGN), (dict(tree_masks=P + 4), ALIGN),
    (dict(history=P + 2), ALIGN), (dict(allowed=P + 2), ALIGN), (dict(room=P + 4), ALIGN), (dict(out_stride=31999), ARG), (dict(out=P, out_stride=40000), ARG),
    (dict(batch=0), B.OK), (dict(nodes=0), B.OK), (dict(out=None, best=None), B.OK),
])
def test_logits_refusals(what, status):
    assert logits(**what) == status


def test_logits_workspace_and_bytes():
    assert D.logits_workspace_bytes(3, 4, 8192, "bf16") >= 0 and D.logits_workspace_bytes(3, 4, 152000, "fp32") % 96 == 0
    assert D.logits_algorithmic_bytes(2, 3, 1000, "bf16", 50, 7, True, True) == 6 * 1000 * 4 + 6 * 32 * 4 + 200 + 2 * 7 * 8 + 24
    assert D.logits_algorithmic_bytes(2, 3, 1000, "fp32", 0, 0, False, False) == 6 * 1000 * 4 + 24
    with pytest.raises(D.AddrmsError):
        D.logits_workspace_bytes(1, 1, 0, "bf16")


def test_binding_refuses_before_the_library_is_asked():
    x = torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    pages, masks, i32 = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.ones(2, 3, dtype=torch.int64), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be"):
        D.treeattn_run(x[0], pages, pages, None, None, None, 0, None, None, masks, x, None, 0.1, "bf16")
    with pytest.raises(ValueError, match="device tensor"):
        D.treeattn_run(x, pages, pages, None, None, None, 0, None, None, masks, x, None, 0.1, "bf16")
    with pytest.raises(ValueError, match="unknown dtype"):
        D.treeattn_run(x, pages, pages, None, None, None, 0, None, None, masks, x, None, 0.1, "fp32")
    with pytest.raises(ValueError, match="nodes=4"):
        D.logits_run(torch.zeros(6, 10), None, None, "fp32", nodes=4)
    with pytest.raises(ValueError, match="but dtype asks for"):
        D.logits_run(torch.zeros(6, 10), None, None, "bf16")
    with pytest.raises(ValueError, match="device tensor"):
        D.logits_run(torch.zeros(6, 10), None, None, "fp32")
    with pytest.raises(ValueError, match="must be"):
        D.treeaccept_run(i32, i32, masks[0], None, None, 16, 0, i32, i32[0], i32[0], None, None)
    with pytest.raises(ValueError, match="device tensor"):
        D.treeaccept_run(i32, i32, masks, None, None, 16, 0, i32, i32[0], i32[0], None, None)
    with pytest.raises(ValueError, match="device tensor"):
        D.kvmove_run(pages, pages, None, None, masks, masks, "bf16")


def test_native_calls_leave_what_is_not_usual_to_the_general_way():
    B._torch()
    n = D._fast()
    assert n is not None
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32)
    pages, m = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int64)
    assert n.treeattn_run(x, pages, pages, None, None, None, 0, None, None, m, x, None, 0.1, "bf16", x) is None            # host tensors
    assert n.logits_run(x[:, 0], None, None, "bf16", 1, *[None] * 10) is None
    assert n.treeaccept_run(i, i, m, None, None, 16, 0, i, i[0], i[0], None, None) is None
    assert n.kvmove_run(pages, pages, None, None, m, m, "bf16") is None
    for call in (n.treeattn_run, n.logits_run, n.treeaccept_run, n.kvmove_run):
        assert call() is None and call(1, 2, 3) is None
    for count in (7, 12, 15):
        for call in (n.treeattn_run, n.logits_run, n.treeaccept_run, n.kvmove_run):
            assert call(*[None] * count) is None and call(*[7] * count) is None
    with pytest.raises(TypeError):
        n.bind_drafting(B.DTYPE_IDS)


def test_the_kernels_take_no_scratch_memory():
    """Its loads and stores would stand between those of keys and values and wait for them (from the build's own reports)."""
    seen = 0
    for name in ["kvmove", "treeaccept", "logits"] + [f"treeattn_d{dt}_f{f}_h{dp}" for dt in (0, 1) for f in (0, 1) for dp in (64, 128, 256)]:
        path = os.path.join(BUILD, name + ".remarks")
        if not os.path.exists(path):
            pytest.skip("the library is not built here")
        with open(path) as f:
            for kernel, r in build.parse_remarks(f.read()).items():
                seen += 1
                assert r["scratch"] == 0, (kernel, r)
    assert seen > 50


def test_what_is_left_out_is_named():
    """A prefix without pages, pages without lengths: the binding's own words, not those of a None that is asked for its shape."""
    x = torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    pages, masks, i32 = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.ones(2, 3, dtype=torch.int64), torch.zeros(2, 3, dtype=torch.int32)
    for run, more in ((D.treeattn_run, (masks,)), (S.prefixattn_run, ())):
        with pytest.raises(ValueError, match="has prefix_pages"):
            run(x, pages, pages, None, None, None, 5, i32, i32[:, 0], *more, x, None, 0.1, "bf16")
        with pytest.raises(ValueError, match="have suffix_lens"):
            run(x, pages, pages, None, None, None, 0, i32, None, *more, x, None, 0.1, "bf16")
        with pytest.raises(ValueError, match="prefix_len must be"):
            run(x, pages, pages, None, None, None, -1, None, None, *more, x, None, 0.1, "bf16")
    for missing in ((None, i32[:, 0]), (i32, None)):
        with pytest.raises(ValueError, match="have suffix_pages and suffix_lens"):
            D.treeaccept_run(i32, i32, masks, *missing, 16, 3, i32, i32[:, 0], i32[:, 0], masks, masks)


def test_logits_workspace_is_that_of_the_longer_of_two_forms():
    """8 bytes of each wave of a row's workgroups, where one of 1024 threads with 32 tokens each does not hold the row: 256 or 512 threads then, which of
    them goes by the histories, which the workspace is not told."""
    for vocab in (1, 8192, 32768):
        assert D.logits_workspace_bytes(3, 4, vocab, "bf16") == 0
    for vocab in (32769, 40960, 49152, 49153, 152000, 1 << 24):
        partials = max(-(-vocab // (32 * t)) * (t // 64) for t in (256, 512))
        assert D.logits_workspace_bytes(3, 4, vocab, "fp32") == 8 * 12 * partials
    assert D.logits_workspace_bytes(1, 1, 40960, "bf16") == 8 * 24 and D.logits_workspace_bytes(1, 1, 40959, "fp16") == 8 * 24      # 5 of 4 waves, 3 of 8
