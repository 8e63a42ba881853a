#!/usr/bin/env python3
"""One attention layer that answers a shared prompt with several sequences at once, token by token (needs an MI355X).

    python examples/shared_prefix_decode.py [--batch 8] [--prompt 1000] [--steps 16] [--cache e4m3|same] [--check]

A prompt of text and of one image (its tokens have positions in time, height and width) goes through the layer once, and its
keys and values into the pages of a cache.  Then every sequence of the batch takes its own steps: add + norm, projection to
queries, keys and values, rotary positions, the new token into its own page, attention over the prompt (read once for all) and
over the sequence's own tokens, output projection.  Weights are random; products with them are torch's.  A step is captured
into a HIP graph after the first one and replayed.  ``--check`` compares the last step with the same layer in plain torch.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2601_12698_amd import binding as B          # noqa: E402
from paper_2601_12698_amd import serving as S          # noqa: E402

HEADS, KV_HEADS, D, HIDDEN, PAGE, EPS = 32, 8, 128, 2048, 16, 1e-6
SECTIONS = (16, 24, 24)                                 # pairs of time, height and width


def prompt_positions(n: int, device):
    """[3, n]: text, then an image of up to 16 x 16 patches in the middle, then text that goes on behind its largest position."""
    side = min(16, int((n // 2) ** 0.5))
    before = (n - side * side) // 2
    pos = torch.arange(n, device=device).repeat(3, 1)
    patch = torch.arange(side * side, device=device)
    pos[0, before:before + side * side] = before
    pos[1, before:before + side * side] = before + patch // side
    pos[2, before:before + side * side] = before + patch % side
    pos[:, before + side * side:] = before + side + torch.arange(n - before - side * side, device=device)
    return pos, int(pos.max()) + 1


class Layer:
    def __init__(self, batch: int, prompt: int, steps: int, cache: str, device="cuda", seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *shape, std: (torch.randn(shape, generator=g, device=device) * std).to(torch.bfloat16)  # noqa: E731
        self.batch, self.prompt, self.device = batch, prompt, device
        self.norm = torch.ones(HIDDEN, dtype=torch.bfloat16, device=device)
        self.qkv = rand(HIDDEN, (HEADS + 2 * KV_HEADS) * D, std=HIDDEN ** -0.5)
        self.proj = rand(HEADS * D, HIDDEN, std=(HEADS * D) ** -0.5)
        self.prompt_states, self.start = rand(prompt, HIDDEN, std=1.0), rand(batch, HIDDEN, std=1.0)
        self.inv_freq, self.pair_axis = S.rotary_plan(D, 10000.0, SECTIONS, device)
        first, own = -(-prompt // PAGE), -(-steps // PAGE)
        pages = first + batch * own
        if cache == "e4m3":
            self.cache = [torch.zeros((pages, KV_HEADS, PAGE, D), dtype=torch.float8_e4m3fn, device=device) for _ in range(2)] + \
                         [torch.full((pages, KV_HEADS, PAGE), 127, dtype=torch.uint8, device=device) for _ in range(2)]
        else:
            self.cache = [torch.zeros((pages, KV_HEADS, PAGE, D), dtype=torch.bfloat16, device=device) for _ in range(2)] + [None, None]
        table = torch.randperm(pages, generator=g, device=device).to(torch.int32)
        self.prefix_pages, self.suffix_pages = table[:first].contiguous(), table[first:].view(batch, own).contiguous()
        self.suffix_lens = torch.zeros(batch, dtype=torch.int32, device=device)
        shape = S.prefixattn_shape(batch, 1, HEADS, KV_HEADS, D, PAGE, pages, prompt, own, "bf16", cache == "e4m3")
        self.workspace = torch.empty(max(16, S.prefixattn_workspace_bytes(shape)), dtype=torch.uint8, device=device)
        # what a step works on: states (in place), the residual stream, positions, slots
        self.x, self.residual = self.start.clone(), torch.zeros_like(self.start)
        self.positions = torch.zeros((3, batch), dtype=torch.int64, device=device)
        self.slots = torch.zeros(batch, dtype=torch.int64, device=device)
        self.out = torch.empty((batch, HEADS, D), dtype=torch.bfloat16, device=device)
        self.lse = torch.empty((batch, HEADS), device=device)
        self.rows = torch.arange(batch, device=device)

    def heads(self, x):
        qkv = (x @ self.qkv).view(x.shape[0], HEADS + 2 * KV_HEADS, D)
        return qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]

    def prefill(self):
        """The prompt's keys and values go into the pages all share."""
        n = self.prompt
        x, residual = self.prompt_states.clone(), torch.zeros_like(self.prompt_states)
        B.addrms_run(x, residual, self.norm, EPS, n, HIDDEN, "bf16")
        q, k, v = self.heads(x)
        pos, following = prompt_positions(n, self.device)
        S.rotary_run(q, k, q, k, pos, self.inv_freq, self.pair_axis, "bf16")
        token = torch.arange(n, device=self.device)
        S.kvcache_write(k, v, self.prefix_pages[token // PAGE].long() * PAGE + token % PAGE, *self.cache, "bf16")
        self.positions.fill_(following)

    def step(self):
        """One token of every sequence.  Nothing here depends on the host: it can be captured."""
        at = self.suffix_lens.long()
        torch.add(self.suffix_pages[self.rows, at // PAGE].long() * PAGE, at % PAGE, out=self.slots)
        self.suffix_lens.add_(1)
        B.addrms_run(self.x, self.residual, self.norm, EPS, self.batch, HIDDEN, "bf16")
        q, k, v = self.heads(self.x)
        S.rotary_run(q, k, q, k, self.positions, self.inv_freq, self.pair_axis, "bf16")
        S.kvcache_write(k, v, self.slots, *self.cache, "bf16")
        S.prefixattn_run(q, *self.cache, self.prefix_pages, self.prompt, self.suffix_pages, self.suffix_lens, self.out, self.lse, D ** -0.5,
                         "bf16", workspace=self.workspace)
        torch.mm(self.out.view(self.batch, HEADS * D), self.proj, out=self.x)
        self.positions.add_(1)
        return q

    def plain_attention(self, q):
        """The last step's attention from what the cache holds, in plain torch and 64 bits."""
        def tokens(pages, scales, table, count):
            x = pages[table.long()].double()
            if scales is not None:
                x = x * torch.exp2(scales[table.long()].double() - 127)[..., None]
            return x.transpose(1, 2).flatten(0, 1)[:count]

        kp, vp = (tokens(self.cache[i], self.cache[i + 2], self.prefix_pages, self.prompt) for i in (0, 1))
        out = torch.empty(self.out.shape, dtype=torch.float64, device=self.device)
        for b in range(self.batch):
            k, v = (torch.cat((p, tokens(self.cache[i], self.cache[i + 2], self.suffix_pages[b], int(self.suffix_lens[b])))) for p, i in ((kp, 0), (vp, 1)))
            k, v = (t.repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1) for t in (k, v))
            w = torch.softmax((k @ q[b].double()[:, :, None])[..., 0] * D ** -0.5, 1)
            out[b] = (w[:, None] @ v)[:, 0]
        return out


def run(batch=8, prompt=1000, steps=16, cache="e4m3", check=False, graph=True):
    layer = Layer(batch, prompt, steps + 1, cache)
    layer.prefill()
    q = layer.step()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    if graph and steps > 2:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured, stream=side):
            q = layer.step()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(steps - 1):
            captured.replay()
        end.record()
        torch.cuda.synchronize()
        us = begin.elapsed_time(end) * 1e3 / (steps - 1)
    else:
        for _ in range(steps - 1):
            q = layer.step()
        torch.cuda.synchronize()
        us = None
    error = None
    if check:
        want = layer.plain_attention(q)
        error = float((layer.out.double() - want).norm() / want.norm())
    return layer, us, error


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--cache", choices=("e4m3", "same"), default="e4m3")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    if a.batch < 1 or a.prompt < 1 or a.steps < 1:
        ap.error("--batch, --prompt and --steps must be at least 1")
    layer, us, error = run(a.batch, a.prompt, a.steps, a.cache, a.check)
    print(f"{a.batch} sequences over a prompt of {a.prompt}: {int(layer.suffix_lens[0])} tokens each"
          + (f", {us:.1f} us a step" if us else "") + (f", attention {error:.1e} from plain torch" if error is not None else ""))


if __name__ == "__main__":
    main()
