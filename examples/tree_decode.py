#!/usr/bin/env python3
"""One attention layer that answers a shared prompt with several sequences at once, several tokens a step (needs an MI355X).

    python examples/tree_decode.py [--batch 8] [--prompt 1000] [--steps 16] [--cache e4m3|same] [--check]

Every step a table guesses a tree of tokens behind each sequence's last one, the layer sees all nodes at once, and the path of guesses
that the layer agrees with is kept: rotary positions by a node's depth, the nodes' keys behind their sequence's, attention over the
prompt (read once for all), the sequence's own tokens and the nodes that a node comes from, logits with penalties for what is
repeated, the best token after each node, the path that agrees, and its keys side by side in the cache.  Weights are random;
products with them are torch's.  A step is captured into a HIP graph and replayed.  ``--check`` compares the last step with plain torch.
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
from paper_2601_12698_amd import drafting as D         # noqa: E402
from paper_2601_12698_amd import serving as S          # noqa: E402

HEADS, KV_HEADS, HEAD, HIDDEN, VOCAB, PAGE, EPS = 16, 4, 128, 1024, 40000, 16, 1e-6
# the tree: three guesses for the next token, two behind the first, then one behind each of the first two, and so on
PARENTS = (-1, 0, 0, 0, 1, 1, 2, 4, 5, 7, 9)
GUESS = (0, 0, 1, 2, 0, 1, 0, 0, 0, 0, 0)               # which of its parent's guesses a node is
DEPTH = 6                                               # nodes of the longest path


def tree():
    """(masks, depths): a node's mask has its own bit and those of the nodes it comes from."""
    masks, depths = [1], [0]
    for i, p in enumerate(PARENTS[1:], 1):
        masks.append(masks[p] | 1 << i)
        depths.append(depths[p] + 1)
    return masks, depths


class Layer:
    def __init__(self, batch: int, prompt: int, steps: int, cache: str, device="cuda", seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *shape, std: (torch.randn(shape, generator=g, device=device) * std).to(torch.bfloat16)  # noqa: E731
        self.batch, self.prompt, self.nodes, self.device = batch, prompt, len(PARENTS), device
        self.embed, self.head = rand(VOCAB, HIDDEN, std=1.0), rand(HIDDEN, VOCAB, std=3 * HIDDEN ** -0.5)
        self.qkv, self.proj = rand(HIDDEN, (HEADS + 2 * KV_HEADS) * HEAD, std=HIDDEN ** -0.5), rand(HEADS * HEAD, HIDDEN, std=(HEADS * HEAD) ** -0.5)
        self.norm = torch.ones(HIDDEN, dtype=torch.bfloat16, device=device)
        self.inv_freq, self.pair_axis = S.rotary_plan(HEAD, 10000.0, (HEAD // 2,), device)
        room = steps * DEPTH + self.nodes
        first, own = -(-prompt // PAGE), -(-room // PAGE)
        self.pages = pages = first + batch * own
        kind = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
        self.cache = [torch.zeros((pages, KV_HEADS, PAGE, HEAD), dtype=kind, device=device) for _ in range(2)]
        self.cache += [torch.full((pages, KV_HEADS, PAGE), 127, dtype=torch.uint8, device=device) for _ in range(2)] if cache == "e4m3" else [None, None]
        table = torch.randperm(pages, generator=g, device=device).to(torch.int32)
        self.prefix_pages, self.suffix_pages = table[:first].contiguous(), table[first:].view(batch, own).contiguous()
        masks, depths = tree()
        self.masks = torch.tensor([masks] * batch, dtype=torch.int64, device=device)
        self.depths = torch.tensor(depths, dtype=torch.int64, device=device)
        # what the table guesses behind each token: the layer's own answers without any attention
        x = self.embed.clone()
        B.addrms_run(x, torch.zeros_like(x), self.norm, EPS, VOCAB, HIDDEN, "bf16")
        self.guesses = torch.cat([(part @ self.head).topk(3, 1).indices for part in x.split(4000)])
        # the prompt, and the token that each sequence begins with, as if drawn after it: node 0 of the first tree, which counts as made
        tokens = torch.randint(0, VOCAB, (prompt + batch,), generator=g, device=device)
        self.prompt_tokens, self.last = tokens[:prompt], tokens[prompt:].to(torch.int32)
        # what a step works on besides: the certain tokens before node 0, and lengths
        self.history = torch.zeros((batch, prompt + room + 1), dtype=torch.int32, device=device)
        self.history[:, :prompt] = self.prompt_tokens
        self.history_lens = torch.full((batch,), prompt, dtype=torch.int32, device=device)
        self.prompt_lens, self.suffix_lens = self.history_lens.clone(), torch.zeros(batch, dtype=torch.int32, device=device)
        self.penalties = torch.tensor([[1.1, 0.2, 0.1]] * batch, device=device)
        rows = batch * self.nodes
        self.tokens, self.best = torch.zeros((batch, self.nodes), dtype=torch.int32, device=device), torch.zeros((batch, self.nodes), dtype=torch.int32, device=device)
        self.path, self.count = torch.zeros((batch, DEPTH), dtype=torch.int32, device=device), torch.zeros(batch, dtype=torch.int32, device=device)
        self.from_slots, self.to_slots = (torch.zeros((batch, DEPTH), dtype=torch.int64, device=device) for _ in range(2))
        self.out, self.lse = torch.empty((rows, HEADS, HEAD), dtype=torch.bfloat16, device=device), torch.empty((rows, HEADS), device=device)
        shape = S.prefixattn_shape(batch, self.nodes, HEADS, KV_HEADS, HEAD, PAGE, pages, prompt, own, "bf16", cache == "e4m3")
        self.workspace = torch.empty(max(16, D.treeattn_workspace_bytes(shape), D.logits_workspace_bytes(batch, self.nodes, VOCAB, "bf16")), dtype=torch.uint8,
                                     device=device)

    def heads(self, x):
        qkv = (x @ self.qkv).view(x.shape[0], HEADS + 2 * KV_HEADS, HEAD)
        return qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]

    def embedded(self, tokens):
        """Normalised embeddings, and the residual stream."""
        x = self.embed[tokens.long()]
        residual = torch.zeros_like(x)
        B.addrms_run(x, residual, self.norm, EPS, x.shape[0], HIDDEN, "bf16")
        return x, residual

    def prefill(self):
        """The prompt's keys and values go into the pages all share."""
        n = self.prompt
        x, _ = self.embedded(self.prompt_tokens)
        q, k, v = self.heads(x)
        token = torch.arange(n, device=self.device)
        S.rotary_run(q, k, q, k, token[None], self.inv_freq, self.pair_axis, "bf16")
        S.kvcache_write(k, v, self.prefix_pages[token // PAGE].long() * PAGE + token % PAGE, *self.cache, "bf16")

    def step(self):
        """One tree of every sequence.  Nothing here depends on the host: it can be captured."""
        batch, nodes = self.batch, self.nodes
        self.tokens[:, 0] = self.last
        for i, p in enumerate(PARENTS[1:], 1):
            self.tokens[:, i] = self.guesses[self.tokens[:, p].long(), GUESS[i]]
        x, residual = self.embedded(self.tokens.flatten())
        q, k, v = self.heads(x)
        begin = self.suffix_lens.long()[:, None]
        at = begin + torch.arange(nodes, device=self.device)
        slots = torch.gather(self.suffix_pages.long(), 1, at // PAGE) * PAGE + at % PAGE
        positions = (self.prompt + begin + self.depths).view(1, -1)
        S.rotary_run(q, k, q, k, positions, self.inv_freq, self.pair_axis, "bf16")
        S.kvcache_write(k, v, slots.flatten(), *self.cache, "bf16")
        D.treeattn_run(q, *self.cache, self.prefix_pages, self.prompt, self.suffix_pages, self.suffix_lens, self.masks, self.out, self.lse, HEAD ** -0.5,
                       "bf16", workspace=self.workspace)
        y = self.out.view(batch * nodes, HEADS * HEAD) @ self.proj
        B.addrms_run(y, residual, self.norm, EPS, batch * nodes, HIDDEN, "bf16")
        logits = y @ self.head
        D.logits_run(logits, None, self.best.view(-1), "bf16", nodes=nodes, history=self.history, history_lens=self.history_lens, prompt_lens=self.prompt_lens,
                     penalties=self.penalties, tree_tokens=self.tokens, tree_masks=self.masks, workspace=self.workspace)
        D.treeaccept_run(self.best, self.tokens, self.masks, self.suffix_pages, self.suffix_lens, PAGE, self.pages, self.path, self.count, self.last,
                         self.from_slots, self.to_slots)
        D.kvmove_run(*self.cache, self.from_slots, self.to_slots, "bf16")
        # the path's tokens are certain now; those beyond it go to a place that nothing reads
        kept = self.tokens.gather(1, self.path.clamp(min=0).long())
        to = torch.where(self.path >= 0, self.history_lens.long()[:, None] + torch.arange(DEPTH, device=self.device), self.history.shape[1] - 1)
        self.history.scatter_(1, to, kept)
        self.history_lens.add_(self.count)
        self.suffix_lens.add_(self.count)
        return q, k, v, logits

    def plain_attention(self, q, k, v, before):
        """The last step's attention in plain torch and 64 bits, from the cache below the trees and the nodes' own keys and values; `before`:
        lengths that the step began with."""
        def tokens(pages, scales, table, count):
            x = pages[table.long()].double()
            if scales is not None:
                x = x * torch.exp2(scales[table.long()].double() - 127)[..., None]
            return x.transpose(1, 2).flatten(0, 1)[:count]

        def stored(x):
            """Keys or values as the cache holds them."""
            if self.cache[2] is None:
                return x
            pages = [torch.zeros((x.shape[0], KV_HEADS, 1, HEAD), dtype=torch.float8_e4m3fn, device=x.device) for _ in range(2)]
            scales = [torch.zeros((x.shape[0], KV_HEADS, 1), dtype=torch.uint8, device=x.device) for _ in range(2)]
            S.kvcache_write(x, x, torch.arange(x.shape[0], device=x.device), *pages, *scales, "bf16")
            return pages[0][:, :, 0].double() * torch.exp2(scales[0][:, :, 0].double() - 127)[..., None]

        kp, vp = (tokens(self.cache[i], self.cache[i + 2], self.prefix_pages, self.prompt) for i in (0, 1))
        k, v = (stored(x.contiguous()).double().view(self.batch, self.nodes, KV_HEADS, HEAD) for x in (k, v))
        out = torch.empty(self.out.shape, dtype=torch.float64, device=self.device).view(self.batch, self.nodes, HEADS, HEAD)
        for b in range(self.batch):
            n = int(before[b])
            own = [tokens(self.cache[i], self.cache[i + 2], self.suffix_pages[b], n) for i in (0, 1)]
            for i in range(self.nodes):
                seen = [j for j in range(self.nodes) if int(self.masks[b, i]) >> j & 1]
                kk, vv = (torch.cat((p, o, x[b, seen])).repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1) for p, o, x in ((kp, own[0], k), (vp, own[1], v)))
                w = torch.softmax((kk @ q.view(self.batch, self.nodes, HEADS, HEAD)[b, i].double()[:, :, None])[..., 0] * HEAD ** -0.5, 1)
                out[b, i] = (w[:, None] @ vv)[:, 0]
        return out.view(self.out.shape)


def run(batch=8, prompt=1000, steps=16, cache="e4m3", check=False, graph=True):
    """(layer, us a step or None, attention's distance from plain torch or None, the last step's (q, k, v, logits), lengths before it)."""
    layer = Layer(batch, prompt, steps, cache)
    layer.prefill()
    last = layer.step()
    before = layer.suffix_lens.clone()
    us = None
    torch.cuda.synchronize()
    if graph and steps > 2:
        captured, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(captured, stream=side):
            last = layer.step()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(steps - 2):
            captured.replay()
        end.record()
        before = layer.suffix_lens.clone()
        captured.replay()
        torch.cuda.synchronize()
        us = begin.elapsed_time(end) * 1e3 / (steps - 2)
    else:
        for _ in range(steps - 1):
            before = layer.suffix_lens.clone()
            last = layer.step()
        torch.cuda.synchronize()
    error = None
    if check:
        if steps == 1:
            before = torch.zeros_like(before)
        want = layer.plain_attention(*last[:3], before)
        error = float((layer.out.double() - want).norm() / want.norm())
    return layer, us, error, last, before


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
    layer, us, error, _, _ = run(a.batch, a.prompt, a.steps, a.cache, a.check)
    print(f"{a.batch} sequences over a prompt of {a.prompt}: {float(layer.suffix_lens.float().mean()) / a.steps:.2f} tokens a step"
          + (f", {us:.1f} us a step" if us else "") + (f", attention {error:.1e} from plain torch" if error is not None else ""))


if __name__ == "__main__":
    main()
