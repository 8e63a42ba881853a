"""Plain forms of the operators that check drafted tokens, in 64 bits or whole numbers on the CPU.  Test infrastructure: no code of the
package."""
from __future__ import annotations

import math
import random

import torch

import serving_ref as R


def signed(x):
    """64 bits as the number that int64 holds."""
    return x - (1 << 64) if x >> 63 else x


def tree_masks(rng, batch, nodes, odd=False):
    """Trees: bit j of a node's mask is itself or an ancestor; some of the last nodes are padding.  odd: some masks are any bits, and bits
    beyond the nodes are set."""
    rows = []
    for b in range(batch):
        real = nodes if b % 3 != 1 else max(1, nodes - rng.randint(0, nodes // 2))
        seen = [1]
        for i in range(1, real):
            seen.append(seen[rng.randint(max(0, i - 4), i - 1)] | 1 << i)
        seen += [0] * (nodes - real)
        if odd:
            for i in range(nodes):
                if rng.random() < 0.2:
                    seen[i] = rng.getrandbits(64)
                elif rng.random() < 0.2:
                    seen[i] |= ((1 << 64) - 1) >> nodes << nodes
        rows.append(seen)
    return rows


def int64_masks(rows):
    return torch.tensor([[signed(m & ((1 << 64) - 1)) for m in row] for row in rows], dtype=torch.int64)


def tree_attention(q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len, suffix_pages, suffix_lens, masks, scale):
    """(out, lse, size) row by row; size = sum of softmax weights times |v|, which roundings of the weights go by."""
    pages, hk, page, d = k_pages.shape
    rows, hq, _ = q.shape
    batch, nodes = masks.shape
    group = hq // hk
    out, size = (torch.zeros(rows, hq, d, dtype=torch.float64) for _ in range(2))
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64)

    def gather(x, s, at):
        if not at:
            return torch.zeros(0, hk, d, dtype=torch.float64)
        p, o = torch.tensor(at).T
        return R.values(x[p, :, o], None if s is None else s[p, :, o])

    pre = [(int(prefix_pages[j // page]), j % page) for j in range(prefix_len)]
    pre = [(p, o) for p, o in pre if 0 <= p < pages]
    kp, vp = gather(k_pages, k_scale, pre), gather(v_pages, v_scale, pre)
    for b in range(batch):
        width = 0 if suffix_pages is None else suffix_pages.shape[1] * page
        n = max(int(suffix_lens[b]), 0) if width else 0
        here = [j for j in range(min(n + nodes, width)) if 0 <= int(suffix_pages[b, j // page]) < pages]
        at = [(int(suffix_pages[b, j // page]), j % page) for j in here]
        k, v = torch.cat((kp, gather(k_pages, k_scale, at))), torch.cat((vp, gather(v_pages, v_scale, at)))
        node = torch.tensor([-1] * len(pre) + [j - n for j in here], dtype=torch.int64)
        for i in range(nodes):
            seen = (node < 0) | ((masks[b, i] >> node.clamp(0, 63) & 1) != 0)
            if not bool(seen.any()):
                continue
            row, heads = b * nodes + i, torch.arange(hq) // group
            kk, vv = k[seen][:, heads].transpose(0, 1), v[seen][:, heads].transpose(0, 1)
            z = (kk @ q[row].double()[:, :, None])[..., 0] * scale
            w = torch.softmax(z, 1)[:, None]
            lse[row], out[row], size[row] = torch.logsumexp(z, 1), (w @ vv)[:, 0], (w @ vv.abs())[:, 0]
    return out, lse, size


def counts(case, b, i):
    """(made, met) of a row's tokens as the lists say."""
    vocab = case["logits"].shape[1]
    made, met = torch.zeros(vocab, dtype=torch.int64), torch.zeros(vocab, dtype=torch.bool)
    if case.get("penalties") is None:
        return made, met
    if case.get("history") is not None:
        width = case["history"].shape[1]
        n = min(max(int(case["history_lens"][b]), 0), width)
        prompt = min(max(int(case["prompt_lens"][b]), 0), n) if case.get("prompt_lens") is not None else 0
        for j, t in enumerate(case["history"][b, :n].tolist()):
            if 0 <= t < vocab:
                met[t] = True
                made[t] += j >= prompt
    if case.get("tree_masks") is not None:
        for j, t in enumerate(case["tree_tokens"][b].tolist()):
            if int(case["tree_masks"][b, i]) >> j & 1 and 0 <= t < vocab:
                made[t] += 1
    return made, met | (made > 0)


def logits(case, nodes, wide):
    """z of every row: in 64 bits, or with every step rounded to fp32, in the order of the steps; and the sum of the magnitudes it goes through."""
    t = torch.float64 if wide else torch.float32
    x = case["logits"].to(t)
    rows, vocab = x.shape
    z, size = torch.empty_like(x), torch.zeros(rows, vocab, dtype=torch.float64)
    for row in range(rows):
        b, i = divmod(row, nodes)
        y = x[row]
        made, met = counts(case, b, i)
        big = y.abs().double()
        if case.get("penalties") is not None:
            r, f, p = case["penalties"][b].to(t)
            y = torch.where(met, torch.where(y > 0, y / r, y * r), y)
            big = torch.maximum(big, y.abs().double()) + f.abs().double() * made + p.abs().double()
            y = torch.where(made > 0, y - f * made.to(t), y)
            y = torch.where(made > 0, y - p, y)
        if case.get("bias_tokens") is not None:
            total, there, mass = torch.zeros(vocab, dtype=t), torch.zeros(vocab, dtype=torch.bool), torch.zeros(vocab, dtype=torch.float64)
            for token, value in zip(case["bias_tokens"][b].tolist(), case["bias_values"][b]):
                if 0 <= token < vocab:
                    total[token] = total[token] + value.to(t) if there[token] else value.to(t)
                    there[token] = True
                    mass[token] += abs(float(value))
            y = torch.where(there, y + total, y)
            big = big + mass
        if case.get("allowed") is not None:
            word = case["allowed"][row].to(torch.int64)
            token = torch.arange(vocab)
            y = torch.where((word[token // 32] >> token % 32 & 1) != 0, y, torch.full_like(y, -math.inf))
        z[row], size[row] = y, big
    return z, size


def best(z):
    """The lowest token of the largest z, NaN being larger than all numbers."""
    got = []
    for row in z:
        nan = row.isnan()
        got.append(int(nan.nonzero()[0]) if nan.any() else int((row == row.max()).nonzero()[0]))
    return torch.tensor(got, dtype=torch.int32)


def accept(chosen, tokens, masks, suffix_pages, suffix_lens, page, pages, depth):
    """(path, count, next_token, from_slots, to_slots), node by node."""
    batch, nodes = masks.shape
    path, count, follows, f, t = [], [], [], [], []
    for b in range(batch):
        sets = [{j for j in range(nodes) if int(m) >> j & 1} for m in masks[b]]
        walk = [0] if 0 in sets[0] else []
        while walk and len(walk) < depth:
            here = walk[-1]
            children = [c for c in range(nodes) if c not in sets[here] and sets[c] == sets[here] | {c} and int(tokens[b, c]) == int(chosen[b, here])]
            if not children:
                break
            walk.append(children[0])

        def slot(position):
            if position >= suffix_pages.shape[1] * page:
                return -1
            p = int(suffix_pages[b, position // page])
            return p * page + position % page if 0 <= p < pages else -1

        fs, ts = [], []
        for k in range(depth):
            x = y = -1
            if k < len(walk) and walk[k] != k and suffix_pages is not None:
                n = max(int(suffix_lens[b]), 0)
                x, y = slot(n + walk[k]), slot(n + k)
                if x < 0 or y < 0:
                    x = y = -1
            fs.append(x)
            ts.append(y)
        path.append(walk + [-1] * (depth - len(walk)))
        count.append(len(walk))
        follows.append(int(chosen[b, walk[-1]]) if walk else -1)
        f.append(fs)
        t.append(ts)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    i64 = lambda x: torch.tensor(x, dtype=torch.int64)  # noqa: E731
    return i32(path), i32(count), i32(follows), i64(f), i64(t)


def move(pages, from_slots, to_slots):
    """A tensor [pages, heads, page, ...] after its tokens have moved, group by group, all of a group read first."""
    x = pages.clone()
    count, page = x.shape[0], x.shape[2]
    for f, t in zip(from_slots.tolist(), to_slots.tolist()):
        pairs = [(a, b) for a, b in zip(f, t) if 0 <= a < count * page and 0 <= b < count * page]
        read = [x[a // page, :, a % page].clone() for a, _ in pairs]
        for (_, b), v in zip(pairs, read):
            x[b // page, :, b % page] = v
    return x


def rng(seed):
    return random.Random(seed)
