"""Plain 64-bit forms of rotary positions, the quantised cache and attention over a shared prefix, on the CPU, and the
distances that roundings to 16 and 8 bits allow.  Test infrastructure: no code of the package."""
from __future__ import annotations

import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF_STEP = {n: torch.finfo(t).eps / 2 for n, t in TYPES.items()}
MOST = {"fp16": 61440.0, "bf16": 15.0 * 2.0 ** 124}          # the largest magnitude of four significant bits


def rotary(x, positions, inv_freq, pair_axis, inverse=False, interleaved=False):
    """[T, H, d] of any type -> fp64."""
    x, pairs = x.double().clone(), inv_freq.numel()
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        angle = positions[int(pair_axis[i])].double() * inv_freq[i]
        c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
        u, v = x[:, :, a].clone(), x[:, :, b].clone()
        x[:, :, a], x[:, :, b] = u * c - v * s, u * s + v * c
    return x


def quantise(x, dtype):
    """fp16 or bf16 rows [..., d] -> (values of the codes in fp64, scale bytes)."""
    x = x.double()
    fine = torch.isfinite(x)
    y = torch.where(fine, x.clamp(-MOST[dtype], MOST[dtype]), torch.full_like(x, math.nan)).numpy()
    a = np.nanmax(np.abs(np.where(fine.numpy(), y, 0.0)), axis=-1)
    e = np.zeros(a.shape, np.int64)
    for at in np.ndindex(a.shape):
        if a[at] > 0:
            n = -200
            while math.ldexp(a[at], -n) > 448:
                n += 1
            e[at] = min(127, max(-126, n))
    z = np.ldexp(y, -e[..., None])
    _, f = np.frexp(np.where(np.isnan(z), 0.0, z))
    step = np.ldexp(1.0, np.maximum(f - 4, -9))
    return torch.from_numpy(np.rint(z / step) * step), torch.from_numpy((e + 127).astype(np.uint8))


def values(codes, scales):
    """What a cache stands for, in fp64; codes of any type."""
    x = codes.double() if codes.dtype != torch.uint8 else codes.view(torch.float8_e4m3fn).double()
    return x if scales is None else torch.from_numpy(np.ldexp(x.numpy(), scales.view(torch.uint8).numpy().astype(np.int64)[..., None] - 127))


def attention(q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len, suffix_pages, suffix_lens, scale, q_len):
    """(out, lse, size) in fp64 on the CPU, row by row; size = sum of softmax weights times |v|, which roundings of the weights go by."""
    pages, hk, page, d = k_pages.shape
    rows, hq, _ = q.shape
    group = hq // hk
    out, lse, size = torch.zeros(rows, hq, d, dtype=torch.float64), torch.full((rows, hq), -math.inf, dtype=torch.float64), torch.zeros(rows, hq, d, dtype=torch.float64)

    def places(table, count):
        got = [(int(table[j // page]), j % page) for j in range(count)]
        return [(p, o) for p, o in got if 0 <= p < pages]

    def tokens(x, s, at):
        if not at:
            return torch.zeros(0, hk, d, dtype=torch.float64)
        p, o = torch.tensor(at).T
        return values(x[p, :, o], None if s is None else s[p, :, o])

    pre = places(prefix_pages, prefix_len) if prefix_len else []
    kp, vp = tokens(k_pages, k_scale, pre), tokens(v_pages, v_scale, pre)
    for b in range(rows // q_len):
        width = 0 if suffix_pages is None else suffix_pages.shape[1] * page
        n = min(max(int(suffix_lens[b]), 0), width) if width else 0
        at = places(suffix_pages[b], n) if n else []
        here = [j for j in range(n) if 0 <= int(suffix_pages[b, j // page]) < pages] if n else []
        k, v = torch.cat((kp, tokens(k_pages, k_scale, at))), torch.cat((vp, tokens(v_pages, v_scale, at)))
        for i in range(q_len):
            row, end = b * q_len + i, len(pre) + sum(j <= n - q_len + i for j in here)
            if end == 0:
                continue
            heads = torch.arange(hq) // group
            kk, vv = k[:end, heads].transpose(0, 1), v[:end, heads].transpose(0, 1)          # [heads, keys, d]
            z = (kk @ q[row].double()[:, :, None])[..., 0] * scale
            w = torch.softmax(z, 1)[:, None]
            lse[row], out[row], size[row] = torch.logsumexp(z, 1), (w @ vv)[:, 0], (w @ vv.abs())[:, 0]
    return out, lse, size
