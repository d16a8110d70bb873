"""The operators of a drafted step in 64 bits on the CPU: trees as masks, attention of their nodes, words drawn by given random numbers, the walk
down a tree, and the cache's tokens that stay.  (Bounds: see step_helpers.)"""
import math
from fractions import Fraction

import numpy as np
import torch

from step_helpers import BLOCK, F8, PAGE, ROUND


def random_parents(rng, n, reach=6):
    return [-1] + [int(rng.integers(max(0, i - reach), i)) for i in range(1, n)] if n else []


def bits_of(mask_row):
    """Numbers of the bits of a row of masks (an int64 tensor or list of words)."""
    return [64 * w + b for w, word in enumerate(mask_row) for b in range(64) if int(word) >> b & 1]


def sees(mask_row, before, rows, window):
    """Tokens that a row attends, in order: cached ones, then the nodes of its mask."""
    tokens = list(range(max(0, before))) if before > 0 else []
    tokens += [before + j for j in bits_of(mask_row) if j < rows]
    # (a token in front of the first has no place, but counts among the last `window`)
    return [t for t in (tokens[-window:] if window else tokens) if t >= 0]


def attend_tree(cache, masks, q, scale, window, dtype):
    """Outputs [rows][heads][dim] in 64 bits and the bound on a result's error."""
    n, heads, dim = q.shape
    out = torch.zeros((n, heads, dim), dtype=torch.float64)
    slack = torch.zeros_like(out)
    part = {"bf16": 2.0 ** -11, "fp32": 2.0 ** -20}[dtype]       # of a weight in f16 parts
    for s, (b, r) in enumerate(zip(cache.before, cache.rows)):
        k, v, there = cache.tokens(s, b + r)
        for i in range(r):
            row = int(cache.start[s]) + i
            see = torch.tensor([t for t in sees(masks[row].tolist(), b, r, window) if bool(there[t])], dtype=torch.long)
            if not len(see):
                continue
            for h in range(heads):
                kk, vv, qq = k[h * cache.kv // heads][see], v[h * cache.kv // heads][see], q[row, h].cpu().double()
                x = kk @ qq * scale
                p = torch.softmax(x, 0)
                size = p @ vv.abs()
                # a score's error: 22 bits of a product's operands, the sum in fp32
                score = float((kk.abs() @ qq.abs()).nan_to_num(0, 0, 0).max() * abs(scale)) * 2.0 ** -20
                out[row, h] = p @ vv
                slack[row, h] = size * (2 * part + 2 * score + 2.0 ** -18) + out[row, h].abs() * ROUND[dtype] + 1e-30
    return out, slack


def drawn(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Word and chance of one row of logits, from the definition: the words from the largest down, until a limit is met."""
    x = x.double().numpy().copy()
    x[np.isnan(x)] = -np.inf
    x += 0.0
    most = x.max()
    if most == -np.inf:
        return -1, 0.0
    if not temperature > 0 or u is None:
        return int(np.argmax(x)), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        bits = np.where(x == most, 0.0, (x - most) / temperature * math.log2(math.e))
    live = np.flatnonzero((bits >= -64) & (x > -np.inf))
    live = live[np.lexsort((live, -x[live]))]
    if top_k > 0:
        live = live[:top_k]
    # sums in whole numbers, 2^-117 each: none of them is rounded, so that equal weights are cut where their number says
    w = [int(v * 2.0 ** 64) << 53 | int(math.ldexp(math.fmod(v * 2.0 ** 64, 1.0), 53)) for v in np.exp2(bits[live])]
    if top_p < 1:
        need, front = Fraction(top_p) * sum(w), 0
        for n, v in enumerate(w):
            if n and front >= need:
                live, w = live[:n], w[:n]
                break
            front += v
    least = Fraction(min_p) * 2 ** 117 if min_p > 0 else 0
    left = sorted((int(i), v) for n, (i, v) in enumerate(zip(live, w)) if n == 0 or v >= least)
    total, upto = sum(v for _, v in left), 0
    target = Fraction(u if u >= 0 else 0.0) * total
    for i, v in left:
        upto += v
        if upto > target:
            break
    return i, v / total


def walk(masks, words, answers):
    """Nodes of one tree from the root on, and the answer behind the last."""
    n = min(len(words), 64 * masks.shape[1])
    if n == 0:
        return [], -1
    parent = [max([b for b in bits_of(masks[i].tolist()) if b < i], default=-1) for i in range(n)]
    line = [0]
    while True:
        below = [i for i in range(n) if parent[i] == line[-1] and words[i] == answers[line[-1]] and words[i] >= 0]
        if not below:
            return line, answers[line[-1]]
        line.append(below[0])


def kept(cache, path, count):
    """Codes and scales of the cache after the nodes `path` (of all rows) of each sequence have been kept: copies of k, v, k_scale, v_scale."""
    out = {n: getattr(cache, n).clone() for n in ("k", "v", "k_scale", "v_scale")}
    page_of = lambda s, t: int(cache.pages[s, t // PAGE]) if 0 <= t and t // PAGE < cache.pages.shape[1] and 0 <= int(cache.pages[s, t // PAGE]) < cache.k.shape[0] else -1  # noqa: E731
    for s, (b, r) in enumerate(zip(cache.before, cache.rows)):
        line, row0 = [], int(cache.start[s])
        for j in range(min(max(count[s], 0), r)):
            p = path[row0 + j]
            if p < 0 or p >= r or (line and p <= line[-1]):
                break
            line.append(p)
        moved = {b + j: b + p for j, p in enumerate(line) if p != j}
        first = min(moved, default=0)
        for begin in sorted({t // BLOCK * BLOCK for t in moved if t >= 0}):
            page, blk = page_of(s, begin), begin % PAGE // BLOCK
            come = {t: moved[t] for t in range(max(begin, 0), begin + BLOCK) if t in moved and page_of(s, moved[t]) >= 0}
            if page < 0 or not come:
                continue
            for name in ("k", "v"):
                codes, scales = getattr(cache, name), getattr(cache, name + "_scale").view(torch.uint8)
                token = lambda c, g, t: c[g, :, t % PAGE] if name == "k" else c[g, :, :, t % PAGE]  # noqa: E731
                new = out[name]
                had = scales[page, :, blk].int()
                stay = [t for t in range(begin, begin + BLOCK) if t < first]
                came = {t: scales[page_of(s, at), :, at % PAGE // BLOCK].int() for t, at in come.items()}
                now = torch.stack(list(came.values()) + ([had] if stay else [])).amax(0)
                turned = lambda x, was: (x.double() * torch.exp2((was - now).double())[:, None]).float().to(F8)  # noqa: E731
                for t in stay:
                    if bool((now > had).any()):
                        token(new, page, t).copy_(torch.where((now > had)[:, None], turned(token(codes, page, t), had).float(), token(codes, page, t).float()).to(F8))
                for t, at in come.items():
                    token(new, page, t).copy_(turned(token(codes, page_of(s, at), at), came[t]))
                out[name + "_scale"].view(torch.uint8)[page, :, blk] = now.to(torch.uint8)
    return out


def same_codes(got, want, what):
    """Equal bytes, but that a NaN may be either of its two codes."""
    got, want = got.cpu(), want.cpu()
    a, b = got.view(torch.uint8), want.view(torch.uint8)
    off = (a != b) & ~(torch.isnan(got.float()) & torch.isnan(want.float()))
    assert not bool(off.any()), f"{what}: {int(off.sum())} codes differ, the first at {off.nonzero()[0].tolist()}"
