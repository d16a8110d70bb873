"""The operators of a generation step in 64 bits on the CPU, and how far a result may be from them.

Every bound is derived from the roundings that the definition allows, not from results: an e4m3 number is within 2^-4 of its value (half
a step of three bits) or half a subnormal step, 2^-10 scales; bf16 within 2^-8, fp32 within 2^-24; sums of n products in fp32 within n 2^-24 of
the sum of their sizes, for which a bound of 2^-20 (2^-17 where the kernel's sums are larger than its results) stands.
"""
import numpy as np
import torch

PAGE, BLOCK = 64, 16
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
ROUND = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}     # half a step, of seven and of 23 bits, relative to the smallest number that has it


def two_to(byte):
    """Powers of two of e8m0 bytes, in 64 bits."""
    return torch.exp2(byte.view(torch.uint8).double() - 127)


def scale_exponent(most):
    """The least e >= -100 with most <= 448 * 2^e, for a 64-bit tensor."""
    e = torch.ceil(torch.log2(most.clamp(min=1e-300) / 448))
    e = torch.where(448 * torch.exp2(e - 1) >= most, e - 1, e)     # log2 of a power of two is not always exact
    return e.clamp(min=-100)


def e4m3_slack(value, scale):
    return value.abs() * 2.0 ** -4 * (1 + 1e-5) + scale * 2.0 ** -10


def e4m3(x):
    """x rounded to e4m3 numbers (to nearest, ties to even), in 64 bits; |x| <= 448."""
    a = x.abs()
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.sign(x) * torch.round(a / step) * step


def close(got, want, slack, what):
    """Elementwise |got - want| <= slack; NaN and infinities where the other has them."""
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    slack = slack.detach().cpu().double() if torch.is_tensor(slack) else torch.full_like(want, slack)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: {int((fine != torch.isfinite(got)).sum())} values are finite on one side only"
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN on one side only"
    off = ((got - want).abs() - slack)[fine]
    if off.numel():
        i = int(off.argmax())
        assert off[i] <= 0, f"{what}: {float(got[fine][i])!r} for {float(want[fine][i])!r}, {float(slack[fine][i]):.3g} allowed"


# ---- norm ---------------------------------------------------------------------------------------------------------------------


def norm(x, res, weight, eps):
    h = x.cpu().double() + (res.cpu().double() if res is not None else 0)
    return h, h / (h.square().mean(1, keepdim=True) + eps).sqrt() * weight.cpu().double()


# ---- cache ----------------------------------------------------------------------------------------------------------------------


class Cache:
    """A paged cache with random contents on the CPU, and its copy on the GPU.  before, rows: of each sequence."""

    def __init__(self, seed, before, rows, kv, dim, spare_pages=2, extra_entries=1, garbage=True):
        g = torch.Generator().manual_seed(seed)
        self.before, self.rows, self.kv, self.dim = before, rows, kv, dim
        need = [max(0, -(-(b + r) // PAGE)) for b, r in zip(before, rows)]
        n = sum(need) + spare_pages
        self.pages = torch.full((len(before), max(need + [0]) + extra_entries), -1, dtype=torch.int32)
        order = torch.randperm(n, generator=g).int()
        at = 0
        for s, p in enumerate(need):
            self.pages[s, :p] = order[at:at + p]
            at += p
        self.k = (torch.randn((n, kv, PAGE, dim), generator=g) * 60).clamp(-448, 448).to(F8)
        self.v = (torch.randn((n, kv, dim, PAGE), generator=g) * 60).clamp(-448, 448).to(F8)
        self.k_scale = torch.randint(117, 123, (n, kv, 4), generator=g, dtype=torch.uint8).view(E8)
        self.v_scale = torch.randint(117, 123, (n, kv, 4), generator=g, dtype=torch.uint8).view(E8)
        if garbage:      # places that hold no token hold NaN codes and the largest scale
            used = torch.zeros((n, PAGE), dtype=torch.bool)
            for s, b in enumerate(before):
                for t in range(max(0, b)):
                    if int(self.pages[s, t // PAGE]) >= 0:
                        used[int(self.pages[s, t // PAGE]), t % PAGE] = True
            self.k.view(torch.uint8).masked_fill_(~used[:, None, :, None], 0x7F)
            self.v.view(torch.uint8).masked_fill_(~used[:, None, None, :], 0xFF)
            free = ~used.view(n, 4, BLOCK).any(2)
            self.k_scale.view(torch.uint8).masked_fill_(free[:, None, :], 0xFE)
            self.v_scale.view(torch.uint8).masked_fill_(free[:, None, :], 0xFE)
        self.start = torch.tensor(np.cumsum([0] + list(rows)), dtype=torch.int32)

    def gpu(self, D):
        c = [t.cuda() for t in (self.k, self.v, self.k_scale, self.v_scale, self.pages, torch.tensor(self.before, dtype=torch.int32))]
        self.on_gpu = c
        return D.make_cache(*c)

    def filled(self, seed):
        """Writes the step's own tokens too (random codes), as an append would have."""
        g = torch.Generator().manual_seed(seed)
        for s, (b, r) in enumerate(zip(self.before, self.rows)):
            for t in range(max(0, b), b + r):
                page = int(self.pages[s, t // PAGE])
                if page < 0:
                    continue
                i = t % PAGE
                self.k[page, :, i] = (torch.randn((self.kv, self.dim), generator=g) * 60).clamp(-448, 448).to(F8)
                self.v[page, :, :, i] = (torch.randn((self.kv, self.dim), generator=g) * 60).clamp(-448, 448).to(F8)
                for sc in (self.k_scale, self.v_scale):
                    u = sc.view(torch.uint8)[page, :, i // BLOCK]
                    u[u == 0xFE] = 119
        return self

    def tokens(self, s, total):
        """Keys and values [kv][total][dim] of a sequence in 64 bits, and which of them are there."""
        k = torch.zeros((self.kv, max(total, 0), self.dim), dtype=torch.float64)
        v = torch.zeros_like(k)
        there = torch.zeros(max(total, 0), dtype=torch.bool)
        ks, vs = two_to(self.k_scale), two_to(self.v_scale)
        for t in range(total):
            page = int(self.pages[s, t // PAGE]) if t // PAGE < self.pages.shape[1] else -1
            if 0 <= page < self.k.shape[0]:
                i = t % PAGE
                there[t] = True
                k[:, t] = self.k[page, :, i].double() * ks[page, :, i // BLOCK, None]
                v[:, t] = self.v[page, :, :, i].double() * vs[page, :, i // BLOCK, None]
        return k, v, there


def turn_table(positions, rot, base=10000.0):
    at = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([at.cos(), at.sin()], 1).float()


def turned(x, row, rot, pairs):
    """x [heads][dim] in 64 bits turned by a row of the table."""
    y = x.clone()
    c, s = row[:rot // 2].double(), row[rot // 2:].double()
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def attend(cache, q, scale, window, dtype):
    """Outputs [rows][heads][dim] in 64 bits and the bound on a result's error."""
    n, heads, dim = q.shape
    out = torch.zeros((n, heads, dim), dtype=torch.float64)
    slack = torch.zeros_like(out)
    part = {"bf16": 2.0 ** -11, "fp32": 2.0 ** -20}[dtype]       # of a weight in f16 parts
    for s, (b, r) in enumerate(zip(cache.before, cache.rows)):
        k, v, there = cache.tokens(s, b + r)
        for i in range(r):
            row, pos = int(cache.start[s]) + i, b + i
            t = torch.arange(k.shape[1])
            see = there & (t <= pos)
            if window:
                see &= t > pos - window
            if not bool(see.any()):
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


# ---- 4-bit products -----------------------------------------------------------------------------------------------------------


def matvec(x, w, w_scale, gate, dtype):
    """Outputs in 64 bits (x in 64 bits) and the bound on a result's error."""
    codes = torch.stack([w & 15, w >> 4], 2).view(w.shape[0], -1).double() - 8
    group = codes.shape[1] // w_scale.shape[1]
    ww = codes * w_scale.double().repeat_interleave(group, 1)
    y, size = x @ ww.t(), x.abs() @ (w_scale.double().abs().repeat_interleave(group, 1) * 8).t()
    off = size * {"bf16": 2.0 ** -17, "fp32": 2.0 ** -20}[dtype]
    if gate:
        a, b = y[:, 0::2], y[:, 1::2]
        s = a * torch.sigmoid(a)
        off = off[:, 0::2] * 1.1 * b.abs() + (s.abs() + off[:, 0::2] * 1.1) * off[:, 1::2] + (s * b).abs() * 2.0 ** -20     # |d silu| <= 1.1
        y = s * b
    return y, off + y.abs() * ROUND[dtype] + 1e-30
