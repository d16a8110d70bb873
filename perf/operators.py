"""What is measured of the operators of a generation step: norm, cache append, attention over the cache, 4-bit products.

A step of a decoder block is  norm -> product -> append -> attend -> product -> norm -> gated product -> product.  Each case
here is one such operator on sizes that a step meets: single tokens, where the launch counts, batches of sequences of unequal
lengths, and chunks of a prompt.  The sizes are generic ones (rows of 4096, 32 query heads on 8 key heads of 128 channels)
and, where a product is wanted that is no decoder's, VGG-16's classifier (25088 -> 4096) of this repository's own networks.

Eight bits are an e4m3 number and a power of two (e8m0) that a group of them shares:

* norm     ``group`` neighbouring channels of a row share a scale
* cache    pages of 64 tokens, keys [page][head][token][channel], values [page][head][channel][token]; 16 tokens of a
           head share a scale, the smallest power of two that leaves none of them above 448
* product  weights are whole numbers from -8 to 7, two to a byte (the earlier channel in the low half, 8 added), with a bf16
           scale for each ``wgroup`` channels of an output

`own` says which side ``run`` takes: elementary torch operations in 32 bits, or the library's calls.
"""
import math

import torch

own = False

PAGE, BLOCK = 64, 16
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5
LEAST = 27  # exponent bits of the smallest scale, 2^-100


def listed():
    return [
        # one token of one stream in front of an 8-bit product: nothing but latency
        dict(name="norm one token", op="norm", rows=1, width=4096, dtype="bf16", res=True, group=128),
        # rows of no round size, read from a wider buffer, in full precision
        dict(name="norm odd fp32", op="norm", rows=173, width=2050, dtype="fp32", res=False, group=0),
        # a prompt of 8192 tokens: the longest rows x width that a chunk brings
        dict(name="norm prompt", op="norm", rows=8192, width=4096, dtype="bf16", res=True, group=128),
        # one new token for each of 32 streams
        dict(name="append 32 streams", op="append", seqs=32, rows=1, ctx=4000, heads=32, kv=8, dim=128, rot=128, pairs=False, dtype="bf16"),
        # prompts of unequal lengths, half of the channels rotated, neighbours as pairs
        dict(name="append prompts fp32", op="append", seqs=9, rows=1000, ctx=100, heads=16, kv=4, dim=64, rot=32, pairs=True, dtype="fp32"),
        # a single stream with a long past: the long axis has to be split
        dict(name="attend one stream", op="attend", seqs=1, rows=1, ctx=8001, heads=32, kv=8, dim=128, window=0, dtype="bf16"),
        # a server's batch, lengths from a page to 8192
        dict(name="attend 64 streams", op="attend", seqs=64, rows=1, ctx=8192, heads=32, kv=8, dim=128, window=0, dtype="bf16"),
        # a chunk of a prompt behind 4100 tokens
        dict(name="attend chunk", op="attend", seqs=1, rows=2048, ctx=4100, heads=32, kv=8, dim=128, window=0, dtype="bf16"),
        # a few drafted tokens a stream, a head of its own for each key head, a window, full precision
        dict(name="attend drafts fp32", op="attend", seqs=6, rows=5, ctx=2000, heads=12, kv=12, dim=64, window=700, dtype="fp32"),
        # projection of one token whose norm left eight bits
        dict(name="matvec one token", op="matvec", rows=1, n=4096, k=4096, wgroup=128, dtype="bf16", xgroup=128, gate=False),
        # gated hidden layer for 16 streams
        dict(name="matvec gated 16", op="matvec", rows=16, n=22016, k=4096, wgroup=128, dtype="bf16", xgroup=0, gate=True),
        # VGG-16's first classifier layer with 4-bit weights, full precision around them
        dict(name="matvec classifier fp32", op="matvec", rows=1, n=4096, k=25088, wgroup=64, dtype="fp32", xgroup=0, gate=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "append", "attend", "attend", "matvec", "matvec"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "norm":
        group = rng.choice([0, 0, 32, 64, 128])
        rows = _log(rng, 1, 8192)
        width = _log(rng, 64, min(16384, 8192 * 4096 // rows))
        return dict(op=op, rows=rows, width=max(width // group * group, group) if group else width, dtype=dtype, res=rng.random() < 0.5, group=group)
    kv = rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
    dim = rng.choice([64, 128, 128, 256])
    if op == "append":
        rows = rng.choice([1, 1, _log(rng, 2, 2000)])
        seqs = _log(rng, 1, max(1, min(64, 2_000_000 // (rows * heads * dim))))
        rot = dim // rng.choice([1, 1, 2, 4])
        return dict(op=op, seqs=seqs, rows=rows, ctx=_log(rng, 1, 4000), heads=heads, kv=kv, dim=dim, rot=rot, pairs=rng.random() < 0.5, dtype=dtype)
    if op == "attend":
        if rng.random() < 0.3:  # a chunk of a prompt
            rows = _log(rng, 16, 2048)
            seqs = rng.choice([1, 1, 2, 3])
            ctx = _log(rng, rows, max(rows, min(8000, 4_000_000_000 // (rows * seqs * heads * dim) // 8)))
        else:
            rows = rng.choice([1, 1, 1, 2, 3, 5])
            seqs = _log(rng, 1, 64)
            ctx = _log(rng, rows, max(rows, min(16384, 500_000_000 // (seqs * kv * dim))))
        return dict(op=op, seqs=seqs, rows=rows, ctx=ctx, heads=heads, kv=kv, dim=dim, window=rng.choice([0, 0, 0, _log(rng, 1, 2000)]), dtype=dtype)
    wgroup = rng.choice([32, 64, 128, 128])
    xgroup = rng.choice([0, 0, 128]) if wgroup == 128 else 0
    gate = rng.random() < 0.25
    rows = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 128)])
    k = max(1, _log(rng, 256, 25088) // wgroup) * wgroup
    n = _log(rng, 32, min(32768, max(64, min(100_000_000, 1_500_000_000 // rows) // k)))
    return dict(op=op, rows=rows, n=n // 2 * 2 if gate else n, k=k, wgroup=wgroup, dtype=dtype, xgroup=xgroup, gate=gate)


# ---- eight bits -------------------------------------------------------------------------------------------------------------


def _scale_bits(most):
    """Exponent bits of the smallest power of two s with most <= 448 s (int32)."""
    return (((most.float().view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=LEAST)


def _two_to(bits):
    return (bits.to(torch.int32) << 23).view(torch.float32)


def _e8(bits):
    return bits.to(torch.uint8).view(E8)


# ---- inputs -------------------------------------------------------------------------------------------------------------------


def _lengths(case):
    """Tokens of each sequence in front of this step, and its new rows: unequal ones, the longest first."""
    s = case["seqs"]
    before = [int(case["ctx"] * (1 - i / s) ** 2) for i in range(s)]
    rows = [1 + int((case["rows"] - 1) * (1 - i * 0.618 % 1)) for i in range(s)]
    return before, rows


def _sequences(case, seed, dev):
    before, rows = _lengths(case)
    pages = [-(-(b + r) // PAGE) for b, r in zip(before, rows)]
    total = sum(pages)
    table = torch.full((len(pages), max(pages)), -1, dtype=torch.int32)
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).int()
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = order[at:at + p]
        at += p
    start = torch.tensor([0] + rows).cumsum(0).int()
    return dict(before=torch.tensor(before, dtype=torch.int32).to(dev), start=start.to(dev), table=table.to(dev), n_pages=total, n_rows=sum(rows), most_rows=max(rows),
                longest=max(b + r for b, r in zip(before, rows)))


def _cache(case, pages, g, dev):
    """Pages that earlier steps filled: normal keys and values, some heads far larger than others."""
    h, d = case["kv"], case["dim"]
    out = {}
    for name, shape, over in (("k", (pages, h, 4, BLOCK, d), (3, 4)), ("v", (pages, h, d, 4, BLOCK), (2, 4))):
        x = torch.randn(shape, generator=g, device=dev)
        x *= torch.exp2(torch.randn((1, h, 1, 1, 1), generator=g, device=dev))
        bits = _scale_bits(x.abs().amax(dim=over))
        s = _two_to(bits)
        x /= s[:, :, :, None, None] if name == "k" else s[:, :, None, :, None]
        out[name] = x.to(F8).reshape((pages, h, PAGE, d) if name == "k" else (pages, h, d, PAGE))
        out[name + "_scale"] = _e8(bits)
        del x
    return out


def _randn(shape, dtype, g, dev, scale=1.0):
    return (torch.randn(shape, generator=g, device=dev) * scale).to(dtype)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DT[case["dtype"]]
    st = {"case": case}
    if case["op"] == "norm":
        r, w, grp = case["rows"], case["width"], case["group"]
        st["x"] = _randn((r, w + 8), dt, g, dev)[:, :w]  # a slice of a wider buffer
        st["res"] = _randn((r, w), dt, g, dev, 4.0) if case["res"] else None
        st["weight"] = _randn((w,), dt, g, dev, 0.2) + 1
        st["sum"] = torch.empty((r, w), dtype=dt, device=dev) if case["res"] else None
        st["y"] = torch.empty((r, w), dtype=F8 if grp else dt, device=dev)
        st["scale"] = torch.empty((r, w // grp), dtype=E8, device=dev) if grp else None
    elif case["op"] == "append":
        st.update(_sequences(case, seed, dev))
        st.update(_cache(case, st["n_pages"], g, dev))
        h, hk, d, rot, n = case["heads"], case["kv"], case["dim"], case["rot"], st["n_rows"]
        qkv = _randn((n, h + 2 * hk, d), dt, g, dev, 1.5)  # what one product leaves
        st["q"], st["new_k"], st["new_v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        st["q_out"] = torch.empty((n, h, d), dtype=dt, device=dev)
        at = torch.arange(st["longest"], dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        st["turn"] = torch.cat([at.cos(), at.sin()], 1).float().to(dev)
    elif case["op"] == "attend":
        st.update(_sequences(case, seed, dev))
        st.update(_cache(case, st["n_pages"], g, dev))
        st["q"] = _randn((st["n_rows"], case["heads"], case["dim"]), dt, g, dev, 1.5)
        st["out"] = torch.empty_like(st["q"])
    else:
        r, n, k = case["rows"], case["n"], case["k"]
        st["w"] = torch.randint(0, 256, (n, k // 2), generator=g, device=dev, dtype=torch.uint8)
        st["w_scale"] = (torch.rand((n, k // case["wgroup"]), generator=g, device=dev) * 0.02 + 0.002).bfloat16()
        x = _randn((r, k), dt, g, dev)
        if case["xgroup"]:
            x = x.float().view(r, -1, case["xgroup"])
            bits = _scale_bits(x.abs().amax(2))
            st["x_scale"] = _e8(bits)
            x = (x / _two_to(bits)[:, :, None]).to(F8).view(r, k)
        st["x"] = x
        st["y"] = torch.empty((r, n // 2 if case["gate"] else n), dtype=dt, device=dev)
    if own:
        st["plan"] = _plan(st)
    return st


# ---- the library's side -----------------------------------------------------------------------------------------------------


_part = None


def _plan(st):
    """The operator as a program keeps it from step to step: a descriptor that names its buffers."""
    global _part
    import paper_2504_08795_amd as D
    if _part is None:
        D.daris_init(0, 0, 0)
        _part = D.daris_create_partition(256)
    c = st["case"]
    if c["op"] == "norm":
        op = D.make_norm(st["x"], st["weight"], st["y"], EPS, res=st["res"], sum=st["sum"], scale=st["scale"])
    elif c["op"] == "matvec":
        op = D.make_matvec(st["x"], st["w"], st["w_scale"], st["y"], x_scale=st.get("x_scale"), gate=c["gate"])
    else:
        cache = D.make_cache(st["k"], st["v"], st["k_scale"], st["v_scale"], st["table"], st["before"])
        if c["op"] == "append":
            op = D.make_append(cache, st["new_k"], st["new_v"], row_start=st["start"], q=st["q"], q_out=st["q_out"], turn=st["turn"], rot_dim=c["rot"], pairs=c["pairs"])
        else:
            op = D.make_attend(cache, st["q"], st["out"], row_start=st["start"], scale=c["dim"] ** -0.5, window=c["window"])
    return D.make_ops([op])


def _run_own(st):
    import paper_2504_08795_amd as D
    D.daris_run_ops(st["plan"], _part)
    return _outputs(st)


def _outputs(st):
    names = {"norm": ("sum", "y", "scale"), "append": ("q_out", "k", "v", "k_scale", "v_scale"), "attend": ("out",), "matvec": ("y",)}[st["case"]["op"]]
    return {n: st[n] for n in names if st[n] is not None}


# ---- the plain forms --------------------------------------------------------------------------------------------------------


def _norm(st):
    c = st["case"]
    h = st["x"].float()
    out = {}
    if c["res"]:
        h = h + st["res"].float()
        out["sum"] = h.to(DT[c["dtype"]])
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * st["weight"].float()
    if not c["group"]:
        return {**out, "y": y.to(DT[c["dtype"]])}
    y = y.view(c["rows"], -1, c["group"])
    bits = _scale_bits(y.abs().amax(2))
    return {**out, "y": (y / _two_to(bits)[:, :, None]).to(F8).view(c["rows"], -1), "scale": _e8(bits)}


def _rows(st):
    """Sequence, place in it and position of every row."""
    start = st["start"].long()
    seq = torch.repeat_interleave(torch.arange(len(start) - 1, device=start.device), start[1:] - start[:-1], output_size=st["n_rows"])
    i = torch.arange(st["n_rows"], device=start.device) - start[seq]
    return seq, i, st["before"].long()[seq] + i


def _turned(x, table, pos, rot, pairs):
    x = x.float()
    c, s = table[pos, None, :rot // 2], table[pos, None, rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if pairs else torch.cat([u, v], -1), x[..., rot:]], -1)


def _append(st):
    c = st["case"]
    n, hk, d = st["n_rows"], c["kv"], c["dim"]
    seq, _, pos = _rows(st)
    page, block, slot = st["table"][seq, pos // PAGE].long(), pos % PAGE // BLOCK, pos % BLOCK
    first = pos - slot  # where the row's block begins
    old = (st["before"].long()[seq] - first).clamp(0, BLOCK)  # tokens that the block held before this step
    new = {"k": _turned(st["new_k"], st["turn"], pos, c["rot"], c["pairs"]), "v": st["new_v"].float()}
    slots = torch.arange(BLOCK, device=pos.device)
    for name, x in new.items():
        codes = st[name].view(torch.uint8)
        codes = codes.view(-1, hk, 4, BLOCK, d) if name == "k" else codes.view(-1, hk, d, 4, BLOCK)
        bits = st[name + "_scale"].view(torch.uint8)
        where = (page * 4 + block)[:, None].expand(n, hk)
        most = torch.zeros((st["n_pages"] * 4, hk), device=x.device).scatter_reduce(0, where, x.abs().amax(2), "amax")
        had = torch.where(old[:, None] > 0, bits[page, :, block].int(), LEAST)
        now = torch.maximum(had, _scale_bits(most)[page * 4 + block])
        s = _two_to(now)
        shrink = _two_to(had) / s
        if name == "k":  # the block's earlier tokens under its new scale, then the new ones
            held = codes[page, :, block]
            held = torch.where((slots < old[:, None])[:, None, :, None], (held.view(F8).float() * shrink[:, :, None, None]).to(F8).view(torch.uint8), held)
            codes[page, :, block] = held
            codes[page, :, block, slot] = (x / s[:, :, None]).to(F8).view(torch.uint8)
        else:
            held = codes[page, :, :, block]
            held = torch.where((slots < old[:, None])[:, None, None, :], (held.view(F8).float() * shrink[:, :, None, None]).to(F8).view(torch.uint8), held)
            codes[page, :, :, block] = held
            codes[page, :, :, block, slot] = (x / s[:, :, None]).to(F8).view(torch.uint8)
        bits[page, :, block] = now.to(torch.uint8)
    q = _turned(st["q"], st["turn"], pos, c["rot"], c["pairs"]).to(DT[c["dtype"]])
    return {"q_out": q, "k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _attend(st):
    c = st["case"]
    s, n, h, hk, d = c["seqs"], st["most_rows"], c["heads"], c["kv"], c["dim"]
    dev = st["q"].device
    seq, i, pos = _rows(st)
    q = torch.zeros((s, n, h, d), device=dev)
    q[seq, i] = st["q"].float()
    at = torch.full((s, n), -1, dtype=torch.long, device=dev)
    at[seq, i] = pos
    pages = -(-st["longest"] // PAGE)
    t = st["table"][:, :pages].long().clamp(min=0)
    k = (st["k"][t].float().view(s, pages, hk, 4, BLOCK, d) * _two_to(st["k_scale"].view(torch.uint8)[t])[..., None, None]).view(s, pages, hk, PAGE, d)
    k = k.transpose(1, 2).reshape(s, hk, pages * PAGE, d)
    q = q.view(s, n, hk, h // hk, d).transpose(1, 2).reshape(s, hk, n * (h // hk), d)
    x = torch.matmul(q, k.transpose(2, 3)).view(s, hk, n, h // hk, pages * PAGE) * d ** -0.5
    del k
    token = torch.arange(pages * PAGE, device=dev)
    seen = token <= at[:, :, None]
    if c["window"]:
        seen &= token > at[:, :, None] - c["window"]
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    x = x / torch.where(total == 0, 1.0, total)
    v = (st["v"][t].float().view(s, pages, hk, d, 4, BLOCK) * _two_to(st["v_scale"].view(torch.uint8)[t])[:, :, :, None, :, None]).view(s, pages, hk, d, PAGE)
    v = v.permute(0, 2, 1, 4, 3).reshape(s, hk, pages * PAGE, d)
    y = torch.matmul(x.view(s, hk, -1, pages * PAGE), v).view(s, hk, n, h // hk, d).transpose(1, 2).reshape(s, n, h, d)
    return {"out": y[seq, i].to(DT[c["dtype"]])}


def _matvec(st):
    c = st["case"]
    w = torch.stack([st["w"] & 15, st["w"] >> 4], 2).view(c["n"], -1, c["wgroup"]).float() - 8
    w = (w * st["w_scale"].float()[:, :, None]).view(c["n"], c["k"])
    x = st["x"].float()
    if c["xgroup"]:
        x = (x.view(c["rows"], -1, c["xgroup"]) * st["x_scale"].float()[:, :, None]).view(c["rows"], -1)
    y = torch.matmul(x, w.t())
    if c["gate"]:
        a = y[:, 0::2]
        y = a / (1 + torch.exp(-a)) * y[:, 1::2]
    return {"y": y.to(DT[c["dtype"]])}


def run(st):
    if own:
        return _run_own(st)
    return {"norm": _norm, "append": _append, "attend": _attend, "matvec": _matvec}[st["case"]["op"]](st)


# ---- what an operator cannot do without --------------------------------------------------------------------------------------


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        out = n + n // case["group"] if case["group"] else n * e
        return {"bytes": n * e * (3 if case["res"] else 1) + out + case["width"] * e, "flops": 5 * n}
    if case["op"] == "matvec":
        r, n, k = case["rows"], case["n"], case["k"]
        x = r * k + r * k // case["xgroup"] if case["xgroup"] else r * k * e
        return {"bytes": n * k // 2 + n * k // case["wgroup"] * 2 + x + r * (n // 2 if case["gate"] else n) * e, "flops": 2 * r * n * k}
    h, hk, d = case["heads"], case["kv"], case["dim"]
    each = list(zip(*_lengths(case)))
    rows = sum(r for _, r in each)
    if case["op"] == "append":
        return {"bytes": rows * d * (2 * h * e + 2 * hk * (e + 1)) + rows * case["rot"] * 4, "flops": 3 * rows * (h + hk) * d}
    most = case["window"] or math.inf
    seen = sum(min(b + r, most + r - 1) for b, r in each)
    pairs = sum(min(b + (r + 1) / 2, most) * r for b, r in each)
    return {"bytes": seen * hk * (2 * d + 2 / BLOCK) + 2 * rows * h * d * e, "flops": 4 * pairs * h * d}


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------------------------


def _in_eight(x, dim):
    """x in e4m3 numbers and the powers of two that the groups along `dim` share, from the definition: 2^e >= most / 448."""
    most = x.abs().amax(dim, keepdim=True)
    s = torch.exp2(torch.ceil(torch.log2(most.clamp(min=1e-300) / 448)).clamp(min=-100))
    return (x / s).float().to(F8).double(), s


def _rotated(x, pos, rot, pairs):
    """Each pair of channels as a complex number, turned by position x 10000^(-2j/rot)."""
    j = torch.arange(rot // 2, dtype=torch.float64, device=x.device)
    angle = pos[:, None, None].double() * 10000.0 ** (-2 * j / rot)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    z = torch.complex(a, b) * torch.polar(torch.ones_like(angle), angle)
    y = x.clone()
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        h = st["x"].double()
        out = {}
        if case["res"]:
            h = h + st["res"].double()
            out["sum"] = h
        y = h / ((h ** 2).sum(1, keepdim=True) / case["width"] + EPS).sqrt() * st["weight"].double()
        if not case["group"]:
            return {**out, "y": y}
        q, s = _in_eight(y.view(case["rows"], -1, case["group"]), 2)
        return {**out, "y": q.view(case["rows"], -1), "scale": s[:, :, 0]}
    if case["op"] == "matvec":
        r, n, k = case["rows"], case["n"], case["k"]
        y = torch.empty((r, n), dtype=torch.float64, device="cuda")
        x = st["x"].double()
        if case["xgroup"]:
            x = x * st["x_scale"].double().repeat_interleave(case["xgroup"], 1)
        for lo in range(0, n, 1024):
            b = st["w"][lo:lo + 1024].short()
            w = torch.empty((b.shape[0], k), dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = (b % 16 - 8).double(), (b // 16 - 8).double()
            y[:, lo:lo + 1024] = x @ (w * st["w_scale"][lo:lo + 1024].double().repeat_interleave(case["wgroup"], 1)).t()
        return {"y": y[:, 0::2] * torch.sigmoid(y[:, 0::2]) * y[:, 1::2] if case["gate"] else y}
    start, before, table = st["start"].tolist(), st["before"].tolist(), st["table"].long()
    d, hk, g = case["dim"], case["kv"], case["heads"] // case["kv"]
    k_scale, v_scale = st["k_scale"].double(), st["v_scale"].double()
    if case["op"] == "append":
        q = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
        k, v = st["k"].double(), st["v"].double()
        for s in range(case["seqs"]):
            a, b, past = start[s], start[s + 1], before[s]
            pos = torch.arange(past, past + b - a, device="cuda")
            q[a:b] = _rotated(st["q"][a:b].double(), pos, case["rot"], case["pairs"])
            new = {"k": _rotated(st["new_k"][a:b].double(), pos, case["rot"], case["pairs"]), "v": st["new_v"][a:b].double()}
            for begin in range(past // BLOCK * BLOCK, past + b - a, BLOCK):
                page, blk = int(table[s, begin // PAGE]), begin % PAGE // BLOCK
                held, end = max(0, past - begin), min(past + b - a - begin, BLOCK)
                for name, x in new.items():
                    codes, scales = (k, k_scale) if name == "k" else (v, v_scale)
                    codes = codes[page] if name == "k" else codes[page].transpose(1, 2)
                    codes = codes[:, blk * BLOCK:blk * BLOCK + end]
                    added = x[begin + held - past:begin + end - past].transpose(0, 1)  # [head][token][channel]
                    _, least = _in_eight(added, (1, 2))
                    was = scales[page, :, blk].clone()
                    now = torch.maximum(was, least[:, 0, 0]) if held else least[:, 0, 0]
                    if held:
                        codes[:, :held] = (codes[:, :held] * (was / now)[:, None, None]).float().to(F8).double()
                    codes[:, held:] = (added / now[:, None, None]).float().to(F8).double()
                    scales[page, :, blk] = now
        return {"q_out": q, "k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for s in range(case["seqs"]):
        a, b, past = start[s], start[s + 1], before[s]
        pages = table[s, :-(-(past + b - a) // PAGE)]
        pos = torch.arange(past, past + b - a, device="cuda")
        token = torch.arange(len(pages) * PAGE, device="cuda")
        unseen = token[None] > pos[:, None]
        if case["window"]:
            unseen |= token[None] <= pos[:, None] - case["window"]
        for h in range(hk):
            k = (st["k"][pages, h].double().view(-1, 4, BLOCK, d) * k_scale[pages, h][:, :, None, None]).view(-1, d)
            v = (st["v"][pages, h].double().view(-1, d, 4, BLOCK) * v_scale[pages, h][:, None, :, None]).view(-1, d, PAGE).transpose(1, 2).reshape(-1, d)
            for j in range(h * g, (h + 1) * g):
                x = (st["q"][a:b, j].double() @ k.t() / math.sqrt(d)).masked_fill(unseen, -math.inf)
                out[a:b, j] = torch.softmax(x, 1) @ v
    return {"out": out}
