"""What is measured of the operators of a drafted step: a tree of drafted words over the paged cache, and the words that come of it.

A program that drafts words hangs them on the last word of a sequence as a tree and takes the whole tree through the model at
once: its nodes are the step's new rows, each of which sees the cached tokens and the nodes above itself.  Then a word is drawn
behind every node, the drafted words that were drawn are accepted from the root on, and the cache keeps their tokens only:

    append (tree) -> attend (tree) -> ... -> sample -> accept -> keep          and copy, where one sequence becomes two

* tree     [row][words of 64 bits]: bit j of a row is node j of its sequence, which it sees; itself and what is above it.  A node's
           position is that of the first new token and the number of nodes above it
* cache    pages of 64 tokens, keys [page][head][token][channel], values [page][head][channel][token], e4m3; 16 tokens of a head
           share a scale, the smallest power of two that leaves none of them above 448
* sample   weights exp((x - largest) / temperature), those below 2^-64 nothing; of these the top_k largest, of these the shortest
           front (largest first) with top_p of their sum, of these what has min_p of the largest; the first of them, by number,
           at which their sum passes random x total.  Equal logits: the lower number first
* accept   from node 0: the first node below the present one whose word is what was drawn behind it
* keep     the tokens of the accepted nodes one behind the other; a sixteenth that gets any has the largest scale of its tokens
* copy     whole pages

Sizes are generic (32 query heads on 8 key heads of 128, trees of a dozen to 200 nodes, vocabularies of 50001 and 131072).

`own` says which side ``run`` takes: elementary torch operations, or the library's calls.
"""
import math

import numpy as np
import torch

own = False

PAGE, BLOCK = 64, 16
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
LEAST = 27  # exponent bits of the smallest scale, 2^-100


def listed():
    return [
        # a dozen nodes of one stream, a window, full precision, heads of their own size: latency
        dict(name="tree attend one stream fp32", op="attend", seqs=1, rows=13, ctx=2000, heads=12, kv=4, dim=64, window=700, dtype="fp32"),
        # a server's batch, trees of up to 64 nodes behind up to 4096 tokens
        dict(name="tree attend 32 streams", op="attend", seqs=32, rows=64, ctx=4096, heads=32, kv=8, dim=128, window=0, dtype="bf16"),
        # one stream's tree into the cache
        dict(name="tree append one stream", op="append", seqs=1, rows=26, ctx=1000, heads=32, kv=8, dim=128, rot=128, pairs=False, dtype="bf16"),
        # trees of unequal sizes, a quarter of the channels turned, neighbours as pairs
        dict(name="tree append 48 streams fp32", op="append", seqs=48, rows=61, ctx=3000, heads=16, kv=4, dim=64, rot=32, pairs=True, dtype="fp32"),
        # a word of one stream from a vocabulary of odd size, the 40 likeliest
        dict(name="sample one row fp32", op="sample", rows=1, n=50001, dtype="fp32", mode="top_k"),
        # a word behind each of 64 nodes, every stream with wishes of its own
        dict(name="sample 64 rows", op="sample", rows=64, n=131072, dtype="bf16", mode="mixed"),
        # the walk down one small tree
        dict(name="accept one stream", op="accept", seqs=1, rows=26),
        # ... down many large ones
        dict(name="accept 512 streams", op="accept", seqs=512, rows=200),
        # five words of a tree stay
        dict(name="keep one stream", op="keep", seqs=1, rows=26, kept=5, ctx=1000, kv=8, dim=128),
        # up to nine words of each stream stay
        dict(name="keep 64 streams", op="keep", seqs=64, rows=64, kept=9, ctx=2000, kv=8, dim=128),
        # the last, partly filled page of a sequence that is continued twice
        dict(name="copy one page", op="copy", pages=1, kv=8, dim=128),
        # pages gathered at one end of the cache
        dict(name="copy 1001 pages", op="copy", pages=1001, kv=8, dim=128),
    ]


MODES = ("mixed", "greedy", "all", "top_k", "top_p", "min_p")


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "sample", "sample", "accept", "keep", "copy"])
    if op == "accept":
        rows = _log(rng, 1, 256)
        return dict(op=op, seqs=_log(rng, 1, min(2000, 100_000 // rows)), rows=rows)
    if op == "sample":
        rows = _log(rng, 1, 256)
        return dict(op=op, rows=rows, n=_log(rng, 100, min(200_000, 64 * 131072 // rows)), dtype=rng.choice(["bf16", "fp32"]), mode=rng.choice(MODES))
    kv = rng.choice([1, 2, 4, 8, 12])
    dim = rng.choice([64, 128, 128, 256])
    if op == "copy":
        return dict(op=op, pages=_log(rng, 1, 1001 * 1024 // (kv * dim)), kv=kv, dim=dim)
    if op == "keep":
        rows = _log(rng, 2, 256)
        ctx = _log(rng, 1, 4000)
        return dict(op=op, seqs=_log(rng, 1, max(1, min(64, 134_000_000 // (ctx * kv * dim)))), rows=rows, kept=_log(rng, 1, min(rows, 24)), ctx=ctx, kv=kv, dim=dim)
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    rows = _log(rng, 2, 256)
    if op == "append":
        seqs = _log(rng, 1, max(1, min(64, 4_000_000 // (rows * heads * dim))))
        return dict(op=op, seqs=seqs, rows=rows, ctx=_log(rng, 1, 3000), heads=heads, kv=kv, dim=dim, rot=dim // rng.choice([1, 1, 2, 4]), pairs=rng.random() < 0.5, dtype=dtype)
    seqs = _log(rng, 1, 64)
    ctx = _log(rng, 1, max(1, min(8192, 134_000_000 // (seqs * kv * dim), 30_000_000_000 // (seqs * rows * heads * dim))))
    rows = max(2, min(rows, 8_000_000 // (seqs * heads * dim), 30_000_000_000 // (seqs * heads * dim * ctx)))
    return dict(op=op, seqs=seqs, rows=rows, ctx=ctx, heads=heads, kv=kv, dim=dim, window=rng.choice([0, 0, 0, _log(rng, 1, 2000)]), dtype=dtype)


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
    """Cached tokens of each sequence and the nodes of its tree: unequal ones, the longest first."""
    s = case["seqs"]
    before = [int(case.get("ctx", 0) * (1 - i / s)) for i in range(s)]
    rows = [1 + int((case["rows"] - 1) * (1 - i * 0.618 % 1)) for i in range(s)]
    return before, rows


def _kept(case):
    return [max(1, min(1 + int((case["kept"] - 1) * (1 - i * 0.382 % 1)), r - 1)) for i, r in enumerate(_lengths(case)[1])]


def _trees(rows, rng):
    """A tree for each sequence, every node below one of the eight in front of it: parents and masks of all rows."""
    s, n = len(rows), max(rows)
    words = -(-n // 64)
    parent = np.full((s, n), -1, np.int64)
    mask = np.zeros((s, n, words), np.uint64)
    at = np.arange(s)
    for i in range(n):
        if i:
            parent[:, i] = i - 1 - np.minimum(rng.integers(0, 8, s), i - 1)
            mask[:, i] = mask[at, parent[:, i]]
        mask[:, i, i // 64] |= np.uint64(1 << (i % 64))
    there = np.arange(n)[None] < np.array(rows)[:, None]
    return parent[there], np.ascontiguousarray(mask[there]).view(np.int64)


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
    parent, mask = _trees(rows, np.random.default_rng(seed))
    start = torch.tensor([0] + rows).cumsum(0).int()
    return dict(before=torch.tensor(before, dtype=torch.int32).to(dev), start=start.to(dev), table=table.to(dev), n_pages=total, n_rows=sum(rows), most_rows=max(rows),
                longest=max(b + r for b, r in zip(before, rows)), tree=torch.from_numpy(mask).to(dev)), parent


def _cache(case, pages, g, dev):
    """Pages that earlier steps filled: normal keys and values, some heads far larger than others."""
    h, d = case["kv"], case["dim"]
    out = {}
    for name, shape, over in (("k", (pages, h, 4, BLOCK, d), (3, 4)), ("v", (pages, h, d, 4, BLOCK), (2, 4))):
        x = torch.randn(shape, generator=g, device=dev)
        x *= torch.exp2(torch.randn((1, h, 1, 1, 1), generator=g, device=dev))
        if case["op"] != "attend":  # sixteenths of unequal scales, as single large tokens leave them
            x *= torch.exp2(torch.randint(-1, 2, (pages, h, 4), generator=g, device=dev).float()).view((pages, h, 4, 1, 1) if name == "k" else (pages, h, 1, 4, 1))
        bits = _scale_bits(x.abs().amax(dim=over))
        s = _two_to(bits)
        x /= s[:, :, :, None, None] if name == "k" else s[:, :, None, :, None]
        out[name] = x.to(F8).reshape((pages, h, PAGE, d) if name == "k" else (pages, h, d, PAGE))
        out[name + "_scale"] = _e8(bits)
        del x
    return out


def _randn(shape, dtype, g, dev, scale=1.0):
    return (torch.randn(shape, generator=g, device=dev) * scale).to(dtype)


def _logits(case, g, dev):
    """Rows of a model's answers: a bulk, a few words far above it, and in some rows words that the program forbids."""
    r, n = case["rows"], case["n"]
    x = torch.randn((r, n), generator=g, device=dev) * (1 + 2 * torch.rand((r, 1), generator=g, device=dev))
    few = torch.randint(0, n, (r, 24), generator=g, device=dev)
    x.scatter_add_(1, few, torch.rand((r, 24), generator=g, device=dev) * 12)
    banned = (torch.rand((r, 1), generator=g, device=dev) < 0.25) & (torch.rand((r, n), generator=g, device=dev) < 0.5)
    return x.masked_fill_(banned, -math.inf).to(DT[case["dtype"]])


def _wishes(case, rng, dev):
    """Temperature, top_k, top_p and min_p of each row."""
    r, mode = case["rows"], case["mode"]
    kinds = [MODES[1:][i % 5] if mode == "mixed" else mode for i in range(r)]
    pick = lambda kind, among, none: [rng.choice(among) if k == kind else none for k in kinds]  # noqa: E731
    out = {
        "temperature": torch.tensor([0.0 if k == "greedy" else round(float(rng.uniform(0.5, 1.2)), 2) for k in kinds]),
        "top_k": torch.tensor(pick("top_k", [40] if r == 1 else [1, 5, 40, 1000], 0), dtype=torch.int32),
        "top_p": torch.tensor(pick("top_p", [0.5, 0.9, 0.95], 1.0), dtype=torch.float32),
        "min_p": torch.tensor(pick("min_p", [0.02, 0.1], 0.0), dtype=torch.float32),
    }
    if mode == "mixed":  # one row with all of them
        out["top_k"][-1], out["top_p"][-1], out["min_p"][-1] = 200, 0.9, 0.01
    return {k: v.to(dev) for k, v in out.items()}


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = np.random.default_rng(seed)
    st = {"case": case}
    op = case["op"]
    if op in ("attend", "append", "keep"):
        more, _ = _sequences(case, seed, dev)
        st.update(more)
        st.update(_cache(case, st["n_pages"], g, dev))
    if op == "attend":
        st["q"] = _randn((st["n_rows"], case["heads"], case["dim"]), DT[case["dtype"]], g, dev, 1.5)
        st["out"] = torch.empty_like(st["q"])
    elif op == "append":
        h, hk, d, rot, n = case["heads"], case["kv"], case["dim"], case["rot"], st["n_rows"]
        qkv = _randn((n, h + 2 * hk, d), DT[case["dtype"]], g, dev, 1.5)  # what one product leaves
        st["q"], st["new_k"], st["new_v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        st["q_out"] = torch.empty((n, h, d), dtype=DT[case["dtype"]], device=dev)
        at = torch.arange(st["longest"], dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        st["turn"] = torch.cat([at.cos(), at.sin()], 1).float().to(dev)
    elif op == "keep":
        path = np.full(st["n_rows"], -1, np.int32)
        at = 0
        for r, c in zip(_lengths(case)[1], _kept(case)):
            path[at] = 0
            if c > 1:
                path[at + 1:at + c] = np.sort(rng.choice(np.arange(min(2, r - c + 1), r), c - 1, replace=False))
            at += r
        st["path"], st["count"] = torch.from_numpy(path).to(dev), torch.tensor(_kept(case), dtype=torch.int32).to(dev)
    elif op == "accept":
        more, parent = _sequences(case, seed, dev)
        st.update(more)
        n = st["n_rows"]
        first = np.repeat(more["start"].cpu().numpy()[:-1], _lengths(case)[1])
        words, answers = rng.integers(0, 30000, n), rng.integers(0, 30000, n)
        drawn = (parent >= 0) & (rng.random(n) < 0.7)  # the word of one of the nodes below
        answers[(first + parent)[drawn]] = words[drawn]
        st["words"], st["answers"] = torch.from_numpy(words.astype(np.int32)).to(dev), torch.from_numpy(answers.astype(np.int32)).to(dev)
        st["path"] = torch.empty(n, dtype=torch.int32, device=dev)
        st["count"], st["word"], st["after"] = (torch.empty(case["seqs"], dtype=torch.int32, device=dev) for _ in range(3))
    elif op == "sample":
        st["logits"] = _logits(case, g, dev)
        st.update(_wishes(case, rng, dev))
        st["random"] = torch.rand(case["rows"], generator=g, device=dev)
        st["word"] = torch.empty(case["rows"], dtype=torch.int32, device=dev)
        st["chance"] = torch.empty(case["rows"], dtype=torch.float32, device=dev)
    else:
        n = case["pages"]
        st["n_pages"] = 2 * n + 1
        st.update(_cache(case, st["n_pages"], g, dev))
        order = torch.from_numpy(rng.permutation(2 * n + 1)[:2 * n].astype(np.int32))
        st["pairs"] = order.view(n, 2).contiguous().to(dev)
        st["table"], st["before"] = torch.arange(st["n_pages"], dtype=torch.int32, device=dev)[None], torch.zeros(1, dtype=torch.int32, device=dev)
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
    if c["op"] == "sample":
        op = D.make_sample(st["logits"], st["word"], st["random"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"], chance=st["chance"])
    elif c["op"] == "accept":
        op = D.make_accept(st["tree"], st["words"], st["answers"], st["path"], st["count"], st["word"], row_start=st["start"], before=st["before"], after=st["after"])
    else:
        cache = D.make_cache(st["k"], st["v"], st["k_scale"], st["v_scale"], st["table"], st["before"])
        if c["op"] == "append":
            op = D.make_append(cache, st["new_k"], st["new_v"], row_start=st["start"], q=st["q"], q_out=st["q_out"], turn=st["turn"], rot_dim=c["rot"], pairs=c["pairs"], tree=st["tree"])
        elif c["op"] == "attend":
            op = D.make_attend(cache, st["q"], st["out"], row_start=st["start"], scale=c["dim"] ** -0.5, window=c["window"], tree=st["tree"])
        elif c["op"] == "keep":
            op = D.make_keep(cache, st["path"], st["count"], row_start=st["start"])
        else:
            op = D.make_copy(cache, st["pairs"])
    return D.make_ops([op])


def _run_own(st):
    import paper_2504_08795_amd as D
    D.daris_run_ops(st["plan"], _part)
    names = {"attend": ("out",), "append": ("q_out", "k", "v", "k_scale", "v_scale"), "sample": ("word", "chance"), "accept": ("path", "count", "word", "after")}
    return {n: st[n] for n in names.get(st["case"]["op"], ("k", "v", "k_scale", "v_scale"))}


# ---- the plain forms --------------------------------------------------------------------------------------------------------


def _rows(st):
    """Sequence, node and place in the cache of every row."""
    start = st["start"].long()
    seq = torch.repeat_interleave(torch.arange(len(start) - 1, device=start.device), start[1:] - start[:-1], output_size=st["n_rows"])
    i = torch.arange(st["n_rows"], device=start.device) - start[seq]
    return seq, i, st["before"].long()[seq] + i


def _bits(st):
    """The masks as truth values [row][node]."""
    t = st["tree"]
    return ((t[:, :, None] >> torch.arange(64, device=t.device)) & 1).bool().flatten(1)


def _turned(x, table, pos, rot, pairs):
    x = x.float()
    c, s = table[pos, None, :rot // 2], table[pos, None, rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if pairs else torch.cat([u, v], -1), x[..., rot:]], -1)


def _append(st):
    c = st["case"]
    n, hk, d = st["n_rows"], c["kv"], c["dim"]
    seq, _, at = _rows(st)
    pos = st["before"].long()[seq] + _bits(st).sum(1) - 1  # where the row stands in its sequence, beside where its token lies
    page, block, slot = st["table"][seq, at // PAGE].long(), at % PAGE // BLOCK, at % BLOCK
    old = (st["before"].long()[seq] - (at - slot)).clamp(0, BLOCK)  # tokens that the block held before this step
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
    seq, i, _ = _rows(st)
    q = torch.zeros((s, n, h, d), device=dev)
    q[seq, i] = st["q"].float()
    pages = -(-st["longest"] // PAGE)
    token = torch.arange(pages * PAGE, device=dev)
    bits = _bits(st)
    # tokens that a row sees: those of the cache, then the nodes of its mask; under a window the last of these
    node = token - st["before"].long()[seq, None]
    sees = torch.where(node < 0, True, bits.gather(1, node.clamp(0, bits.shape[1] - 1)) & (node < bits.shape[1]))
    if c["window"]:
        sees &= torch.cumsum(sees, 1) > sees.sum(1, keepdim=True) - c["window"]
    seen = torch.zeros((s, n, pages * PAGE), dtype=torch.bool, device=dev)
    seen[seq, i] = sees
    t = st["table"][:, :pages].long().clamp(min=0)
    k = (st["k"][t].float().view(s, pages, hk, 4, BLOCK, d) * _two_to(st["k_scale"].view(torch.uint8)[t])[..., None, None]).view(s, pages, hk, PAGE, d)
    k = k.transpose(1, 2).reshape(s, hk, pages * PAGE, d)
    q = q.view(s, n, hk, h // hk, d).transpose(1, 2).reshape(s, hk, n * (h // hk), d)
    x = torch.matmul(q, k.transpose(2, 3)).view(s, hk, n, h // hk, pages * PAGE) * d ** -0.5
    del k
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    x = x / torch.where(total == 0, 1.0, total)
    v = (st["v"][t].float().view(s, pages, hk, d, 4, BLOCK) * _two_to(st["v_scale"].view(torch.uint8)[t])[:, :, :, None, :, None]).view(s, pages, hk, d, PAGE)
    v = v.permute(0, 2, 1, 4, 3).reshape(s, hk, pages * PAGE, d)
    y = torch.matmul(x.view(s, hk, -1, pages * PAGE), v).view(s, hk, n, h // hk, d).transpose(1, 2).reshape(s, n, h, d)
    return {"out": y[seq, i].to(DT[c["dtype"]])}


def _sample(st):
    r, n = st["logits"].shape
    x = st["logits"].double()  # in 64 bits: a word changes where a sum passes the random number by a last bit
    top = x.amax(1, keepdim=True)
    t = st["temperature"].double()[:, None]
    greedy = t <= 0
    w = torch.where(x == top, 1.0, torch.exp((x - top) / torch.where(greedy, 1.0, t)))
    w = torch.where((w >= 2.0 ** -64) & (x > -math.inf), w, 0.0)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    rank = torch.arange(n, device=x.device)
    k = torch.where(greedy[:, 0], 1, torch.where(st["top_k"] > 0, st["top_k"].long(), n))[:, None]
    s = torch.where(rank < k, w.gather(1, order), 0.0)
    in_front = torch.cumsum(s, 1)
    need = torch.where(st["top_p"] < 1, st["top_p"].double(), 2.0)[:, None] * in_front[:, -1:]
    in_front = torch.cat([torch.zeros_like(need), in_front[:, :-1]], 1)
    s = torch.where(((in_front < need) & (s >= st["min_p"].double()[:, None])) | (rank == 0), s, 0.0)
    w = torch.zeros_like(w).scatter(1, order, s)
    upto = torch.cumsum(w, 1)
    total = upto[:, -1:]
    last = (n - 1 - torch.argmax((w.flip(1) > 0).int(), 1)).clamp(min=0)
    word = torch.minimum((upto <= st["random"].double()[:, None] * total).sum(1), last)
    none = total[:, 0] == 0
    chance = w.gather(1, word[:, None])[:, 0] / torch.where(none, 1.0, total[:, 0])
    return {"word": torch.where(none, -1, word).int(), "chance": chance.float()}


def _accept(st):
    seq, i, _ = _rows(st)
    first = st["start"].long()[seq]
    n, s = st["n_rows"], st["case"]["seqs"]
    bits = _bits(st)
    node = torch.arange(bits.shape[1], device=i.device)
    above = bits & (node < i[:, None])
    parent = torch.where(above, node, -1).amax(1)
    up = first + parent.clamp(min=0)
    fits = (parent >= 0) & (st["answers"][up] >= 0) & (st["words"] == st["answers"][up])
    child = torch.full((n,), n, dtype=torch.long, device=i.device).scatter_reduce(0, up, torch.where(fits, i, n), "amin")  # the first node below that fits
    good = (i == 0) | (fits & (child[up] == i))
    good_of = torch.zeros((s, bits.shape[1]), dtype=torch.bool, device=i.device)
    good_of[seq, i] = good
    on = good & ((i == 0) | (above[:, 0] & ~(above & ~good_of[seq]).any(1)))  # it and everything above it
    count = torch.zeros(s, dtype=torch.long, device=i.device).scatter_add(0, seq, on.long())
    place = torch.cumsum(on, 0)
    place = first + place - place[first]  # (the root is on)
    path = torch.full((n + 1,), -1, dtype=torch.int32, device=i.device)
    path[torch.where(on, place, n)] = i.int()
    path = path[:n]
    last = st["start"].long()[:-1] + path[st["start"].long()[:-1] + count - 1]
    return {"path": path, "count": count.int(), "word": st["answers"][last], "after": st["before"] + count.int()}


def _keep(st):
    c = st["case"]
    hk, d = c["kv"], c["dim"]
    seq, j, to = _rows(st)
    moved = (j < st["count"].long()[seq]) & (st["path"] != j)
    seq, j, to, node = seq[moved], j[moved], to[moved], st["path"].long()[moved]
    at = to - j + node
    page = lambda t: st["table"][seq, t // PAGE].long()  # noqa: E731
    from_page, to_page = page(at), page(to)
    f_block, f_slot, block, slot = at % PAGE // BLOCK, at % BLOCK, to % PAGE // BLOCK, to % BLOCK
    where = to_page * 4 + block
    n = st["n_pages"] * 4
    first = torch.full((n,), BLOCK, dtype=torch.long, device=to.device).scatter_reduce(0, where, slot, "amin")  # tokens of the block that stay
    # (a sequence's first kept token always stays; in its first block so does what lies in front of the first that moves)
    stay = first[where]
    slots = torch.arange(BLOCK, device=to.device)
    for name in ("k", "v"):
        codes = st[name].view(torch.uint8)
        codes = codes.view(-1, hk, 4, BLOCK, d) if name == "k" else codes.view(-1, hk, d, 4, BLOCK)
        bits = st[name + "_scale"].view(torch.uint8)
        had, came = bits[to_page, :, block].int(), bits[from_page, :, f_block].int()
        most = torch.zeros((n, hk), dtype=torch.int32, device=to.device).scatter_reduce(0, where[:, None].expand(-1, hk), came, "amax")
        now = torch.maximum(torch.where(stay[:, None] > 0, had, 0), most[where])
        shrink, turn = _two_to(had) / _two_to(now), _two_to(came) / _two_to(now)
        if name == "k":
            x = (codes[from_page, :, f_block, f_slot].view(F8).float() * turn[:, :, None]).to(F8).view(torch.uint8)
            held = codes[to_page, :, block]
            held = torch.where((slots < stay[:, None])[:, None, :, None], (held.view(F8).float() * shrink[:, :, None, None]).to(F8).view(torch.uint8), held)
            codes[to_page, :, block] = held
            codes[to_page, :, block, slot] = x
        else:
            x = (codes[from_page, :, :, f_block, f_slot].view(F8).float() * turn[:, :, None]).to(F8).view(torch.uint8)
            held = codes[to_page, :, :, block]
            held = torch.where((slots < stay[:, None])[:, None, None, :], (held.view(F8).float() * shrink[:, :, None, None]).to(F8).view(torch.uint8), held)
            codes[to_page, :, :, block] = held
            codes[to_page, :, :, block, slot] = x
        bits[to_page, :, block] = now.to(torch.uint8)
    return {"k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _copy(st):
    at, to = st["pairs"].long().unbind(1)
    for name in ("k", "v", "k_scale", "v_scale"):
        x = st[name].view(torch.uint8)
        x[to] = x[at]
    return {"k": st["k"], "v": st["v"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def run(st):
    if own:
        return _run_own(st)
    return {"attend": _attend, "append": _append, "sample": _sample, "accept": _accept, "keep": _keep, "copy": _copy}[st["case"]["op"]](st)


# ---- what an operator cannot do without --------------------------------------------------------------------------------------


def work(case):
    op = case["op"]
    if op == "copy":
        return {"bytes": 2 * case["pages"] * case["kv"] * (2 * PAGE * case["dim"] + 8), "flops": 0}
    if op == "sample":
        return {"bytes": case["rows"] * (case["n"] * (2 if case["dtype"] == "bf16" else 4) + 28), "flops": 4 * case["rows"] * case["n"]}
    each = list(zip(*_lengths(case)))
    rows, words = sum(r for _, r in each), -(-case["rows"] // 64)
    if op == "accept":
        return {"bytes": rows * (8 * words + 12) + 20 * case["seqs"], "flops": rows}
    if op == "keep":
        moved = sum(_kept(case)) - case["seqs"]
        return {"bytes": 2 * moved * case["kv"] * 2 * case["dim"] + 8 * case["seqs"], "flops": 2 * moved * case["kv"] * case["dim"]}
    h, hk, d = case["heads"], case["kv"], case["dim"]
    e = 2 if case["dtype"] == "bf16" else 4
    if op == "append":
        return {"bytes": rows * d * (2 * h * e + 2 * hk * (e + 1)) + rows * (case["rot"] * 4 + 8 * words), "flops": 3 * rows * (h + hk) * d}
    most = case["window"] or math.inf
    seen = sum(min(b, most) + r for b, r in each)
    pairs = sum(min(b + math.log2(1 + r), most) * r for b, r in each)  # (a node of n sees a few of the others)
    return {"bytes": seen * hk * (2 * d + 2 / BLOCK) + 2 * rows * h * d * e + 8 * words * rows, "flops": 4 * pairs * h * d}


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


def _ancestors(case, seed):
    """Lists of the nodes from the root to every row, and the parents."""
    rows = _lengths(case)[1]
    parent, _ = _trees(rows, np.random.default_rng(seed))
    lines, at = [], 0
    for r in rows:
        own_lines = []
        for i in range(r):
            own_lines.append((own_lines[parent[at + i]] if i else []) + [i])
        lines.append(own_lines)
        at += r
    return lines


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "sample":
        return _exact_sample(st)
    if op == "copy":
        out = {n: st[n].double() for n in ("k", "v", "k_scale", "v_scale")}
        for x in out.values():
            x[st["pairs"][:, 1].long()] = x[st["pairs"][:, 0].long()]
        return out
    start, before, table = st["start"].tolist(), st["before"].tolist(), st["table"].long()
    if op == "accept":
        return _exact_accept(st, start, before, _ancestors(case, seed))
    k_scale, v_scale = st["k_scale"].double(), st["v_scale"].double()
    d, hk = case["dim"], case["kv"]
    if op == "keep":
        k, v = st["k"].double(), st["v"].double()
        path, count = st["path"].tolist(), st["count"].tolist()
        tbl = table.tolist()
        for s in range(case["seqs"]):
            line, b = path[start[s]:start[s] + count[s]], before[s]
            if all(i == j for j, i in enumerate(line)):
                continue
            moved = [j for j, i in enumerate(line) if i != j]
            held = {b + j: b + i for j, i in enumerate(line)}  # place -> where its token is now
            for codes, scales, by in ((k, k_scale, 2), (v, v_scale, 3)):
                value = {}
                for to, at in held.items():
                    page, blk = tbl[s][at // PAGE], at % PAGE // BLOCK
                    value[to] = codes[page].select(by - 1, at % PAGE) * scales[page, :, blk, None], scales[page, :, blk].clone()
                for begin in range((b + moved[0]) // BLOCK * BLOCK, b + count[s], BLOCK):
                    page, blk = tbl[s][begin // PAGE], begin % PAGE // BLOCK
                    for t in range(begin, b):  # tokens of the cache in front of the step's
                        value[t] = codes[page].select(by - 1, t % PAGE) * scales[page, :, blk, None], scales[page, :, blk].clone()
                    tokens = [t for t in range(begin, min(begin + BLOCK, b + count[s]))]
                    now = torch.stack([value[t][1] for t in tokens]).amax(0)
                    for t in tokens:
                        codes[page].select(by - 1, t % PAGE).copy_((value[t][0] / now[:, None]).float().to(F8).double())
                    scales[page, :, blk] = now
        return {"k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale}
    lines = _ancestors(case, seed)
    if op == "append":
        q = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
        k, v = st["k"].double(), st["v"].double()
        for s in range(case["seqs"]):
            a, b, past = start[s], start[s + 1], before[s]
            pos = past + torch.tensor([len(line) - 1 for line in lines[s]], device="cuda")
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
    g = case["heads"] // hk
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for s in range(case["seqs"]):
        a, b, past = start[s], start[s + 1], before[s]
        pages = table[s, :-(-(past + b - a) // PAGE)]
        unseen = torch.ones((b - a, len(pages) * PAGE), dtype=torch.bool)
        for i, line in enumerate(lines[s]):
            tokens = np.array(list(range(past)) + [past + node for node in line])
            unseen[i, tokens[-case["window"]:] if case["window"] else tokens] = False
        unseen = unseen.cuda()
        for h in range(hk):
            k = (st["k"][pages, h].double().view(-1, 4, BLOCK, d) * k_scale[pages, h][:, :, None, None]).view(-1, d)
            v = (st["v"][pages, h].double().view(-1, d, 4, BLOCK) * v_scale[pages, h][:, None, :, None]).view(-1, d, PAGE).transpose(1, 2).reshape(-1, d)
            for j in range(h * g, (h + 1) * g):
                x = (st["q"][a:b, j].double() @ k.t() / math.sqrt(d)).masked_fill(unseen, -math.inf)
                out[a:b, j] = torch.softmax(x, 1) @ v
    return {"out": out}


def _exact_sample(st):
    """Row by row: the words from the largest down, until a limit is met."""
    x_all, u = st["logits"].double().cpu().numpy(), st["random"].double().cpu().numpy()
    t_all, k_all = st["temperature"].double().cpu().numpy(), st["top_k"].cpu().numpy()
    p_all, m_all = st["top_p"].double().cpu().numpy(), st["min_p"].double().cpu().numpy()
    word, chance = np.zeros(len(u), np.int32), np.zeros(len(u))
    for r, x in enumerate(x_all):
        if t_all[r] <= 0:
            word[r], chance[r] = int(np.argmax(x)), 1.0
            continue
        bits = (x - x.max()) / t_all[r] * math.log2(math.e)
        live = np.flatnonzero(bits >= -64)
        live = live[np.lexsort((live, -x[live]))]
        if k_all[r] > 0:
            live = live[:k_all[r]]
        w = np.exp2(bits[live])
        if p_all[r] < 1:
            n = 1 + int(np.searchsorted(np.cumsum(w), p_all[r] * w.sum(), side="left"))
            live, w = live[:n], w[:n]
        on = (w >= m_all[r]) | (np.arange(len(w)) == 0)
        live, w = live[on], w[on]
        order = np.argsort(live)
        live, w = live[order], w[order]
        i = min(int(np.searchsorted(np.cumsum(w), u[r] * w.sum(), side="right")), len(w) - 1)
        word[r], chance[r] = live[i], w[i] / w.sum()
    return {"word": torch.from_numpy(word), "chance": torch.from_numpy(chance)}


def _exact_accept(st, start, before, lines):
    """The walk itself."""
    words, answers = st["words"].tolist(), st["answers"].tolist()
    path, count, word = np.full(st["n_rows"], -1, np.int32), [], []
    for s, own_lines in enumerate(lines):
        a, at, line = start[s], 0, [0]
        while True:
            below = [i for i in range(at + 1, len(own_lines)) if own_lines[i][-2] == at and words[a + i] == answers[a + at]]
            if not below:
                break
            at = below[0]
            line.append(at)
        path[a:a + len(line)] = line
        count.append(len(line))
        word.append(answers[a + at])
    return {"path": torch.from_numpy(path), "count": torch.tensor(count, dtype=torch.int32), "word": torch.tensor(word, dtype=torch.int32),
            "after": torch.tensor([b + c for b, c in zip(before, count)], dtype=torch.int32)}
