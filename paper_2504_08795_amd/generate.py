"""A small generating decoder on a partition: every operator of daris_ops.h as a model runs it.

A block is norm (8 bits) -> product -> append -> attend -> product -> norm (8 bits) -> gated product -> product, with the residual taken
along by the norms.  Prompts of several streams go through it as one ragged set of rows, then each step appends one token to every
stream; a step is one list of operators, planned once.  Weights are random: this is an example and a measurement, not a model.

    python -m paper_2504_08795_amd.generate --streams 4 --prompt 100 --tokens 64 --check
"""
import argparse
import json
import time

import numpy as np
import torch

from . import binding as D

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


class Weights:
    """4-bit weights [n][k / 2] and their scales, such that products of rows of size 1 have size 1."""

    def __init__(self, n, k, group, rng):
        self.codes = torch.randint(0, 256, (n, k // 2), generator=rng, dtype=torch.uint8).cuda()
        spread = (torch.rand((n, k // group), generator=rng) * 0.5 + 0.75) / (4.6 * k ** 0.5)     # (codes - 8 have size 4.6)
        self.scales = spread.bfloat16().cuda()


class Block:
    def __init__(self, m, rng):
        heads = (m.q_heads + 2 * m.kv_heads) * m.dim
        self.norms = [torch.ones(m.width, dtype=m.dtype, device="cuda") for _ in range(2)]
        self.qkv = Weights(heads, m.width, m.group, rng)
        self.out = Weights(m.width, m.q_heads * m.dim, m.group, rng)
        self.gated = Weights(2 * m.hidden, m.width, m.group, rng)       # gate and value of a channel are neighbours
        self.down = Weights(m.width, m.hidden, m.group, rng)
        shape = (m.n_pages, m.kv_heads)
        self.k = torch.zeros(shape + (D.PAGE_TOKENS, m.dim), dtype=F8, device="cuda")
        self.v = torch.zeros(shape + (m.dim, D.PAGE_TOKENS), dtype=F8, device="cuda")
        self.k_scale, self.v_scale = (torch.zeros(shape + (D.PAGE_TOKENS // D.SCALE_TOKENS,), dtype=torch.uint8, device="cuda").view(E8) for _ in range(2))
        self.cache = D.make_cache(self.k, self.v, self.k_scale, self.v_scale, m.pages, m.before)


class Rows:
    """Buffers for `rows` rows, and the operators that take them through the blocks."""

    def __init__(self, m, rows, row_start=None):
        def make(width, dtype=m.dtype):
            return torch.zeros((rows, width), dtype=dtype, device="cuda")
        self.x = make(m.width)                                          # the residual
        self.add = make(m.width)                                        # what a block adds to it last
        self.mid = make(m.width)                                        # ... after its attention
        self.codes, self.scales = [make(m.width, F8) for _ in range(2)], [make(m.width // m.group, torch.uint8).view(E8) for _ in range(2)]
        self.qkv = make((m.q_heads + 2 * m.kv_heads) * m.dim).view(rows, -1, m.dim)
        self.seen, self.gated = make(m.q_heads * m.dim), make(m.hidden)
        q, k, v = self.qkv.split([m.q_heads, m.kv_heads, m.kv_heads], 1)
        self.ops = []
        for i, b in enumerate(m.blocks):
            first = dict(res=self.x, sum=self.x) if i else {}
            self.ops += [
                D.make_norm(self.add if i else self.x, b.norms[0], self.codes[0], m.eps, scale=self.scales[0], **first),
                D.make_matvec(self.codes[0], b.qkv.codes, b.qkv.scales, self.qkv.view(rows, -1), x_scale=self.scales[0]),
                D.make_append(b.cache, k, v, row_start=row_start, q=q, q_out=q, turn=m.turn, rot_dim=m.dim),
                D.make_attend(b.cache, q, self.seen.view(rows, m.q_heads, m.dim), row_start=row_start, scale=m.dim ** -0.5, window=m.window),
                D.make_matvec(self.seen, b.out.codes, b.out.scales, self.mid),
                D.make_norm(self.mid, b.norms[1], self.codes[1], m.eps, res=self.x, sum=self.x, scale=self.scales[1]),
                D.make_matvec(self.codes[1], b.gated.codes, b.gated.scales, self.gated, x_scale=self.scales[1], gate=True),
                D.make_matvec(self.gated, b.down.codes, b.down.scales, self.add),
            ]


class Decoder:
    """streams: texts that grow side by side, max_tokens each at most."""

    def __init__(self, streams, max_tokens, blocks=4, width=1024, q_heads=16, kv_heads=4, dim=64, hidden=2816, vocabulary=8192, group=128, window=0, dtype=torch.bfloat16, part=0, seed=1):
        rng = torch.Generator().manual_seed(seed)
        self.streams, self.max_tokens, self.part = streams, max_tokens, part
        self.width, self.q_heads, self.kv_heads, self.dim, self.hidden, self.group = width, q_heads, kv_heads, dim, hidden, group
        self.dtype, self.window, self.eps = dtype, window, 1e-5
        entries = -(-max_tokens // D.PAGE_TOKENS)
        self.n_pages = streams * entries
        self.free = torch.randperm(self.n_pages, generator=rng).tolist()
        self.table = np.full((streams, entries), -1, np.int32)
        self.pages = torch.full((streams, entries), -1, dtype=torch.int32, device="cuda")
        self.before = torch.zeros(streams, dtype=torch.int32, device="cuda")
        self.lengths = [0] * streams
        angles = torch.arange(max_tokens, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
        self.turn = torch.cat([angles.cos(), angles.sin()], 1).float().cuda()
        self.words = torch.randn((vocabulary, width), generator=rng).to(dtype).cuda()
        self.blocks = [Block(self, rng) for _ in range(blocks)]
        self.last_norm, self.classifier = torch.ones(width, dtype=dtype, device="cuda"), Weights(vocabulary, width, group, rng)
        self.rows = Rows(self, streams)
        self.normed, self.logits = torch.zeros((streams, width), dtype=dtype, device="cuda"), torch.zeros((streams, vocabulary), dtype=dtype, device="cuda")
        head = [D.make_norm(self.rows.add, self.last_norm, self.normed, self.eps, res=self.rows.x),
                D.make_matvec(self.normed, self.classifier.codes, self.classifier.scales, self.logits)]
        self.step_ops, self.head_ops = D.make_ops(self.rows.ops + head), D.make_ops(head)

    def _grow(self, counts):
        """Pages for counts[s] more tokens of stream s."""
        for s, n in enumerate(counts):
            if self.lengths[s] + n > self.max_tokens:
                raise ValueError(f"stream {s} has {self.lengths[s]} tokens, {n} more are over {self.max_tokens}")
        new = False
        for s, n in enumerate(counts):
            for e in range(-(-self.lengths[s] // D.PAGE_TOKENS), -(-(self.lengths[s] + n) // D.PAGE_TOKENS)):
                self.table[s, e], new = self.free.pop(), True
        if new:
            self.pages.copy_(torch.from_numpy(self.table))

    def _grown(self, counts):
        self.lengths = [a + n for a, n in zip(self.lengths, counts)]
        self.before.copy_(torch.tensor(self.lengths, dtype=torch.int32))

    def prompt(self, texts):
        """Appends a text (a list of words' numbers, not empty) to every stream; the words that follow.  Returns them and the rows' buffers."""
        counts = [len(t) for t in texts]
        if len(texts) != self.streams or min(counts) < 1:
            raise ValueError("a text for every stream")
        if min(map(min, texts)) < 0 or max(map(max, texts)) >= len(self.words):
            raise ValueError(f"a word outside 0 .. {len(self.words) - 1}")
        self._grow(counts)
        ends = np.cumsum([0] + counts)
        rows = Rows(self, int(ends[-1]), torch.tensor(ends, dtype=torch.int32, device="cuda"))
        torch.index_select(self.words, 0, torch.tensor(sum(map(list, texts), []), device="cuda"), out=rows.x)
        D.daris_run_ops(D.make_ops(rows.ops), self.part)
        last = torch.tensor(ends[1:] - 1, device="cuda")
        torch.index_select(rows.x, 0, last, out=self.rows.x)
        torch.index_select(rows.add, 0, last, out=self.rows.add)
        D.daris_run_ops(self.head_ops, self.part)
        self._grown(counts)
        return self.logits.argmax(1), rows

    def step(self, words):
        """Appends a word to every stream (a tensor, as prompt and step return them); the words that follow."""
        if words.shape != (self.streams,):
            raise ValueError(f"{tuple(words.shape)} words for {self.streams} streams")
        self._grow([1] * self.streams)
        torch.index_select(self.words, 0, words, out=self.rows.x)
        D.daris_run_ops(self.step_ops, self.part)
        self._grown([1] * self.streams)
        return self.logits.argmax(1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--streams", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=100, help="tokens of the longest prompt; the others are shorter by one each")
    ap.add_argument("--tokens", type=int, default=64, help="steps after the prompts")
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=2816)
    ap.add_argument("--q-heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "fp32"])
    ap.add_argument("--ncu", type=int, default=256, help="partition size")
    ap.add_argument("--check", action="store_true", help="generate twice and compare the words")
    a = ap.parse_args(argv)
    D.daris_init(0, 0, 0)
    part = D.daris_create_partition(a.ncu)
    texts = [[(7 * s + 13 * t) % 8192 for t in range(max(1, a.prompt - s))] for s in range(a.streams)]
    runs = []
    for again in range(2 if a.check else 1):
        m = Decoder(a.streams, a.prompt + a.tokens + 1, a.blocks, a.width, a.q_heads, a.kv_heads, a.dim, a.hidden, window=a.window,
                    dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32, part=part)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        words, _ = m.prompt(texts)
        torch.cuda.synchronize()
        t1, list_us, out = time.perf_counter(), [], [words.tolist()]
        for _ in range(a.tokens):
            words = m.step(words)
            out.append(words.tolist())
        t2 = time.perf_counter()
        for _ in range(20):                                             # the next step's list by itself, at one position
            t = time.perf_counter()
            D.daris_run_ops(m.step_ops, part)
            list_us.append((time.perf_counter() - t) * 1e6)
        runs.append(out)
    line = dict(streams=a.streams, prompt_rows=sum(map(len, texts)), prompt_ms=round((t1 - t0) * 1e3, 3), steps=a.tokens,
                step_us=round((t2 - t1) / max(1, a.tokens) * 1e6, 1), list_us=round(sorted(list_us)[10], 1), operators=len(m.step_ops))
    if a.check:
        line["same"] = runs[0] == runs[1]
    print(json.dumps(line))
    D.daris_shutdown()
    return 0 if line.get("same", True) else 1


if __name__ == "__main__":
    raise SystemExit(main())
