"""A small generating decoder on a partition: every operator of daris_ops.h as a model runs it.

A block is norm (8 bits) -> product -> append -> attend -> product -> norm (8 bits) -> gated product -> product, with the residual taken
along by the norms.  Prompts of several streams go through it as one ragged set of rows, then each step appends one token to every
stream; a step is one list of operators, planned once.  Weights are random: this is an example and a measurement, not a model.

Words are the likeliest ones or drawn (temperature, top_k, top_p, min_p).  A step may carry drafts: a tree of words behind every stream's last one, which goes
through the blocks at once; the words that the model would have given itself stand, and the cache keeps their tokens only.  Such a step makes its buffers and its list
anew, as its rows differ each time: 1.5 ms in place of 0.23 for four streams and four blocks, so it shows the calls and is no gain.  A stream can be continued twice
(fork): full pages are shared and the last one is copied.

    python -m paper_2504_08795_amd.generate --streams 4 --prompt 100 --tokens 64 --check
    python -m paper_2504_08795_amd.generate --temperature 0.8 --top-k 40 --drafts 8
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
    """Buffers for `rows` rows, and the operators that take them through the blocks; tree: masks of rows that are nodes of trees."""

    def __init__(self, m, rows, row_start=None, tree=None):
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
                D.make_append(b.cache, k, v, row_start=row_start, q=q, q_out=q, turn=m.turn, rot_dim=m.dim, tree=tree),
                D.make_attend(b.cache, q, self.seen.view(rows, m.q_heads, m.dim), row_start=row_start, scale=m.dim ** -0.5, window=m.window, tree=tree),
                D.make_matvec(self.seen, b.out.codes, b.out.scales, self.mid),
                D.make_norm(self.mid, b.norms[1], self.codes[1], m.eps, res=self.x, sum=self.x, scale=self.scales[1]),
                D.make_matvec(self.codes[1], b.gated.codes, b.gated.scales, self.gated, x_scale=self.scales[1], gate=True),
                D.make_matvec(self.gated, b.down.codes, b.down.scales, self.add),
            ]


def checked(words, streams, vocabulary):
    """words: a tensor with a word in 0 .. vocabulary - 1 for each stream, or a ValueError.  (-1 is what a row of logits without a number gives: it must not become an index.)"""
    if words.shape != (streams,):
        raise ValueError(f"{tuple(words.shape)} words for {streams} streams")
    for s, w in enumerate(words.tolist()):
        if not 0 <= w < vocabulary:
            raise ValueError(f"stream {s}: word {w} is outside 0 .. {vocabulary - 1}")
    return words


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
        self.users = [0] * self.n_pages                                 # streams that hold a page
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
        # what a stream's words are drawn with: by default the likeliest one
        self.temperature, self.top_p, self.min_p = torch.zeros(streams, device="cuda"), torch.ones(streams, device="cuda"), torch.zeros(streams, device="cuda")
        self.top_k, self.word = torch.zeros(streams, dtype=torch.int32, device="cuda"), torch.zeros(streams, dtype=torch.int32, device="cuda")
        self.random = torch.zeros(streams, device="cuda")
        self.numbers = torch.Generator(device="cuda").manual_seed(seed)
        head = [D.make_norm(self.rows.add, self.last_norm, self.normed, self.eps, res=self.rows.x),
                D.make_matvec(self.normed, self.classifier.codes, self.classifier.scales, self.logits)]
        self.drawn = vocabulary <= D.SAMPLE_WORDS                       # longer rows are not drawn from: their words are the likeliest ones
        if self.drawn:
            head.append(self._sample(self.logits, self.word, self.random, slice(None)))
        self.step_ops, self.head_ops = D.make_ops(self.rows.ops + head), D.make_ops(head)

    def wish(self, temperature=None, top_k=None, top_p=None, min_p=None):
        """What words are drawn with from now on: a number for all streams or one for each (see daris_sample); temperature 0 gives the likeliest."""
        if not self.drawn and temperature is not None and bool((torch.as_tensor(temperature) > 0).any()):
            raise ValueError(f"words are drawn from {D.SAMPLE_WORDS} at most, not from {len(self.words)}")
        for mine, value in ((self.temperature, temperature), (self.top_k, top_k), (self.top_p, top_p), (self.min_p, min_p)):
            if value is not None:
                mine.copy_(torch.as_tensor(value, dtype=mine.dtype).expand(self.streams))

    def _sample(self, logits, word, random, which):
        """Draws a word for each row of logits; which: the rows' streams."""
        return D.make_sample(logits, word, random, temperature=self.temperature[which], top_k=self.top_k[which], top_p=self.top_p[which], min_p=self.min_p[which])

    def _run(self, ops):
        """A list that ends with the streams' words."""
        if self.drawn:
            self.random.uniform_(generator=self.numbers)
        D.daris_run_ops(ops, self.part)
        return self.word.long() if self.drawn else self.logits.argmax(1)

    def _page(self):
        page = self.free.pop()
        self.users[page] = 1
        return page

    def _grow(self, counts):
        """Pages for counts[s] more tokens of stream s."""
        for s, n in enumerate(counts):
            if self.lengths[s] + n > self.max_tokens:
                raise ValueError(f"stream {s} has {self.lengths[s]} tokens, {n} more are over {self.max_tokens}")
        new = False
        for s, n in enumerate(counts):
            for e in range(-(-self.lengths[s] // D.PAGE_TOKENS), -(-(self.lengths[s] + n) // D.PAGE_TOKENS)):
                if self.table[s, e] < 0:                                 # (a step of drafts may have left some)
                    self.table[s, e], new = self._page(), True
        if new:
            self.pages.copy_(torch.from_numpy(self.table))

    def _grown(self, counts):
        self.lengths = [a + n for a, n in zip(self.lengths, counts)]
        self.before += torch.tensor(counts, dtype=torch.int32, device="cuda")

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
        words = self._run(self.head_ops)
        self._grown(counts)
        return words, rows

    def step(self, words):
        """Appends a word to every stream (a tensor, as prompt and step return them); the words that follow."""
        checked(words, self.streams, len(self.words))
        self._grow([1] * self.streams)
        torch.index_select(self.words, 0, words, out=self.rows.x)
        words = self._run(self.step_ops)
        self.lengths = [n + 1 for n in self.lengths]
        self.before += 1                                                # (nothing to copy, which would be waited for)
        return words

    def draft_step(self, words, drafts):
        """Appends a word to every stream with drafts[s] = (words, parents) behind it: parents[i] is the number of the drafted word that drafted word i follows, or -1 for the
        appended one.  The drafts that the model would have given stand.  Returns them (a list for every stream) and the words that follow."""
        checked(words, self.streams, len(self.words))
        if not self.drawn:
            raise ValueError(f"drafts of up to {D.SAMPLE_WORDS} words, not {len(self.words)}")
        if len(drafts) != self.streams:
            raise ValueError(f"{len(drafts)} drafts for {self.streams} streams")
        for texts, parents in drafts:
            if len(texts) != len(parents) or any(not 0 <= w < len(self.words) for w in texts):
                raise ValueError(f"drafts of words in 0 .. {len(self.words) - 1}, each with its parent")
        counts = [1 + len(texts) for texts, _ in drafts]
        tree = D.tree_masks([[-1] + [p + 1 for p in parents] for _, parents in drafts]).cuda()
        self._grow(counts)
        ends = np.cumsum([0] + counts)
        start, n = torch.tensor(ends, dtype=torch.int32, device="cuda"), int(ends[-1])
        nodes = torch.tensor(sum(([0] + list(texts) for texts, _ in drafts), []), dtype=torch.int32).cuda()
        nodes[start[:-1].long()] = words.int()
        rows = Rows(self, n, start, tree)
        torch.index_select(self.words, 0, nodes, out=rows.x)
        normed, logits = torch.empty_like(rows.x), torch.empty((n, len(self.words)), dtype=self.dtype, device="cuda")
        answers, path = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
        count, word, after = (torch.empty(self.streams, dtype=torch.int32, device="cuda") for _ in range(3))
        which = torch.repeat_interleave(torch.arange(self.streams), torch.tensor(counts)).cuda()
        random = torch.rand(n, generator=self.numbers, device="cuda")
        D.daris_run_ops(D.make_ops(rows.ops + [
            D.make_norm(rows.add, self.last_norm, normed, self.eps, res=rows.x), D.make_matvec(normed, self.classifier.codes, self.classifier.scales, logits),
            self._sample(logits, answers, random, which), D.make_accept(tree, nodes, answers, path, count, word, row_start=start, before=self.before, after=after)]
            + [D.make_keep(b.cache, path, count, row_start=start) for b in self.blocks]), self.part)
        self.before.copy_(after)
        kept = count.tolist()
        self.lengths = [a + k for a, k in zip(self.lengths, kept)]
        path = path.tolist()
        return [[drafts[s][0][i - 1] for i in path[ends[s] + 1:ends[s] + k]] for s, k in enumerate(kept)], word.long()

    def release(self, stream):
        """Forgets a stream's text and gives up its pages."""
        for e, page in enumerate(self.table[stream]):
            if page >= 0:
                self.users[page] -= 1
                if self.users[page] == 0:
                    self.free.append(int(page))
                self.table[stream, e] = -1
        self.lengths[stream] = 0
        self._tell()

    def fork(self, stream, to):
        """Stream `to` forgets its text and goes on from stream's: full pages belong to both, the last one is copied."""
        if not (0 <= stream < self.streams and 0 <= to < self.streams) or stream == to:
            raise ValueError(f"stream {stream} continued as {to} of {self.streams}")
        self.release(to)
        full, n = self.lengths[stream] // D.PAGE_TOKENS, self.lengths[stream]
        for e in range(full):
            self.table[to, e] = self.table[stream, e]
            self.users[self.table[to, e]] += 1
        if n % D.PAGE_TOKENS:
            self.table[to, full] = self._page()
            pair = torch.tensor([[self.table[stream, full], self.table[to, full]]], dtype=torch.int32, device="cuda")
            D.daris_run_ops(D.make_ops([D.make_copy(b.cache, pair) for b in self.blocks]), self.part)
        self.lengths[to] = n
        self._tell()

    def _tell(self):
        self.pages.copy_(torch.from_numpy(self.table))
        self.before.copy_(torch.tensor(self.lengths, dtype=torch.int32))


def looked_up(text, most):
    """Drafts behind a text's last word: what followed it where it stood before, the two latest times, `most` words in all."""
    words, parents, starts = [], [], [i + 1 for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:2]
    for i, at in enumerate(starts):
        for j, w in enumerate(text[at:at + (most + 1 - i) // 2]):
            if len(words) < most:
                parents.append(len(words) - 1 if j else -1)
                words.append(w)
    return words, parents


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
    ap.add_argument("--temperature", type=float, default=0.0, help="0: the likeliest word")
    ap.add_argument("--top-k", type=int, default=0)
    ap.add_argument("--top-p", type=float, default=1.0)
    ap.add_argument("--min-p", type=float, default=0.0)
    ap.add_argument("--drafts", type=int, default=0, help="words that a step drafts for a stream from what its text holds already")
    ap.add_argument("--ncu", type=int, default=256, help="partition size")
    ap.add_argument("--check", action="store_true", help="generate twice and compare the words")
    a = ap.parse_args(argv)
    D.daris_init(0, 0, 0)
    part = D.daris_create_partition(a.ncu)
    texts = [[(7 * s + 13 * t) % 8192 for t in range(max(1, a.prompt - s))] for s in range(a.streams)]
    runs = []
    for again in range(2 if a.check else 1):
        m = Decoder(a.streams, a.prompt + a.tokens * (1 + a.drafts) + 1, a.blocks, a.width, a.q_heads, a.kv_heads, a.dim, a.hidden, window=a.window,
                    dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32, part=part)
        m.wish(a.temperature, a.top_k, a.top_p, a.min_p)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        words, _ = m.prompt(texts)
        torch.cuda.synchronize()
        t1, list_us, out = time.perf_counter(), [], [words.tolist()]
        held = [list(t) + [w] for t, w in zip(texts, out[0])]
        for _ in range(a.tokens):
            if a.drafts:
                stood, words = m.draft_step(words, [looked_up(t, a.drafts) for t in held])
                for t, drafted, w in zip(held, stood, words.tolist()):
                    t += drafted + [w]
            else:
                words = m.step(words)
            out.append(words.tolist())
        t2 = time.perf_counter()
        for _ in range(20):                                             # the next step's list by itself, at one position
            t = time.perf_counter()
            D.daris_run_ops(m.step_ops, part)
            list_us.append((time.perf_counter() - t) * 1e6)
        runs.append((out, held))
    line = dict(streams=a.streams, prompt_rows=sum(map(len, texts)), prompt_ms=round((t1 - t0) * 1e3, 3), steps=a.tokens,
                step_us=round((t2 - t1) / max(1, a.tokens) * 1e6, 1), list_us=round(sorted(list_us)[10], 1), operators=len(m.step_ops))
    if a.drafts:
        line["words_a_step"] = round(sum(len(t) - len(u) - 1 for t, u in zip(held, texts)) / (a.streams * max(1, a.tokens)), 2)
    if a.check:
        line["same"] = runs[0] == runs[1]
    print(json.dumps(line))
    D.daris_shutdown()
    return 0 if line.get("same", True) else 1


if __name__ == "__main__":
    raise SystemExit(main())
