"""The example decoder: each operator of a block against 64 bits on the numbers it was given, and the words it generates."""
import pytest
import torch

import paper_2504_08795_amd as D
from paper_2504_08795_amd.generate import Decoder
from step_helpers import Cache, DT, ROUND, attend, close, e4m3_slack, matvec, norm, turned, two_to

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(256)
    D.daris_shutdown()


def small(part, streams, dtype, **more):
    return Decoder(streams, 160, blocks=1, width=256, q_heads=6, kv_heads=2, dim=64, hidden=384, vocabulary=320, group=128, dtype=DT[dtype], part=part, **more)


def rows_of(codes, scales):
    s = two_to(scales.cpu())
    return codes.cpu().double() * s.repeat_interleave(codes.shape[1] // s.shape[1], 1)


def block_case(m, rows, x, before, counts, dtype):
    """rows: the buffers after a run of the only block over x (on the CPU)."""
    b, r = m.blocks[0], ROUND[dtype]
    for i, (inp, res) in enumerate(((x, None), (rows.mid, x))):
        h, want = norm(inp, res, b.norms[i], m.eps)
        s = two_to(rows.scales[i].cpu()).repeat_interleave(m.group, 1)
        close(rows_of(rows.codes[i], rows.scales[i]), want, e4m3_slack(want, s), f"norm {i}")
    close(rows.x, h, h.abs() * (r + 2.0 ** -24) + 1e-38, "residual")
    q, k, v = rows.qkv.split([m.q_heads, m.kv_heads, m.kv_heads], 1)
    want, slack = matvec(rows_of(rows.codes[0], rows.scales[0]), b.qkv.codes.cpu(), b.qkv.scales.cpu(), False, dtype)
    want, slack = (t.view(rows.qkv.shape) for t in (want, slack))
    close(k, want[:, m.q_heads:m.q_heads + m.kv_heads], slack[:, m.q_heads:m.q_heads + m.kv_heads], "keys")
    close(v, want[:, m.q_heads + m.kv_heads:], slack[:, m.q_heads + m.kv_heads:], "values")
    turn, at = m.turn.cpu(), 0
    c = Cache(1, before, counts, m.kv_heads, m.dim, garbage=False)
    c.pages, c.k, c.v, c.k_scale, c.v_scale = m.pages.cpu(), b.k.cpu(), b.v.cpu(), b.k_scale.cpu(), b.v_scale.cpu()
    for s, n in enumerate(counts):
        held_k, held_v, there = c.tokens(s, before[s] + n)
        assert bool(there.all())
        for i in range(n):
            pos = before[s] + i
            asked = turned(want[at, :m.q_heads], turn[pos], m.dim, False)
            off = turned(slack[at, :m.q_heads], turn[pos].abs() * 1.0, m.dim, False).abs() + 2 * slack[at, :m.q_heads].amax()     # each output takes two inputs
            close(q[at], asked, off + asked.abs() * r + want[at, :m.q_heads].abs().amax() * (2 * r + 2.0 ** -22), "queries")
            # scales only grow while a sixteenth fills: a token is within two roundings of its value
            for held, new, scales in ((held_k, turned(k[at].cpu().double(), turn[pos], m.dim, False), c.k_scale), (held_v, v[at].cpu().double(), c.v_scale)):
                page = int(c.pages[s, pos // 64])
                close(held[:, pos], new, 2 * e4m3_slack(new, two_to(scales)[page, :, pos % 64 // 16, None]), "cache")
            at += 1
    want, slack = attend(c, q.cpu(), m.dim ** -0.5, m.window, dtype)
    close(rows.seen, want.flatten(1), slack.flatten(1), "attention")
    for y, x_, w, gate, what in ((rows.mid, rows.seen.cpu().double(), b.out, False, "output"), (rows.gated, rows_of(rows.codes[1], rows.scales[1]), b.gated, True, "gated"),
                                 (rows.add, rows.gated.cpu().double(), b.down, False, "down")):
        want, slack = matvec(x_, w.codes.cpu(), w.scales.cpu(), gate, dtype)
        close(y, want, slack, what)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [0, 20])
def test_every_operator_of_a_block_on_what_it_was_given(part, dtype, window):
    m = small(part, 3, dtype, window=window)
    texts = [[(5 * s + 3 * t) % 320 for t in range(n)] for s, n in enumerate((40, 1, 17))]
    words, rows = m.prompt(texts)
    block_case(m, rows, m.words[torch.tensor(sum(texts, []), device="cuda")].cpu(), [0, 0, 0], [40, 1, 17], dtype)
    for i in range(30):                       # past a page's end, too
        x, before = m.words[words].cpu(), list(m.lengths)
        words = m.step(words)
        if i in (0, 25):
            block_case(m, m.rows, x, before, [1, 1, 1], dtype)
        _, want = norm(m.rows.add, m.rows.x, m.last_norm, m.eps)
        close(m.normed, want, want.abs() * (2.0 ** -20 + ROUND[dtype]) + 1e-38, "last norm")
        want, slack = matvec(m.normed.cpu().double(), m.classifier.codes.cpu(), m.classifier.scales.cpu(), False, dtype)
        close(m.logits, want, slack, "logits")
        assert torch.equal(words, m.logits.argmax(1))


def test_generating_twice_gives_the_same_words_and_too_long_a_text_is_refused(part):
    out = []
    for _ in range(2):
        m = Decoder(2, 70, blocks=3, width=256, q_heads=4, kv_heads=1, dim=128, hidden=512, vocabulary=320, part=part)
        words, _ = m.prompt([[1, 2, 3], [4] * 20])
        out.append([words.tolist()] + [m.step(words).tolist() for _ in range(45)])
    assert out[0] == out[1] and m.lengths == [48, 65]
    before = m.table.copy()
    with pytest.raises(ValueError):
        m.prompt([[1], [2] * 6])
    with pytest.raises(ValueError):
        m.prompt([[1], []])
    assert m.lengths == [48, 65] and (before == m.table).all()
