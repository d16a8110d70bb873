"""The example decoder's words by random numbers, its steps with drafts, and streams that are continued twice."""
import pytest
import torch

import paper_2504_08795_amd as D
from draft_helpers import drawn
from paper_2504_08795_amd.generate import Decoder, looked_up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(256)
    D.daris_shutdown()


def small(part, streams, **more):
    return Decoder(streams, 400, blocks=2, width=256, q_heads=6, kv_heads=2, dim=64, hidden=384, vocabulary=320, group=128, part=part, dtype=torch.float32, **more)


def test_words_are_drawn_as_wished(part):
    m = small(part, 3)
    m.wish(temperature=[0.7, 0.0, 1.5], top_k=[5, 0, 0], top_p=0.9, min_p=[0.0, 0.0, 0.01])
    words, _ = m.prompt([[1, 2, 3], [4] * 20, [7]])
    for _ in range(4):
        x, u = m.logits.cpu(), m.random.tolist()
        assert words.tolist() == [drawn(x[s], u[s], t, k, p, mp)[0] for s, (t, k, p, mp) in enumerate(zip(m.temperature.tolist(), m.top_k.tolist(), m.top_p.tolist(), m.min_p.tolist()))]
        words = m.step(words)


def test_drafts_stand_where_the_model_says_the_same(part):
    """The likeliest words, drafted as they come, wrong from some place on, and on a second branch: what stands is what steps of one word give."""
    texts = [[5, 6, 7, 8], [9] * 70]
    m = small(part, 2)
    words, _ = m.prompt(texts)
    want = [words.tolist()]
    for _ in range(12):
        words = m.step(words)
        want.append(words.tolist())
    want = list(zip(*want))                                 # of each stream
    m = small(part, 2)
    words, _ = m.prompt(texts)
    assert words.tolist() == [w[0] for w in want]
    right, wrong = lambda s, n, m: list(want[s][n:m]), lambda w: (w + 1) % 320  # noqa: E731
    # stream 0: five right words behind a wrong branch; stream 1: two right ones, then a wrong one
    first = ([wrong(want[0][1]), 11] + right(0, 1, 6), [-1, 0, -1, 2, 3, 4, 5])
    second = (right(1, 1, 3) + [wrong(want[1][3]), 3], [-1, 0, 1, 2])
    stood, words = m.draft_step(words, [first, second])
    assert stood == [right(0, 1, 6), right(1, 1, 3)] and words.tolist() == [want[0][6], want[1][3]] and m.lengths == [4 + 6, 70 + 3]
    stood, words = m.draft_step(words, [([], []), (right(1, 4, 5), [-1])])
    assert stood == [[], right(1, 4, 5)] and words.tolist() == [want[0][7], want[1][5]]
    words = m.step(words)                                   # a step of one word goes on from there
    assert words.tolist() == [want[0][8], want[1][6]]
    with pytest.raises(ValueError):
        m.draft_step(words, [([320], [-1]), ([], [])])
    with pytest.raises(ValueError):
        m.draft_step(words, [([1], [-1])])
    with pytest.raises(D.DarisError):
        m.draft_step(words, [([1], [0]), ([], [])])         # below itself


def test_a_stream_is_continued_twice(part):
    m = small(part, 3)
    words, _ = m.prompt([[3 + i % 50 for i in range(150)], [1], [2] * 90])
    free = len(m.free)
    m.fork(0, 1)
    assert m.lengths == [150, 150, 90] and m.users[m.table[0, 0]] == 2 and m.table[1, 0] == m.table[0, 0] and m.table[1, 2] != m.table[0, 2]
    assert len(m.free) == free                              # one page given up, one taken
    words[1] = words[0]
    for _ in range(6):
        words = m.step(words)
        assert int(words[0]) == int(words[1])               # the same text
    other = words.clone()
    other[1] = (other[1] + 1) % 320
    words = m.step(other)                                   # and now another
    alone = small(part, 3)
    again, _ = alone.prompt([[3 + i % 50 for i in range(150)], [1], [2] * 90])
    for _ in range(6):
        again = alone.step(again)
    again = alone.step(again)
    assert int(again[0]) == int(words[0]) and int(again[2]) == int(words[2])
    m.release(0)
    assert m.users[m.table[1, 0]] == 1 and m.lengths[0] == 0
    m.release(1)
    m.release(2)
    assert sorted(m.free) == list(range(m.n_pages))
    with pytest.raises(ValueError):
        m.fork(1, 1)


def test_drafts_from_a_text():
    assert looked_up([1, 2, 3, 1, 4, 1], 5) == ([4, 1, 2, 3], [-1, 0, -1, 2])
    assert looked_up([1, 2], 5) == ([], []) and looked_up([7], 3) == ([], []) and looked_up([5, 5, 5], 1) == ([5], [-1])
