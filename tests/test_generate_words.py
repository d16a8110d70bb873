"""Which words the example decoder takes: those that its steps get are indices on the GPU.  No GPU for the check itself."""
import pytest
import torch

import paper_2504_08795_amd as D
from paper_2504_08795_amd.generate import Decoder, checked


@pytest.mark.parametrize("words,named", [([3, -1], "stream 1"), ([320, 0], "stream 0"), ([2 ** 40, 0], "stream 0"), ([-2 ** 63, 1], "stream 0"), ([1], "for 2 streams"), ([1, 2, 3], "for 2 streams")])
def test_words_that_are_none_are_refused(words, named):
    with pytest.raises(ValueError, match=named):
        checked(torch.tensor(words), 2, 320)


@pytest.mark.parametrize("words", [[0, 319], [5, 5]])
def test_words_are_given_back(words):
    assert checked(torch.tensor(words), 2, 320).tolist() == words
    assert checked(torch.tensor(words, dtype=torch.int32), 2, 320).tolist() == words


@pytest.mark.gpu
def test_a_stream_whose_logits_are_no_numbers_is_not_continued():
    """Its word is -1, which neither kind of step takes; the other streams' texts stay as they are."""
    D.daris_init(0, 0, 0)
    try:
        m = Decoder(2, 70, blocks=1, width=256, q_heads=4, kv_heads=1, dim=64, hidden=256, vocabulary=320, part=D.daris_create_partition(256))
        m.words[7] = float("nan")
        words, _ = m.prompt([[1, 2], [3, 7]])
        assert words.tolist()[1] == -1 and 0 <= words.tolist()[0] < 320
        for call in (lambda: m.step(words), lambda: m.draft_step(words, [([], []), ([], [])]), lambda: m.step(torch.full_like(words, 320)), lambda: m.draft_step(words[:1], [([], []), ([], [])])):
            with pytest.raises(ValueError):
                call()
        assert m.lengths == [2, 2] and m.before.tolist() == [2, 2]
        words[1] = 0
        m.step(words)
        assert m.lengths == [3, 3]
    finally:
        D.daris_shutdown()


@pytest.mark.gpu
def test_vocabularies_that_are_not_drawn_from_give_their_likeliest_words():
    D.daris_init(0, 0, 0)
    try:
        m = Decoder(2, 70, blocks=1, width=128, q_heads=2, kv_heads=1, dim=64, hidden=128, vocabulary=D.SAMPLE_WORDS + 16, part=D.daris_create_partition(256))
        words, _ = m.prompt([[1, D.SAMPLE_WORDS + 3], [3]])
        for _ in range(2):
            assert torch.equal(m.logits.gather(1, words[:, None])[:, 0], m.logits.amax(1))
            words = m.step(words)
        m.wish(temperature=0.0, top_k=3)
        for call in (lambda: m.wish(temperature=[0.0, 0.5]), lambda: m.draft_step(words, [([], []), ([], [])])):
            with pytest.raises(ValueError, match=str(D.SAMPLE_WORDS)):
                call()
        assert m.lengths == [4, 3] and m.temperature.tolist() == [0, 0]
    finally:
        D.daris_shutdown()


@pytest.mark.gpu
def test_a_step_is_one_list_that_ends_with_its_words(monkeypatch):
    from paper_2504_08795_amd import generate
    lists, run = [], D.daris_run_ops
    monkeypatch.setattr(generate.D, "daris_run_ops", lambda ops, part: (lists.append(ops), run(ops, part))[1])
    D.daris_init(0, 0, 0)
    try:
        m = Decoder(2, 200, blocks=1, width=256, q_heads=4, kv_heads=1, dim=64, hidden=256, vocabulary=320, part=D.daris_create_partition(256))
        m.wish(temperature=0.8)
        words, _ = m.prompt([[1, 2], [3] * 70])
        for _ in range(3):
            lists.clear()
            words = m.step(words)
            assert lists == [m.step_ops] and torch.equal(words, m.word.long()) and m.before.tolist() == m.lengths
        m.fork(1, 0)
        assert m.before.tolist() == m.lengths == [73, 73]
    finally:
        D.daris_shutdown()
