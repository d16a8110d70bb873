"""What the example decoder refuses before anything runs, and its command."""
import pytest
import torch

import paper_2504_08795_amd as D
from paper_2504_08795_amd.generate import Decoder

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(256)
    D.daris_shutdown()


def test_words_that_are_none_and_words_for_other_streams(part):
    m = Decoder(2, 70, blocks=1, width=256, q_heads=4, kv_heads=1, dim=64, hidden=256, vocabulary=320, part=part)
    for texts in ([[1, 320], [2]], [[1], [2, -1]]):
        with pytest.raises(ValueError):
            m.prompt(texts)
    words, _ = m.prompt([[1, 319], [0]])
    at = m.rows.x.data_ptr()
    for wrong in (words[:1], torch.cat([words, words]), words[:, None]):
        with pytest.raises(ValueError):
            m.step(wrong)
    m.step(words)
    assert m.lengths == [3, 2] and m.rows.x.data_ptr() == at


def test_the_command_times_its_list_on_numbers(monkeypatch, capsys):
    from paper_2504_08795_amd import generate
    made = []

    class Kept(Decoder):
        def __init__(self, *args, **more):
            super().__init__(*args, **more)
            made.append(self)
    monkeypatch.setattr(generate, "Decoder", Kept)
    D.daris_shutdown()
    try:
        assert generate.main("--streams 2 --prompt 5 --tokens 10 --blocks 1 --width 256 --hidden 384 --q-heads 4 --kv-heads 2 --check".split()) == 0
    finally:
        D.daris_init(0, 0, 0)
        D.daris_create_partition(256)
    assert '"same": true' in capsys.readouterr().out
    for m in made:
        assert bool(torch.isfinite(m.rows.qkv).all() and torch.isfinite(m.logits).all())
