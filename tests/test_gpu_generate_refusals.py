"""What the example decoder refuses before anything runs."""
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
