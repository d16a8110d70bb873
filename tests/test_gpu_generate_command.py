"""The example decoder's command, which begins and ends with the library."""
import json

import pytest

from paper_2504_08795_amd import generate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("args", [["--drafts", "6"], ["--drafts", "4", "--temperature", "0.8", "--top-k", "20"], ["--top-p", "0.9", "--temperature", "1.1"]])
def test_the_command(capsys, args):
    assert generate.main(["--streams", "2", "--prompt", "40", "--tokens", "8", "--blocks", "1", "--width", "256", "--hidden", "384", "--q-heads", "4", "--kv-heads", "2", "--check"] + args) == 0
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["same"] and ("--drafts" not in args or line["words_a_step"] >= 1)
