"""The cases of trees in wide tiles run in wide tiles, and are cut as they say.  No GPU."""
import pytest

import paper_2504_08795_amd as D
from draft_wide_cases import CASES, CUS, WIDE
from test_host_draft import encode  # noqa: F401

DTYPE = {"bf16": D.BF16, "fp32": D.FP32}


def pages_of_units(before, rows, group, window, target, round_):
    """Pages of each sequence, and how many of them a unit of a wide tile takes."""
    pages = [max(0, -(-(b + r) // 64) - (max(0, b - window) // 64 if window else 0)) for b, r in zip(before, rows)]
    tiles = [-(-r * group // 128) for r in rows]
    work, most = sum(t * p for t, p in zip(tiles, pages)), max(pages)
    c = -(-max(-(-work * 1.0001 // target), -(-most // 16), 1) // 4) * 4
    cut = lambda p: 1 if p <= c else -(-p // c)  # noqa: E731
    if c < most <= 2 * c and sum(t * cut(p) for t, p in zip(tiles, pages)) > target >= sum(tiles):
        c = most
    if c < most <= work / round_ + 10:
        c = most
    return pages, c


@pytest.mark.parametrize("dtype,dim", WIDE)
@pytest.mark.parametrize("name", CASES)
def test_cases_are_what_they_say(encode, name, dtype, dim):  # noqa: F811
    before, rows, kv, heads, window, cut = CASES[name]
    kernel, *_, group, target, units, words = encode(("attend", sum(rows), len(rows), heads, kv, dim, DTYPE[dtype], 2, CUS))[0]
    assert kernel == 3 and group == heads // kv, "wide tiles"
    if not cut:
        return
    assert target > 0
    pages, c = pages_of_units(before, rows, group, window, target, CUS // kv)
    assert max(pages) > c
    if "twelve" in name:
        assert -(-max(pages) // int(c)) == 12
