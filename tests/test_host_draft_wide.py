"""The cases of trees in wide tiles run in wide tiles, those in narrow ones in these, and are cut as they say.  No GPU."""
import pytest

import paper_2504_08795_amd as D
from draft_wide_cases import CASES, CUS, NARROW, WIDE
from test_host_draft import encode  # noqa: F401

DTYPE = {"bf16": D.BF16, "fp32": D.FP32}


def pages_of_units(before, rows, group, window, target, round_, columns=128, most_units=16, more=10):
    """Pages of each sequence, and how many of them a unit takes (of a wide tile, if nothing else is said)."""
    pages = [max(0, -(-(b + r) // 64) - (max(0, b - window) // 64 if window else 0)) for b, r in zip(before, rows)]
    tiles = [-(-r * group // columns) for r in rows]
    work, most = sum(t * p for t, p in zip(tiles, pages)), max(pages)
    c = -(-max(-(-work * 1.0001 // target), -(-most // most_units), 1) // 4) * 4
    cut = lambda p: 1 if p <= c else -(-p // c)  # noqa: E731
    if c < most <= 2 * c and sum(t * cut(p) for t, p in zip(tiles, pages)) > target >= sum(tiles):
        c = most
    if c < most <= work / round_ + more:
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


@pytest.mark.parametrize("dtype", DTYPE)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("name", NARROW)
def test_narrow_cases_are_cut(encode, name, dtype, dim):  # noqa: F811
    before, rows, kv, heads, window, _ = NARROW[name]
    kernel, *_, group, target, units, words = encode(("attend", sum(rows), len(rows), heads, kv, dim, DTYPE[dtype], 1, 256))[0]
    assert kernel == 2 and target > 0
    pages, c = pages_of_units(before, rows, group, window, target, 256 // kv, 16, 256, 30)
    assert max(pages) > 8 * c
