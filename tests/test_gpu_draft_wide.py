"""Attention of trees in wide tiles, whole and cut into units that are merged, and in narrow ones that are cut, against 64 bits (see draft_wide_cases)."""
import numpy as np
import pytest
import torch

import paper_2504_08795_amd as D
from draft_helpers import bits_of
from draft_wide_cases import CASES, CUS, NARROW, WIDE
from step_helpers import DT, PAGE, Cache, close
from test_gpu_draft import attend_case, rand, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    p = D.daris_create_partition(CUS)
    D.daris_create_partition(256)
    yield p
    D.daris_shutdown()


LARGE = 1      # the partition of 256 CUs


@pytest.mark.parametrize("dtype,dim", WIDE)
@pytest.mark.parametrize("name", CASES)
def test_trees(part, name, dtype, dim):
    before, rows, kv, heads, window, _ = CASES[name]
    attend_case(part, 200 + dim, before, rows, kv, dim, heads, dtype, window)


@pytest.mark.parametrize("dtype,dim", WIDE)
@pytest.mark.parametrize("name", ["several", "cut, two tiles"])
@pytest.mark.parametrize("window", [0, 9])
def test_masks_that_are_no_trees(part, name, dtype, dim, window):
    """Any nodes in front and behind, none at all, bits of rows that there are not, two words where one would do."""
    before, rows, kv, heads, _, _ = CASES[name]
    n = sum(rows)
    masks = torch.from_numpy(np.random.default_rng(7).integers(-2 ** 63, 2 ** 63, (n, 2)))
    masks[5] = 0                                            # sees the cached tokens only
    empty = [i for s, b in enumerate(before) if b == 0 for i in range(sum(rows[:s]), sum(rows[:s + 1]))][:2]
    masks[empty[0]] = 0                                     # sees nothing: zeros
    masks[empty[1], 0], masks[empty[1], 1] = 0, 1 << 62     # ... a row that its sequence does not have
    got, _ = attend_case(part, 210 + dim, before, rows, kv, dim, heads, dtype, window, masks, extra_rows=3, skew=8)
    assert bool((got[empty] == 0).all()) and bool((got[5] != 0).any())


@pytest.mark.parametrize("dtype,dim", WIDE)
@pytest.mark.parametrize("name", ["whole", "cut, two tiles"])
def test_nodes_that_a_row_does_not_see_have_no_influence(part, name, dtype, dim):
    before, rows, kv, heads, _, _ = CASES[name]
    s = int(np.argmax(before))
    row0, r, masks, bad = sum(rows[:s]), rows[s], trees(221, rows), 7
    place = lambda c: (int(c.pages[s, (before[s] + bad) // PAGE]), (before[s] + bad) % PAGE)  # noqa: E731

    def among_values(c):
        page, i = place(c)
        c.v.view(torch.uint8)[page, 0, 3, i] = 0x7F

    def both(c):
        among_values(c)
        page, i = place(c)
        c.k.view(torch.uint8)[page, 0, i, 5] = 0xFF
    seen = torch.zeros(sum(rows), dtype=torch.bool)
    for i in range(r):
        seen[row0 + i] = bad in bits_of(masks[row0 + i].tolist())
    assert 1 <= int(seen.sum()) < r
    first = heads // kv                                     # query heads of the first key head
    got, _ = attend_case(part, 222, before, rows, kv, dim, heads, dtype, 0, masks, among_values)
    assert bool(torch.isnan(got[seen][:, :first, 3]).all()) and int(torch.isnan(got).sum()) == int(seen.sum()) * first
    got, _ = attend_case(part, 223, before, rows, kv, dim, heads, dtype, 0, masks, both)
    assert bool(torch.isnan(got[seen][:, :first]).all()) and int(torch.isnan(got).sum()) == int(seen.sum()) * first * dim


@pytest.mark.parametrize("dtype,dim", WIDE)
@pytest.mark.parametrize("window", [0, 50])
def test_a_chain_is_what_follows_row_by_row(part, dtype, dim, window):
    c = Cache(231, [90], [90], 2, dim).filled(232)
    cache, q = c.gpu(D), rand((90, 16, dim), DT[dtype], 233, 0.5).cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    D.daris_run_ops(D.make_ops([D.make_attend(cache, q, a, row_start=c.start.cuda(), scale=0.02, window=window),
                                D.make_attend(cache, q, b, row_start=c.start.cuda(), scale=0.02, window=window, tree=D.tree_masks([list(range(-1, 89))]).cuda())]), part)
    # weights differ by the page at which the running maximum moves: two roundings of the output and of a weight's f16
    close(b, a.cpu().double(), a.cpu().double().abs() * 2.0 ** -7 + 2.0 ** -10 * float(c.tokens(0, 180)[1].abs().max()), "chain")


@pytest.mark.parametrize("dtype,dim", WIDE)
def test_cut_tiles_are_merged_alike_each_time(part, dtype, dim):
    """The units' order of arrival changes nothing, and their counters are ready for the next run."""
    before, rows, kv, heads, _, _ = CASES["cut"]
    c = Cache(241, before, rows, kv, dim).filled(242)
    q = rand((sum(rows), heads, dim), DT[dtype], 243, 0.3).cuda()
    out = torch.empty_like(q)
    ops = D.make_ops([D.make_attend(c.gpu(D), q, out, row_start=c.start.cuda(), scale=0.02, tree=trees(244, rows).cuda())])
    D.daris_run_ops(ops, part)
    first = out.clone()
    for _ in range(10):
        out.zero_()
        D.daris_run_ops(ops, part)
        assert torch.equal(out, first)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("name", NARROW)
def test_narrow_tiles_that_are_cut(part, name, dim, dtype):
    before, rows, kv, heads, window, _ = NARROW[name]
    attend_case(LARGE, 250 + dim, before, rows, kv, dim, heads, dtype, window)

    def bad(c):                                             # a NaN among the values of node 5
        page, i = int(c.pages[0, (before[0] + 5) // PAGE]), (before[0] + 5) % PAGE
        c.v.view(torch.uint8)[page, 0, 3, i] = 0x7F
    masks = trees(251, rows)
    seen = torch.tensor([i < rows[0] and 5 in bits_of(masks[i].tolist()) for i in range(sum(rows))])
    got, _ = attend_case(LARGE, 252, before, rows, kv, dim, heads, dtype, window, masks, bad)
    assert 1 <= int(seen.sum()) < rows[0] and bool(torch.isnan(got[seen][:, :heads // kv, 3]).all()) and int(torch.isnan(got).sum()) == int(seen.sum()) * (heads // kv)
