"""The operators of a drafted step (include/daris_ops.h) against their definitions in 64 bits, at the trees, lengths, masks and values where they
can go wrong."""
import math

import numpy as np
import pytest
import torch

import paper_2504_08795_amd as D
from draft_helpers import attend_tree, bits_of, drawn, kept, random_parents, same_codes, walk
from step_helpers import BLOCK, DT, E8, F8, PAGE, ROUND, Cache, close, e4m3_slack, scale_exponent, turn_table, turned, two_to

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    p = D.daris_create_partition(256)
    D.daris_create_partition(24)
    yield p
    D.daris_shutdown()


SMALL = 1      # the partition of 24 CUs


def rand(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def run(part, *ops):
    D.daris_run_ops(D.make_ops(list(ops)), part)


def trees(seed, rows, words=None):
    rng = np.random.default_rng(seed)
    return D.tree_masks([random_parents(rng, r) for r in rows], words)


# ---- attention ------------------------------------------------------------------------------------------------------------------


def attend_case(part, seed, before, rows, kv, dim, heads, dtype, window=0, masks=None, edit=None, skew=0, extra_rows=0):
    c = Cache(seed, before, rows, kv, dim).filled(seed + 1)
    masks = trees(seed, rows) if masks is None else masks
    if edit:
        edit(c)
    n, dt = sum(rows), DT[dtype]
    q = rand((n + extra_rows, heads, dim), dt, seed + 2, 0.3)
    cache = c.gpu(D)
    wide = torch.zeros((n + extra_rows, heads, dim + skew), dtype=dt, device="cuda")
    wide[:, :, :dim] = q.cuda()
    out = torch.full((n + extra_rows, heads, dim + skew), 7.0, dtype=dt, device="cuda")
    more = torch.zeros((extra_rows, masks.shape[1]), dtype=torch.int64)
    start = None if rows == [1] * len(rows) and seed % 2 else c.start.cuda()
    scale = 0.02
    run(part, D.make_attend(cache, wide[:, :, :dim], out[:, :, :dim], row_start=start, scale=scale, window=window, tree=torch.cat([masks, more]).cuda()))
    want, slack = attend_tree(c, masks, q[:n], scale, window, dtype)
    close(out[:n, :, :dim], want, slack, "attention")
    assert bool((out[n:] == 7).all()) and bool((out[:, :, dim:] == 7).all()), "rows of no sequence, and what lies between rows, are left alone"
    return out[:n, :, :dim].cpu(), want


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("before,rows,kv,dim,heads,window", [
    ([0], [1], 1, 64, 1, 0), ([5], [2], 2, 64, 2, 0), ([63], [13], 1, 128, 4, 0), ([64], [26], 2, 64, 6, 0), ([130], [64], 1, 128, 7, 0), ([300], [65], 1, 64, 4, 0),
    ([61, 0, 640, 7], [5, 9, 33, 1], 2, 64, 4, 0), ([1000, 20], [130, 3], 1, 128, 2, 0), ([77, 200], [9, 17], 2, 256, 4, 0), ([40, 90, 3], [1, 1, 1], 2, 64, 4, 0),
    ([100], [13], 1, 64, 2, 1), ([100], [13], 1, 64, 2, 3), ([300, 10], [40, 40], 2, 64, 4, 64), ([500], [70], 1, 128, 2, 130), ([2000], [13], 4, 64, 12, 700), ([200, 4], [20, 20], 1, 256, 2, 30)])
def test_trees_behind_cached_tokens(part, dtype, before, rows, kv, dim, heads, window):
    attend_case(part, 11 * len(rows) + window, before, rows, kv, dim, heads, dtype, window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("before,rows,kv,dim,heads,window", [([70], [50], 2, 64, 32, 0), ([130, 40], [64, 33], 2, 128, 16, 0), ([129], [150], 1, 128, 10, 60), ([500], [40], 2, 64, 40, 100)])
def test_trees_in_wide_tiles(part, dtype, before, rows, kv, dim, heads, window):
    attend_case(SMALL, 5 + len(rows), before, rows, kv, dim, heads, dtype, window)


@pytest.mark.parametrize("place", [0, SMALL])
@pytest.mark.parametrize("window", [0, 9])
def test_masks_that_are_no_trees(part, place, window):
    """Any nodes in front and behind, none at all, bits of rows that there are not, fewer words than rows."""
    rows, before = [70, 3, 90, 16], [40, 0, 129, 70]
    rng = np.random.default_rng(3)
    masks = torch.from_numpy(rng.integers(-2 ** 63, 2 ** 63, (sum(rows), 1)))
    masks[5] = 0                                            # sees the cached tokens only
    masks[70] = 0                                           # sees nothing: zeros
    masks[71] = 1 << 40                                     # ... a row that its sequence does not have
    masks[80] = -1
    got, want = attend_case(part if place == 0 else place, 21, before, rows, 2, 64, 24, "bf16", window, masks)
    assert bool((got[70:72] == 0).all()) and bool((want[70:72] == 0).all()) and bool((got[72] != 0).any())
    two = torch.cat([masks, torch.from_numpy(rng.integers(-2 ** 63, 2 ** 63, (sum(rows), 1)))], 1)
    attend_case(part if place == 0 else place, 22, before, rows, 1, 128, 12, "fp32", window, two, extra_rows=4, skew=3)


def test_rows_whose_masks_hold_one_word_of_sixteen(part):
    rows = [700]
    masks = torch.zeros((700, 16), dtype=torch.int64)
    for i in range(700):
        masks[i, i // 64] = 1 << (i % 64) if i % 64 < 63 else -2 ** 63
        masks[i, 0] |= 1
    attend_case(part, 30, [50], rows, 1, 64, 1, "bf16", 0, masks)


def test_a_chain_is_what_follows_row_by_row(part):
    """A tree without branches sees what rows see that follow each other."""
    for place, heads, window in ((part, 4, 0), (SMALL, 40, 0), (part, 4, 50)):
        c = Cache(31, [90], [60], 1, 64).filled(32)
        cache, q = c.gpu(D), rand((60, heads, 64), torch.bfloat16, 33, 0.5).cuda()
        a, b = torch.empty_like(q), torch.empty_like(q)
        run(place, D.make_attend(cache, q, a, row_start=c.start.cuda(), scale=0.02, window=window),
            D.make_attend(cache, q, b, row_start=c.start.cuda(), scale=0.02, window=window, tree=D.tree_masks([list(range(-1, 59))]).cuda()))
        # weights differ by the page at which the running maximum moves: two roundings of the output and of a weight's f16
        close(b, a.cpu().double(), a.cpu().double().abs() * 2.0 ** -7 + 2.0 ** -10 * float(c.tokens(0, 150)[1].abs().max()), "chain")


@pytest.mark.parametrize("place,heads", [(0, 4), (SMALL, 40)])
def test_nodes_that_a_row_does_not_see_have_no_influence(part, place, heads):
    rows, masks = [40], trees(41, [40])
    bad = 17

    def edit(c):
        page, i = int(c.pages[0, (100 + bad) // PAGE]), (100 + bad) % PAGE
        c.v.view(torch.uint8)[page, 0, 3, i] = 0x7F         # a NaN among the values of node 17
        c.k.view(torch.uint8)[page, 0, i, 5] = 0xFF         # ... and among its key
    got, want = attend_case(part if place == 0 else place, 41, [100], rows, 1, 64, heads, "bf16", 0, masks, edit)
    seen = torch.tensor([bad in bits_of(masks[i].tolist()) for i in range(40)])
    assert 1 <= int(seen.sum()) < 40 and bool(torch.isnan(got[seen]).all()) and not bool(torch.isnan(got[~seen]).any())

    def values_only(c):
        page, i = int(c.pages[0, (100 + bad) // PAGE]), (100 + bad) % PAGE
        c.v.view(torch.uint8)[page, 0, 3, i] = 0x7F
    got, want = attend_case(part if place == 0 else place, 42, [100], rows, 1, 64, heads, "bf16", 0, masks, values_only)
    assert bool(torch.isnan(got[seen][:, :, 3]).all()) and int(torch.isnan(got).sum()) == int(seen.sum()) * heads


def test_pages_that_are_not_there(part):
    def edit(c):
        c.pages[0, 1] = -1
        c.pages[1, 0] = 10 ** 6
        c.pages[0, 3] = -1                                  # part of the tree
    attend_case(part, 51, [150, 40], [80, 20], 1, 64, 2, "bf16", 0, edit=edit)
    attend_case(SMALL, 52, [150, 40], [80, 20], 1, 64, 40, "bf16", 0, edit=edit)


def test_many_streams_with_trees(part):
    rng = np.random.default_rng(61)
    before, rows = rng.integers(0, 150, 70).tolist(), rng.integers(0, 12, 70).tolist()
    attend_case(part, 61, before, rows, 1, 64, 2, "bf16")
    attend_case(part, 62, before, rows, 2, 64, 4, "fp32", 20)


def test_tokens_in_front_of_the_first(part):
    """before < 0: the first nodes have no place, the others attend what has."""
    attend_case(part, 71, [-3, 5], [9, 4], 1, 64, 2, "bf16")
    attend_case(part, 72, [-3, 5], [9, 4], 1, 64, 2, "bf16", 2)


# ---- append ---------------------------------------------------------------------------------------------------------------------


def append_case(part, seed, before, rows, kv, dim, heads, dtype, rot, pairs, words=None, masks=None, positions=None, in_place=False, edit=None):
    c = Cache(seed, before, rows, kv, dim)
    if edit:
        edit(c)
    n, dt = sum(rows), DT[dtype]
    masks = trees(seed, rows, words) if masks is None else masks
    qkv = rand((n, heads + 2 * kv, dim), dt, seed + 1, 1.5)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    table = turn_table(positions if positions is not None else max(b + r for b, r in zip(before, rows)) + 1, rot) if rot else None
    old = {m: getattr(c, m).clone() for m in ("k", "v", "k_scale", "v_scale")}
    cache, g = c.gpu(D), qkv.cuda()
    gq, gk, gv = g[:, :heads], g[:, heads:heads + kv], g[:, heads + kv:]
    out = gq if in_place else torch.full((n, heads, dim), 7.0, dtype=dt, device="cuda")
    run(part, D.make_append(cache, gk, gv, row_start=None if rows == [1] * len(rows) and seed % 2 else c.start.cuda(), q=gq, q_out=out, turn=table.cuda() if rot else None,
                            rot_dim=rot, pairs=pairs, tree=masks.cuda()))
    got = {m: t.cpu() for m, t in zip(("k", "v", "k_scale", "v_scale"), c.on_gpu)}
    touched = {m: torch.zeros_like(old[m].view(torch.uint8), dtype=torch.bool) for m in old}
    row = lambda p: table[p] if 0 <= p < len(table) else torch.full((rot,), float("nan"))  # noqa: E731
    for s, (b, r) in enumerate(zip(before, rows)):
        pos = [b + len(bits_of(masks[int(c.start[s]) + i].tolist())) - 1 for i in range(r)]
        new = {"k": [turned(k[int(c.start[s]) + i].double(), row(pos[i]), rot, pairs) if rot else k[int(c.start[s]) + i].double() for i in range(r)],
               "v": [v[int(c.start[s]) + i].double() for i in range(r)]}
        for i in range(r):
            a = int(c.start[s]) + i
            want = turned(q[a].double(), row(pos[i]), rot, pairs) if rot else q[a].double()
            close(out[a], want, (want.abs() + q[a].double().abs().amax()) * (2.0 ** -22 + ROUND[dtype]), "queries")
        for name in ("k", "v"):
            scales, codes = got[name + "_scale"].view(torch.uint8).int(), got[name]
            for begin in range(max(b, 0) // BLOCK * BLOCK, b + r, BLOCK):
                page, blk = int(c.pages[s, begin // PAGE]), begin % PAGE // BLOCK
                if page < 0:
                    continue
                tokens = [t for t in range(max(begin, b), min(begin + BLOCK, b + r))]
                held = [t for t in range(begin, min(begin + BLOCK, b))]
                most = torch.stack([new[name][t - b] for t in tokens]).abs().nan_to_num(0, 0, 0).amax((0, 2))      # (what is not finite has no part in it)
                need = scale_exponent(most).int() + 127
                had = old[name + "_scale"].view(torch.uint8)[page, :, blk].int()
                want = torch.maximum(need, had) if held else need
                now = scales[page, :, blk]
                edge = ((most / (448 * torch.exp2((now - 127).double())) - 1).abs() < 1e-5) | ((most / (224 * torch.exp2((now - 127).double())) - 1).abs() < 1e-5)
                assert bool(((now == want) | (edge & ((now - want).abs() <= 1))).all()), (name, now, want)
                step = torch.exp2((now - 127).double())[:, None]
                for t in tokens + held:
                    at = (page, slice(None), t % PAGE) if name == "k" else (page, slice(None), slice(None), t % PAGE)
                    touched[name][at] = True
                    value = new[name][t - b] if t in tokens else old[name][at].double() * torch.exp2((had - 127).double())[:, None]
                    close(codes[at].double() * step, value, e4m3_slack(value.nan_to_num(0, 0, 0), step), f"{name} of token {t}")
                touched[name + "_scale"][page, :, blk] = True
    for m in old:
        assert torch.equal(got[m].view(torch.uint8)[~touched[m]], old[m].view(torch.uint8)[~touched[m]]), f"{m}: places that hold no token changed"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("before,rows,kv,dim,heads,rot,pairs", [
    ([0], [1], 1, 64, 1, 64, False), ([15], [26], 2, 128, 5, 128, False), ([63, 0, 40], [9, 20, 1], 2, 64, 4, 32, True), ([100], [70], 1, 256, 3, 256, False), ([7, 3, 9], [1, 1, 1], 2, 64, 4, 64, True),
    ([30], [18], 3, 128, 9, 0, False), ([130], [200], 1, 64, 2, 16, False)])
def test_tree_append(part, dtype, before, rows, kv, dim, heads, rot, pairs):
    append_case(part, 100 + len(rows) + dim, before, rows, kv, dim, heads, dtype, rot, pairs)


def test_tree_append_positions(part):
    """In place, more words than needed, positions outside the table, masks without a bit, a page that is not there."""
    append_case(part, 120, [20, 4], [30, 11], 2, 64, 4, "bf16", 64, False, words=3, in_place=True)
    append_case(part, 121, [20], [30], 1, 64, 2, "fp32", 64, False, positions=24)
    masks = trees(122, [12])
    masks[4] = 0
    masks[7] = -1
    append_case(part, 122, [9], [12], 1, 128, 2, "fp32", 64, True, masks=masks, positions=100)
    append_case(part, 123, [0], [5], 1, 64, 2, "fp32", 64, True, masks=torch.zeros((5, 1), dtype=torch.int64))

    def edit(c):
        c.pages[0, 1] = -1
    append_case(part, 124, [50], [40], 1, 64, 2, "bf16", 64, False, edit=edit)


# ---- sample -----------------------------------------------------------------------------------------------------------------------


def sample_case(part, x, u, temperature=None, top_k=None, top_p=None, min_p=None, skew=0, chance=True):
    """x [rows][n] on the CPU; the others lists or None."""
    rows, n = x.shape
    wide = torch.zeros((rows, n + skew), dtype=x.dtype, device="cuda")
    wide[:, skew:] = x.cuda()
    f = lambda v, t=torch.float32: None if v is None else torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    word, p = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), -7.0, device="cuda")
    run(part, D.make_sample(wide[:, skew:], word, f(u), temperature=f(temperature), top_k=f(top_k, torch.int32), top_p=f(top_p), min_p=f(min_p), chance=p if chance else None))
    f32 = lambda v, i, none: none if v is None else float(np.float32(v[i]))  # noqa: E731
    want = [drawn(x[i], f32(u, i, None), f32(temperature, i, 1.0), 0 if top_k is None else top_k[i], f32(top_p, i, 1.0), f32(min_p, i, 0.0)) for i in range(rows)]
    assert word.tolist() == [w for w, _ in want], [(i, a, b) for i, (a, b) in enumerate(zip(word.tolist(), [w for w, _ in want])) if a != b][:5]
    if chance:
        want = torch.tensor([c for _, c in want])
        close(p, want.double(), want.double() * 2.0 ** -23 + 1e-38, "chance")


def logits(rows, n, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, n), generator=g) * spread
    few = torch.randint(0, n, (rows, 8), generator=g)
    return x.scatter_add_(1, few, torch.rand((rows, 8), generator=g) * 12).to(DT[dtype])


def uniform(rows, seed):
    return torch.rand(rows, generator=torch.Generator().manual_seed(seed)).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,n,skew", [(1, 1, 0), (3, 2, 0), (5, 7, 1), (4, 511, 0), (4, 512, 0), (4, 513, 3), (9, 5000, 0), (2, 50001, 0), (2, 131072, 8)])
def test_words_of_every_kind(part, dtype, rows, n, skew):
    x = logits(rows, n, dtype, n)
    for seed, more in enumerate((dict(), dict(temperature=[0.7] * rows), dict(top_k=[max(1, n // 3)] * rows), dict(top_k=[1 + i % 5 for i in range(rows)]), dict(top_p=[0.9] * rows), dict(top_p=[0.3] * rows),
                                 dict(min_p=[0.05] * rows), dict(temperature=[1.3] * rows, top_k=[200] * rows, top_p=[0.95] * rows, min_p=[0.01] * rows), dict(temperature=[0.0] * rows),
                                 dict(temperature=[3.0] * rows, top_p=[0.99] * rows))):
        sample_case(part, x, uniform(rows, seed), skew=skew, **more)


def test_a_row_of_the_longest(part):
    x = logits(1, 1 << 20, "bf16", 3)
    for more in (dict(), dict(top_k=[5000]), dict(top_p=[0.97])):
        sample_case(part, x, [0.77], **more)


def test_many_rows_with_wishes_of_their_own(part):
    rows, n = 300, 1000
    rng = np.random.default_rng(5)
    x = logits(rows, n, "bf16", 9)
    sample_case(part, x, uniform(rows, 1), temperature=np.where(rng.random(rows) < 0.2, 0, rng.uniform(0.3, 2, rows)).round(3).tolist(), top_k=rng.choice([0, -1, 1, 10, 999, 1000, 5000], rows).tolist(),
                top_p=rng.choice([1.0, 2.0, 0.9, 0.5, 0.01, 0.0, -1.0, float("nan")], rows).tolist(), min_p=rng.choice([0.0, -1.0, 0.1, 1.0, 3.0, float("nan")], rows).tolist())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [3, 1024, 1025, 5000, 40000])
def test_equal_logits_go_by_number(part, dtype, n):
    """All equal, two values, and few of many: the words of lower numbers stay."""
    x = torch.zeros((3, n))
    x[1, ::2] = -1.5
    x[2] = -4.0
    x[2, n // 2] = -0.0
    x[2, n // 3] = 0.0
    x = x.to(DT[dtype])
    for k in (1, 2, n // 2, n - 1):
        for u in (0.0, 0.5, 0.999):
            sample_case(part, x, [u] * 3, top_k=[k] * 3)
    for p in (0.25, 0.5, 0.75, 0.999):
        for u in (0.0, 0.37, 0.9999):
            sample_case(part, x, [u] * 3, top_p=[p] * 3)
            sample_case(part, x, [u] * 3, top_p=[p] * 3, top_k=[max(1, n // 2)] * 3)
    sample_case(part, x, [0.1] * 3, temperature=[0.0] * 3)


@pytest.mark.parametrize("dtype,n,skew", [("bf16", 131073, 1), ("fp32", 50001, 3), ("bf16", 8193, 0)])
def test_rows_of_many_parts_at_the_ends_of_the_random_numbers(part, dtype, n, skew):
    """A flat row and a steep one, whose words that are left are many and few; random numbers that only the smallest weights answer to."""
    x = torch.cat([logits(2, n, dtype, 12, 0.7), logits(2, n, dtype, 13, 6.0)])
    x[0, :20000] -= 30.0                                    # words of almost no weight in front
    x[1] = x[1].sort().values
    for u in (0.0, 1e-30, 2.0 ** -24, 0.5, 1 - 2.0 ** -24, 1.0):
        for more in (dict(), dict(top_k=[n - 1] * 4), dict(top_k=[600] * 4), dict(top_k=[9000] * 4, top_p=[0.8] * 4), dict(top_p=[0.999] * 4), dict(top_p=[0.9] * 4, min_p=[1e-4] * 4), dict(min_p=[1e-6] * 4)):
            sample_case(part, x, [u] * 4, skew=skew, **{k: [min(v, n) for v in w] for k, w in more.items()})


def test_many_short_rows_and_none(part):
    sample_case(part, logits(3000, 40, "bf16", 14), uniform(3000, 15), top_k=[7] * 3000)
    sample_case(part, logits(9, 8, "fp32", 16), uniform(9, 17), top_p=[0.5] * 9)
    word = torch.full((0,), 1, dtype=torch.int32, device="cuda")
    run(part, D.make_sample(torch.zeros((0, 30), device="cuda"), word, torch.zeros(0, device="cuda")))


def test_random_numbers_at_their_ends_and_between(part):
    x = torch.tensor([[0.0, 0.0, -math.inf, 0.0, 0.0, -100.0]]).repeat(9, 1)
    u = [0.0, 0.2499999, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1.0, 7.0, float("nan")]
    sample_case(part, x, u)
    assert [drawn(x[0], v if v == v else 0.0)[0] for v in u] == [0, 0, 1, 3, 4, 4, 4, 4, 0]
    sample_case(part, x[:3], [-1.0, 0.0, 0.3], chance=False)
    sample_case(part, x[:3], None)                          # without random numbers: the largest


def test_every_word_is_drawn_as_often_as_it_weighs(part):
    rows = 4096
    x = logits(1, 20, "fp32", 4, 1.0)
    p = torch.softmax(x.double()[0], 0)
    word = torch.empty(rows, dtype=torch.int32, device="cuda")
    run(part, D.make_sample(x.cuda().expand(rows, 20), word, (torch.arange(rows, device="cuda") + 0.5) / rows))
    assert float((torch.bincount(word.cpu().long(), minlength=20) / rows - p).abs().max()) <= 1 / rows     # random numbers at even distances


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_numbers(part, dtype):
    n, inf, nan = 1500, math.inf, math.nan
    x = logits(8, n, dtype, 6)
    x[0] = -inf
    x[1] = nan
    x[2, 700:] = -inf
    x[3, 10] = inf
    x[3, 1200] = inf
    x[4] = -inf
    x[4, 1499] = -3.0e38
    x[5, ::3] = nan
    x[6] = torch.tensor(-3.0e38)
    x[7, :] = torch.tensor(1.0e38)
    x[7, 5] = torch.tensor(3.0e38)
    for more in (dict(), dict(top_k=[3] * 8), dict(top_p=[0.6] * 8), dict(min_p=[0.5] * 8), dict(temperature=[0.0] * 8), dict(temperature=[inf] * 8, top_p=[0.5] * 8), dict(temperature=[1e-30] * 8, top_k=[2] * 8),
                 dict(temperature=[1e38] * 8, top_k=[700] * 8, top_p=[0.4] * 8), dict(temperature=[nan] * 8)):
        sample_case(part, x, uniform(8, 2), **more)


def test_logits_near_zero(part):
    """A step of the exponent that holds both signs and all sizes of numbers, in temperatures as small."""
    g = torch.Generator().manual_seed(8)
    x = (torch.randn((4, 30000), generator=g) * torch.exp2(torch.randint(-60, 0, (4, 30000), generator=g).float())).float()
    x[1] *= 1e-3
    x[2] *= 1e-30
    x[3] *= 1e-36
    for t in (1.0, 1e-3, 1e-30, 1e-37):
        for more in (dict(top_k=[9000] * 4), dict(top_p=[0.3] * 4), dict(top_k=[20000] * 4, top_p=[0.7] * 4)):
            sample_case(part, x, uniform(4, 3), temperature=[t] * 4, **more)


# ---- accept -----------------------------------------------------------------------------------------------------------------------


def accept_case(part, seed, rows, vocabulary=3, masks=None, before=True, in_place=False, spare=0, words=None, least=-1):
    rng = np.random.default_rng(seed)
    masks = trees(seed, rows, words) if masks is None else masks
    n, s = sum(rows), len(rows)
    w, a = (torch.from_numpy(rng.integers(least, vocabulary, n + spare).astype(np.int32)) for _ in range(2))
    b = torch.from_numpy(rng.integers(0, 1000, s).astype(np.int32))
    start = torch.tensor(np.cumsum([0] + rows), dtype=torch.int32)
    path = torch.full((n + spare,), -9, dtype=torch.int32, device="cuda")
    count, word, after = (torch.full((s,), -9, dtype=torch.int32, device="cuda") for _ in range(3))
    bd = b.cuda()
    if in_place:
        after = bd
    more = torch.zeros((spare, masks.shape[1]), dtype=torch.int64)
    run(part, D.make_accept(torch.cat([masks, more]).cuda(), w.cuda(), a.cuda(), path, count, word, row_start=None if rows == [1] * s else start.cuda(), before=bd if before else None,
                            after=after if before else None))
    at = 0
    for i, r in enumerate(rows):
        line, last = walk(masks[at:at + r], w[at:at + r].tolist(), a[at:at + r].tolist())
        assert path[at:at + r].tolist() == line + [-1] * (r - len(line)), (seed, i)
        assert int(count[i]) == len(line) and int(word[i]) == last and (not before or int(after[i]) == int(b[i]) + len(line)), (seed, i)
        at += r
    assert bool((path[n:] == -9).all()), "rows of no sequence"
    return count.cpu()


def test_walks(part):
    longest = 0
    for seed in range(8):
        longest = max(longest, int(accept_case(part, seed, [26], 1 + seed % 3).max()))
        accept_case(part, seed, np.random.default_rng(seed).integers(0, 64, 40).tolist(), 2, spare=3)
        longest = max(longest, int(accept_case(part, seed, [65, 0, 200, 64, 1, 63, 128], 1).max()))
    assert longest >= 4
    for seed in range(4):                                   # every word fits: the first node below
        accept_case(part, seed, [65, 0, 200, 64, 1, 63, 1024], 1, least=0)
    accept_case(part, 9, [300] * 9, 2, least=0)
    accept_case(part, 1, [1, 1, 1], 2)
    accept_case(part, 2, [30, 4], 1, in_place=True)
    accept_case(part, 3, [30, 4], 1, before=False)
    accept_case(part, 4, [100, 7], 1, words=16)
    accept_case(part, 5, [1024], 1)
    accept_case(part, 6, [0, 0], masks=torch.zeros((0, 1), dtype=torch.int64))
    accept_case(part, 7, [3] * 3000, 2)


def test_chains_and_bushes(part):
    accept_case(part, 11, [900, 64], 1, masks=D.tree_masks([list(range(-1, 899)), list(range(-1, 63))]))
    whole = accept_case(part, 11, [900, 64], 1, masks=D.tree_masks([list(range(-1, 899)), list(range(-1, 63))]), least=0)
    assert whole.tolist() == [900, 64]
    accept_case(part, 12, [200, 64], 4, masks=D.tree_masks([[-1] + [0] * 199, [-1] + [0] * 63]))
    # more rows than the masks have bits: those behind are no nodes
    masks = torch.zeros((90, 1), dtype=torch.int64)
    for i in range(90):
        masks[i] = (1 << min(i + 1, 63)) - 1
    accept_case(part, 13, [90], 1, masks=masks)


# ---- keep and copy ----------------------------------------------------------------------------------------------------------------


def keep_case(part, seed, before, rows, path, count, kv=2, dim=64, edit=None, extra=0):
    c = Cache(seed, before, rows, kv, dim).filled(seed + 1)
    g = torch.Generator().manual_seed(seed + 2)
    for t in (c.k_scale, c.v_scale):                        # sixteenths of unequal scales
        t.view(torch.uint8).copy_(torch.randint(118, 128, t.shape, generator=g))
    if edit:
        edit(c)
    path = path + [-5] * extra
    cache = c.gpu(D)
    run(part, D.make_keep(cache, torch.tensor(path, dtype=torch.int32, device="cuda"), torch.tensor(count, dtype=torch.int32, device="cuda"),
                          row_start=None if rows == [1] * len(rows) else c.start.cuda()))
    want = kept(c, path, count)
    for name, got in zip(("k", "v", "k_scale", "v_scale"), c.on_gpu):
        if "scale" in name:
            assert torch.equal(got.cpu().view(torch.uint8), want[name].view(torch.uint8)), name
        else:
            same_codes(got, want[name], name)
    return any(not torch.equal(want[n].view(torch.uint8), getattr(c, n).view(torch.uint8)) for n in want)


def some_path(rng, rows, counts):
    path = []
    for r, n in zip(rows, counts):
        line = sorted(rng.choice(np.arange(1, r), n - 1, replace=False).tolist()) if n > 1 else []
        path += ([0] + line + [-1] * (r - n))[:r]
    return path


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("before,rows,count", [([100], [26], [5]), ([0], [64], [9]), ([63, 15, 200], [20, 33, 7], [3, 17, 6]), ([40], [200], [90]), ([61], [130], [40]), ([5, 5], [1, 1], [1, 1])])
def test_kept_tokens(part, dim, before, rows, count):
    for seed in range(3):
        rng = np.random.default_rng(seed + dim)
        changed = keep_case(part, seed, before, rows, some_path(rng, rows, count), count, 2, dim)
    assert changed or max(rows) == 1


def test_paths_that_move_nothing_or_end_early(part):
    assert not keep_case(part, 1, [30], [20], list(range(20)), [9])
    assert not keep_case(part, 2, [30], [20], [0] + [-1] * 19, [1])
    assert not keep_case(part, 3, [30], [20], [3, 9, 11] + [-1] * 17, [0])
    assert not keep_case(part, 4, [30], [20], [-1] * 20, [5])
    assert keep_case(part, 5, [30], [20], [0, 4, 4, 9] + [-1] * 16, [4])           # the third does not increase
    assert keep_case(part, 6, [30], [20], [2, 5, 20, 21] + [-1] * 16, [7])         # ... is no row
    assert keep_case(part, 7, [30], [20], [0, 1, 2, 7, 3] + [-1] * 15, [-4 + 9])
    assert not keep_case(part, 8, [30, 9], [20, 4], [3] * 24, [-1, -2 ** 31])
    assert keep_case(part, 9, [30, 0, 9], [3, 0, 4], [1, 2, 3, 0, 2, 3, 9], [2 ** 31 - 1, 5, 100], extra=5)


def test_kept_tokens_whose_pages_are_not_there(part):
    rows, before = [150], [50]
    path = [0, 3, 20, 70, 71, 90, 100, 140] + list(range(141, 149)) + [-1] * 134
    for entry in (0, 1, 2, 3):
        def edit(c):
            c.pages[0, entry] = -1 if entry % 2 else 10 ** 6
        keep_case(part, 20 + entry, before, rows, path, [16], edit=edit)
    keep_case(part, 25, [-4, 20], [30, 3], some_path(np.random.default_rng(1), [30, 3], [12, 2]), [12, 2])


def test_numbers_that_are_not_finite_stay_so(part):
    def edit(c):
        c.k.view(torch.uint8)[:, :, ::5, ::7] = 0x7F
        c.v.view(torch.uint8)[:, :, ::7, ::5] = 0xFF
        c.k_scale.view(torch.uint8)[::2] = 27
        c.v_scale.view(torch.uint8)[::2] = 200
    assert keep_case(part, 30, [40], [40], some_path(np.random.default_rng(2), [40], [15]), [15], edit=edit)


@pytest.mark.parametrize("kv,dim,pages,pairs", [(1, 64, 5, [(0, 4)]), (3, 128, 9, [(8, 0), (1, 2), (1, 3)]), (8, 128, 4, [(2, 1)]), (12, 256, 6, [(5, 0), (3, 3)]), (2, 64, 300, [(i, 299 - i) for i in range(150)]),
                                                (2, 64, 7, [(-1, 3), (3, 7), (2, 5), (2 ** 31 - 1, 0), (0, -2 ** 31)]), (1, 64, 3, [])])
def test_copied_pages(part, kv, dim, pages, pairs):
    c = Cache(7, [PAGE * pages - 1], [1], kv, dim, spare_pages=0)
    want = {n: getattr(c, n).view(torch.uint8).clone() for n in ("k", "v", "k_scale", "v_scale")}
    for a, b in pairs:
        if 0 <= a < pages and 0 <= b < pages:
            for n in want:
                want[n][b] = getattr(c, n).view(torch.uint8)[a]
    run(part, D.make_copy(c.gpu(D), torch.tensor(pairs, dtype=torch.int32, device="cuda").view(-1, 2)))
    for n, got in zip(want, c.on_gpu):
        assert torch.equal(got.cpu().view(torch.uint8), want[n]), n


# ---- the step ---------------------------------------------------------------------------------------------------------------------


def test_a_drafted_step_in_one_list(part):
    """append -> attend -> sample -> accept -> keep, then a token behind what was kept: the next step sees the kept tokens and nothing else."""
    kv, heads, dim, vocabulary = 2, 4, 64, 50
    before, rows = [70, 0, 300], [26, 13, 40]
    n, masks = sum(rows), trees(81, rows)
    c = Cache(81, before, rows, kv, dim)
    cache, start, table = c.gpu(D), c.start.cuda(), turn_table(400, dim).cuda()
    qkv = rand((n, heads + 2 * kv, dim), torch.bfloat16, 82).cuda()
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    out, word = torch.empty((n, heads, dim), dtype=torch.bfloat16, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    x = logits(n, vocabulary, "bf16", 83).cuda()
    u = torch.tensor(uniform(n, 84), device="cuda")
    tree = masks.cuda()
    path, (count, last, after) = torch.empty(n, dtype=torch.int32, device="cuda"), (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(3))
    answers = torch.tensor([drawn(x[i].cpu(), float(u[i]))[0] for i in range(n)], dtype=torch.int32)
    words = torch.randint(0, vocabulary, (n,), generator=torch.Generator().manual_seed(85), dtype=torch.int32)
    for s, r in enumerate(rows):                            # drafts that stand, most of them
        for i in range(1, r):
            at = int(c.start[s]) + i
            parent = bits_of(masks[at].tolist())[-2]
            if i % 4:
                words[at] = answers[int(c.start[s]) + parent]
    plan = D.make_ops([D.make_append(cache, k, v, row_start=start, q=q, q_out=q, turn=table, rot_dim=dim, tree=tree), D.make_attend(cache, q, out, row_start=start, scale=0.1, tree=tree),
                       D.make_sample(x, word, u), D.make_accept(tree, words.cuda(), word, path, count, last, row_start=start, before=c.on_gpu[5], after=after), D.make_keep(cache, path, count, row_start=start)])
    D.daris_run_ops(plan, part)
    assert torch.equal(word.cpu(), answers)
    lines = [walk(masks[int(c.start[s]):int(c.start[s]) + r], words[int(c.start[s]):int(c.start[s]) + r].tolist(), answers[int(c.start[s]):int(c.start[s]) + r].tolist()) for s, r in enumerate(rows)]
    assert count.tolist() == [len(line) for line, _ in lines] and last.tolist() == [w for _, w in lines] and max(count.tolist()) >= 4
    assert after.tolist() == [b + len(line) for b, (line, _) in zip(before, lines)]
    # attention over what the append alone leaves
    fresh = rand((n, heads + 2 * kv, dim), torch.bfloat16, 82).cuda()
    names = ("k", "v", "k_scale", "v_scale")

    def back(cache):
        for name, g in zip(names, cache.on_gpu):
            setattr(cache, name, g.cpu())
    e = Cache(81, before, rows, kv, dim)
    f = fresh.clone()
    run(part, D.make_append(e.gpu(D), f[:, heads:heads + kv], f[:, heads + kv:], row_start=start, q=f[:, :heads], q_out=f[:, :heads], turn=table, rot_dim=dim, tree=tree))
    back(e)
    assert torch.equal(q, f[:, :heads])
    want, slack = attend_tree(e, masks, q, 0.1, 0, "bf16")
    close(out, want, slack, "attention")
    # the kept nodes appended row by row
    stay = torch.tensor([int(c.start[s]) + i for s, (line, _) in enumerate(lines) for i in line], device="cuda")
    d = Cache(81, before, rows, kv, dim)
    other = d.gpu(D)
    fewer = torch.tensor(np.cumsum([0] + [len(line) for line, _ in lines]), dtype=torch.int32, device="cuda")
    f = fresh[stay].contiguous()
    run(part, D.make_append(other, f[:, heads:heads + kv], f[:, heads + kv:], row_start=fewer, q=f[:, :heads], q_out=f[:, :heads], turn=table, rot_dim=dim))
    assert torch.equal(q[stay], f[:, :heads]), "kept nodes are turned as rows that follow each other"
    back(c)
    back(d)
    for s, (line, _) in enumerate(lines):
        got, want = c.tokens(s, before[s] + len(line)), d.tokens(s, before[s] + len(line))
        for name, a, b, scales in (("k", got[0], want[0], c.k_scale), ("v", got[1], want[1], c.v_scale)):
            # scales may be larger than those of the kept tokens alone (a rejected one's): two roundings on either side
            close(a, b, 4 * e4m3_slack(b, two_to(scales)[c.pages[s][c.pages[s] >= 0].long()].max()), name)


def test_keys_and_values_that_lie_apart(part):
    """With a tree, k and v have the same distances; of one row or one head the distance does not count."""
    c = Cache(95, [3], [1], 2, 64)
    cache, tree = c.gpu(D), torch.ones((1, 1), dtype=torch.int64, device="cuda")
    k, v = torch.randn((1, 2, 64), device="cuda"), torch.randn((1, 4, 64), device="cuda")[:, :2]
    run(part, D.make_append(cache, k, v, row_start=c.start.cuda(), tree=tree))
    back = [t.cpu() for t in c.on_gpu[:4]]
    page, s = int(c.pages[0, 0]), two_to(back[3])
    close(back[1][page, :, :, 3].double() * s[page, :, 0, None], v[0].cpu().double(), e4m3_slack(v[0].cpu().double(), s[page, :, 0, None]), "values")
    with pytest.raises(D.DarisError):
        D.make_append(cache, torch.zeros((2, 2, 64), device="cuda"), torch.zeros((2, 4, 64), device="cuda")[:, :2], row_start=c.start.cuda(), tree=torch.ones((2, 1), dtype=torch.int64, device="cuda"))
    for wrong in (lambda: D.make_attend(cache, k.repeat(1, 2, 1), k.repeat(1, 2, 1), tree=tree[:, :0]), lambda: D.make_attend(cache, k, torch.empty_like(k), tree=tree.repeat(2, 1)),
                  lambda: D.make_attend(cache, k, torch.empty_like(k), tree=tree.int()), lambda: D.make_sample(k[0], torch.zeros(2, device="cuda")), lambda: D.make_copy(cache, tree.int()),
                  lambda: D.make_keep(cache, tree.int()[0], torch.zeros(3, dtype=torch.int32, device="cuda")), lambda: D.make_sample(k[0], torch.zeros(2, dtype=torch.int32, device="cuda"), top_k=torch.zeros(2, device="cuda"))):
        with pytest.raises(D.DarisError) as e:
            wrong()
        assert e.value.code == D.EINVAL


def test_plans_of_two_partitions_take_turns(part):
    """Sampling of long rows and cut attention share a partition's workspace with each other, and none with another partition's."""
    x, u = logits(6, 40000, "bf16", 96).cuda(), torch.tensor(uniform(6, 97), device="cuda")
    words = [torch.full((6,), -5, dtype=torch.int32, device="cuda") for _ in range(2)]
    c = Cache(98, [3000, 100], [30, 9], 1, 64).filled(99)
    masks, q = trees(98, [30, 9]), rand((39, 4, 64), torch.bfloat16, 100, 0.3).cuda()
    outs = [torch.zeros_like(q) for _ in range(2)]
    cache = c.gpu(D)
    lists = [D.make_ops([D.make_sample(x, words[i], u, top_p=torch.full((6,), 0.9, device="cuda")), D.make_attend(cache, q, outs[i], row_start=c.start.cuda(), scale=0.02, tree=masks.cuda()),
                         D.make_sample(x, words[i], u, top_p=torch.full((6,), 0.9, device="cuda"))]) for i in range(2)]
    want = [drawn(x[i].cpu(), float(u[i]), top_p=float(np.float32(0.9)))[0] for i in range(6)]
    ref, slack = attend_tree(c, masks, q, 0.02, 0, "bf16")
    for _ in range(3):
        for i, place in ((0, part), (1, SMALL)):
            words[i].fill_(-5)
            outs[i].zero_()
            D.daris_run_ops(lists[i], place)
            assert words[i].tolist() == want
            close(outs[i], ref, slack, "attention")


def test_lists_that_are_not_planned_give_the_same(part):
    c = Cache(91, [60, 7], [9, 5], 1, 64)
    n, masks = 14, trees(91, [9, 5]).cuda()
    cache, start = c.gpu(D), c.start.cuda()
    first = [t.clone() for t in c.on_gpu[:4]]
    qkv = rand((n, 4, 64), torch.float32, 92).cuda()
    q, out = qkv[:, :2].contiguous(), torch.empty((n, 2, 64), device="cuda")
    x, u = logits(n, 300, "fp32", 93).cuda(), torch.tensor(uniform(n, 94), device="cuda")
    word, path, (count, last) = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda"), (torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(2))
    ops = D.make_ops([D.make_append(cache, qkv[:, 2:3], qkv[:, 3:], row_start=start, tree=masks), D.make_attend(cache, q, out, row_start=start, scale=0.1, tree=masks), D.make_sample(x, word, u, top_k=torch.full((n,), 20, dtype=torch.int32, device="cuda")),
                      D.make_accept(masks, word, word, path, count, last, row_start=start), D.make_keep(cache, path, count, row_start=start),
                      D.make_copy(cache, torch.tensor([[0, 3], [1, 4]], dtype=torch.int32, device="cuda"))])
    outs = [out, word, path, count, last] + [t.view(torch.uint8) for t in c.on_gpu[:4]]
    results = []
    for place, planned in ((part, True), (part, False), (SMALL, True), (part, True)):
        for t, f in zip(c.on_gpu[:4], first):
            t.view(torch.uint8).copy_(f.view(torch.uint8))
        torch.cuda.synchronize()
        if planned:
            D.daris_run_ops(ops, place)
        else:
            assert D.lib().daris_run_ops(ops.array, len(ops), place) == 0
        results.append([t.clone() for t in outs])
    for r in results[1:]:
        for a, b in zip(results[0], r):
            assert torch.equal(a, b) or (a.dtype == torch.float32 and float((a - b).abs().max()) < 1e-4)


def test_pages_behind_four_gigabytes(part):
    """The last pages of a cache of 70000: what each operator does there is what it does in a small cache."""
    kv, dim, n = 8, 128, 70000
    c = Cache(111, [70, 130], [26, 40], kv, dim).filled(112)
    small = c.gpu(D)
    few = c.k.shape[0]
    big = []
    for t in c.on_gpu[:4]:
        b = torch.zeros((n,) + tuple(t.shape[1:]), dtype=torch.uint8, device="cuda")
        b[n - few:] = t.view(torch.uint8)
        big.append(b.view(t.dtype))
    assert big[0].numel() > 1 << 32
    large = D.make_cache(*big, torch.where(c.pages >= 0, c.pages + n - few, c.pages).cuda(), c.on_gpu[5])
    rows, start, masks = 66, c.start.cuda(), trees(113, [26, 40]).cuda()
    qkv = rand((rows, 4 * kv, dim), torch.bfloat16, 114).cuda()
    path, count = torch.tensor(some_path(np.random.default_rng(115), [26, 40], [6, 9]), dtype=torch.int32, device="cuda"), torch.tensor([6, 9], dtype=torch.int32, device="cuda")
    outs = []
    for cache, base, held in ((small, 0, c.on_gpu), (large, n - few, big)):
        out = torch.empty((rows, 2 * kv, dim), dtype=torch.bfloat16, device="cuda")
        run(part, D.make_append(cache, qkv[:, 2 * kv:3 * kv], qkv[:, 3 * kv:], row_start=start, tree=masks), D.make_attend(cache, qkv[:, :2 * kv], out, row_start=start, scale=0.05, tree=masks),
            D.make_keep(cache, path, count, row_start=start), D.make_copy(cache, torch.tensor([[base, base + few - 1]], dtype=torch.int32, device="cuda")))
        outs.append([out] + [t.view(torch.uint8)[base:] for t in held[:4]])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert not bool(big[0].view(torch.uint8)[:n - few].any()) and not bool(big[1].view(torch.uint8)[:n - few].any())
