"""Words of long rows whose weights lie far apart (daris_sample), against the definition in whole numbers (draft_helpers.drawn)."""

import math

import numpy as np
import pytest
import torch

import paper_2504_08795_amd as D
from draft_helpers import drawn
from step_helpers import DT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(256)
    D.daris_shutdown()


def words(part, x, u, **more):
    """The words of rows x [rows][n] by the lists u, top_k, ..., and those of the definition."""
    f = lambda v, t=torch.float32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    word = torch.full((len(x),), -7, dtype=torch.int32, device="cuda")
    D.daris_run_ops(D.make_ops([D.make_sample(x.cuda(), word, f(u), **{k: f(v, torch.int32 if k == "top_k" else torch.float32) for k, v in more.items()})]), part)
    single = lambda v, i: float(np.float32(v[i]))  # noqa: E731
    return word.tolist(), [drawn(x[i], single(u, i), **{k: v[i] if k == "top_k" else single(v, i) for k, v in more.items()})[0] for i in range(len(x))]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("far", [44.375, 44.5, 44.75])
def test_top_p_counts_where_top_k_ends_among_words_of_no_weight(part, dtype, far):
    """Three heavy words in a row's first numbers and 2^-64 or less of them everywhere else: the top_k likeliest reach into those, top_p does not."""
    x = torch.zeros((4, 50001))
    x[:, 5], x[:, 900], x[:, 7000] = far, far - 0.25, far - 0.5
    x[3, 30000:] = -1.0
    got, want = words(part, x.to(DT[dtype]), [0.0, 0.7, 0.999, 0.999], top_k=[10000, 10000, 49000, 20000], top_p=[0.3, 0.3, 0.3, 0.6])
    assert got == want


@pytest.mark.parametrize("n,rows", [(40, 200), (3000, 40), (50001, 6)])
def test_random_numbers_from_1_on_give_the_last_word_however_little_it_weighs(part, n, rows):
    """The words behind two thirds of a row weigh less than the last bit of the sum in front of them."""
    x = torch.randn((rows, n), generator=torch.Generator().manual_seed(n))
    x[:, n - n // 3:] -= 40.0
    for u in (1.0, 1.5, 1e30):
        for more in (dict(), dict(top_k=[n - 1] * rows), dict(temperature=[0.95] * rows), dict(min_p=[1e-19] * rows)):
            got, want = words(part, x, [u] * rows, **more)
            assert got == want, (u, more)


def test_top_p_among_a_million_words_that_together_weigh_a_thousandth_of_the_first(part):
    """One word, and equal ones of 2^-30.3 of it: each of them has its part in the sums, to a last word that is told from its neighbours."""
    n = 1 << 20
    x = torch.full((3, n), -21.0)
    x[0, 600000] = x[1, 0] = x[2, n - 1] = 0.0
    last = 1 - 2.0 ** -24
    got, want = words(part, x, [last] * 3, top_p=[0.9995, 0.9993, 0.9999])
    assert got == want and 100 < abs(want[1] - want[0]) < n - 1000
    got, want = words(part, x[:2], [1 - 2.0 ** -13, last], top_k=[n // 2, n - 7])
    assert got == want


@pytest.mark.parametrize("u", [2.0 ** -36, 2.0 ** -37, 1.3 * 2.0 ** -38])
def test_many_parts_of_little_weight_come_to_what_a_random_number_asks(part, u):
    """A word of 2^-42.5 in each 8192 numbers, and one of weight 1 behind them."""
    n = 1 << 20
    x = torch.full((1, n), -math.inf)
    x[0, 17:n - 8192:8192] = -42.5 * math.log(2.0)
    x[0, n - 5] = 0.0
    got, want = words(part, x, [u], top_k=[n - 1])
    assert got == want and want[0] < n - 8192


def test_words_of_no_weight_have_no_part_in_the_sum_that_a_small_random_number_passes(part):
    """Words of just under 2^-40, each among 8191 of less than 2^-64: eight of them do not pass 2^-37, for which 511 others beside each would be enough."""
    n = 1 << 20
    x = torch.full((1, n), -44.4)
    x[0, 17:n - 8192:8192] = -40 * math.log(2.0) - 2.0 ** -16
    x[0, n - 5] = 0.0
    assert 8 * math.exp(float(x[0, 17])) < 2.0 ** -37 < 8 * math.exp(float(x[0, 17])) + 7 * 511 * math.exp(-44.4) and math.exp(-44.4) < 2.0 ** -64
    for more in (dict(top_k=[n - 1]), dict()):
        got, want = words(part, x, [2.0 ** -37], **more)
        assert got == want == [17 + 8 * 8192], more


@pytest.mark.parametrize("n", [9, 700, 20001])
def test_min_p_of_1_leaves_all_that_weigh_1(part, n):
    """Logits so near each other, or a temperature so high, that their weights are 1 in 64 bits, and two that weigh less."""
    x = torch.randn((4, n), generator=torch.Generator().manual_seed(n))
    x[0] *= 1e-30
    x[1] *= 1e-20
    x[:, n // 3] = x[:, n // 2] = torch.tensor([-1.0, -1e-3, -3.0e38, -1e30])
    for u in (0.0, 0.37, 0.9999, 1.0):
        for more in (dict(), dict(top_k=[n - 2] * 4), dict(top_p=[0.7] * 4)):
            got, want = words(part, x, [u] * 4, temperature=[1.0, 0.5, 1e30, math.inf], min_p=[1.0] * 4, **more)
            assert got == want, (u, more)
    assert got[0] not in (n // 3, n // 2)
