"""The operators of a generation step at the ends of their numbers' ranges, against 64 bits."""
import pytest
import torch

import paper_2504_08795_amd as D
from step_helpers import PAGE, Cache, close, matvec
from test_gpu_steps import attend_case, rand, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def parts():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(256), D.daris_create_partition(8)
    D.daris_shutdown()


# ---- attend ---------------------------------------------------------------------------------------------------------------------


def zeros_beside(byte, is_zero):
    """Values of all pages: zeros under the smallest scale where is_zero(token), the others under 2^(byte - 127)."""
    def edit(c):
        for s in range(len(c.before)):
            for e in range(c.pages.shape[1]):
                page = int(c.pages[s, e])
                for i in range(4):
                    zero = is_zero(e * PAGE + i * 16)
                    if page >= 0:
                        c.v_scale.view(torch.uint8)[page, :, i] = 27 if zero else byte
                        if zero:
                            c.v.view(torch.uint8)[page, :, :, i * 16:i * 16 + 16] = 0
    return edit


# what the outputs take from each token is the same wherever the zeros lie: on a wave's first pages, its last ones, a wave's of four, a sixteenth of each page, a unit
ZEROS = {"first pages": lambda t: t < 320, "last pages": lambda t: t >= 320, "every fourth page": lambda t: t // 64 % 4 == 0, "all but every fourth": lambda t: t // 64 % 4 != 2,
         "first of a page": lambda t: t % 64 < 16, "last of a page": lambda t: t % 64 >= 48}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("where", list(ZEROS))
@pytest.mark.parametrize("byte", [120, 160, 240])
def test_zeros_beside_large_values_keep_their_weights(parts, dtype, where, byte):
    edit = zeros_beside(byte, ZEROS[where])
    for q_scale in (0.0, 1.0):
        attend_case(parts[0], 10, [639], [1], 1, 3, 64, dtype, edit=edit, q_scale=q_scale)                       # four waves' pages
        attend_case(parts[1], 11, [500, 610], [30, 30], 1, 16, 128 if q_scale else 64, dtype, edit=edit, q_scale=q_scale)     # wide tiles
    attend_case(parts[0], 12, [639], [2], 2, 1, 256, dtype, edit=edit)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("zero", [lambda t: t < 3000, lambda t: t >= 3000])
def test_units_of_zeros_keep_their_weights(parts, dtype, zero):
    attend_case(parts[0], 20, [6000], [1], 1, 2, 64, dtype, edit=zeros_beside(220, zero))
    attend_case(parts[1], 21, [4000], [65], 1, 12, 64, dtype, edit=zeros_beside(220, zero))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_table_of_rows_that_decreases_spoils_no_later_call(parts, dtype):
    # 160 rows three times (the last time 40 of them, behind 6360 tokens): 20 tiles of one unit and 3 of 5, of which 32 units are launched -- two of the last tile
    starts, before, units = [0, 160, 0, 160, 0, 40], [0, 0, 0, 0, 6360], 160 // 16 + 5 + 16 + 1
    pages = [-(-(b + max(0, y - x)) // PAGE) for b, x, y in zip(before, starts, starts[1:])]
    tiles = [-(-max(0, y - x) // 16) for x, y in zip(starts, starts[1:])]
    per = (-(-int(sum(t * q for t, q in zip(tiles, pages)) * 1.0001 + 1) // 16) + 3) // 4 * 4
    firsts = [20 + i * -(-pages[4] // per) for i in range(tiles[4])]
    assert tiles == [10, 0, 10, 0, 3] and -(-pages[4] // per) == 5 and firsts[2] < units < firsts[2] + 5
    c = Cache(30, before, [160, 0, 0, 0, 40], 1, 64).filled(31)
    q = rand((160, 1, 64), dtype, 32).cuda()
    out = torch.zeros_like(q)
    run(parts[1], D.make_attend(c.gpu(D), q, out, row_start=torch.tensor(starts, dtype=torch.int32).cuda(), scale=0.1))
    # a tile whose units meet at the counter of that last one
    name = "bf16" if dtype == torch.bfloat16 else "fp32"
    attend_case(parts[1], 33, [10] * firsts[2] + [9000], [1] * (firsts[2] + 1), 1, 2, 64, name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30 + 1, 2 ** 30])
def test_windows_that_reach_everything(parts, dtype, window):
    attend_case(parts[0], 40, [-5], [8], 1, 1, 64, dtype, window)
    attend_case(parts[0], 41, [0, 100], [40, 3], 1, 2, 64, dtype, window)
    attend_case(parts[1], 42, [0, -5], [90, 80], 2, 4, 64, dtype, window)
    attend_case(parts[1], 43, [300], [130], 2, 5, 128, dtype, window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_narrow_tiles_of_prompts_stay_whole(parts, dtype):
    attend_case(parts[1], 50, [70], [40], 1, 16, 256, dtype)                                    # one sequence, more tiles than places
    attend_case(parts[1], 51, [70, 0, 200], [300, 1, 41], 8, 6, 256, dtype, window=50)          # 128 a key head, 64 for each of its two places


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [40, 63, 64, 65, 100, 127, 128, 129, 200])
def test_wide_tiles_in_less_and_more_than_two_rounds(parts, dtype, rows):
    attend_case(parts[1], 55, [70], [rows], 1, 16, 64, dtype)               # 8 tiles of 128 columns have a CU each
    attend_case(parts[1], 56, [300, 10], [rows, 50], 1, 16, 64, dtype, window=90)


# ---- 4-bit products -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows,n,k,group", [(3, 40, 512, 128), (16, 17, 4096, 64), (1, 4096, 256, 32), (1, 40, 25088, 128)])
@pytest.mark.parametrize("one_sign", [False, True])
def test_rows_of_the_largest_numbers(parts, rows, n, k, group, one_sign):
    g = torch.Generator().manual_seed(60 + rows)
    w = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8)
    ws = (torch.rand((n, k // group), generator=g) * (0.1 / k)).bfloat16()                # the sizes of all terms together stay below 0.8 of the largest number
    x = (torch.rand((rows, k), generator=g) * 0.1 + 0.9) * 3.38e38
    if not one_sign:
        x *= torch.randint(0, 2, (rows, k), generator=g) * 2 - 1
    x = x.bfloat16()
    assert bool(torch.isfinite(x).all())
    y = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    run(parts[0], D.make_matvec(x.cuda(), w.cuda(), ws.cuda(), y))
    want, slack = matvec(x.double(), w, ws, False, "bf16")
    close(y, want, slack, "y")
