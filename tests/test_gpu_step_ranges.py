"""The operators of a generation step at the ends of their numbers' ranges, against 64 bits."""
import pytest
import torch

import paper_2504_08795_amd as D
from step_helpers import PAGE
from test_gpu_steps import attend_case

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
