"""Attention on partitions so small that narrow tiles do not fit them at once: wide tiles, in whole and in units, against 64 bits."""
import pytest
import torch

import paper_2504_08795_amd as D
import test_gpu_steps as steps
from test_gpu_steps import attend_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def parts():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(8), D.daris_create_partition(24)
    D.daris_shutdown()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 70])
def test_chunks_of_a_prompt(parts, dtype, dim, window):
    for p in parts:
        steps.test_attend_chunks_of_a_prompt(p, dtype, dim, window)
    attend_case(parts[0], 890, [130, 0], [70, 33], 2, 6, dim, dtype, window)
    attend_case(parts[0], 891, [300], [130], 2, 5, dim, dtype, window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [0, 900])
def test_units_of_a_tile(parts, dtype, window):
    p = parts[0]
    attend_case(p, 900, [4000], [65], 1, 12, 64, dtype, window)                       # 7 tiles in 16 units
    attend_case(p, 901, [1500], [80], 1, 14, 128, dtype, window)
    attend_case(p, 902, [20, 2600, 0, 70], [33, 34, 40, 70], 1, 6, 64, dtype, window)  # one sequence of four is long
    attend_case(p, 903, [2600, 0, 1], [40, 33, 40], 2, 5, 128, dtype, window)


def test_a_long_sequence_among_short_ones_in_many_units(parts):
    attend_case(parts[0], 910, [9000] + [0] * 3, [32] * 4, 1, 7, 64, "bf16")
    attend_case(parts[0], 911, [0, 9000], [230, 32], 1, 4, 128, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_masks_nans_and_sizes(parts, dtype):
    for p in parts:
        steps.test_attend_nothing_and_pages_that_are_not_there(p, dtype, [200, 3, 60, 190])
        for rows, window in (([80], 0), ([80], 20), ([400], 0), ([400], 200)):
            steps.test_attend_nan_only_where_it_is_seen(p, dtype, rows, window)
        steps.test_attend_sizes_of_queries_and_scales(p, dtype)
        attend_case(p, 920, [100], [300], 1, 3, 64, dtype, strided=True)
        attend_case(p, 921, [200], [90], 1, 12, 128, dtype, scale=-0.05)
        steps.test_attend_nan_on_pages_that_every_row_sees(p, dtype, 128, [140], [260], 4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("seqs", [3, 8, 12, 15, 16, 40])
def test_cuts_of_tiles_alike(parts, dtype, seqs):
    # narrow tiles, fewer than the partition's places, as many and more
    attend_case(parts[0], 930, [300] * seqs, [2] * seqs, 1, 8, 64, dtype)
    attend_case(parts[0], 931, [300 + 61 * i for i in range(seqs)], [1] * seqs, 1, 4, 64, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("seqs", [64, 65, 256, 257, 530])
def test_more_sequences_than_a_wave_holds(parts, dtype, seqs):
    before = [(37 * i) % 130 for i in range(seqs)]
    attend_case(parts[1], 940 + seqs, before, [1] * seqs, 1, 2, 64, dtype, gpu_start=False)
    attend_case(parts[1], 941 + seqs, before[:-1] + [700], [(5 * i) % 3 for i in range(seqs - 1)] + [2], 1, 1, 64, dtype)
