"""Launches and refusals of the operators of a generation step at the ends of their ranges, on the host.  No GPU."""
import pytest
import torch

import paper_2504_08795_amd as D
from lib_helpers import Session
from paper_2504_08795_amd import binding as B
from test_host_steps import HOST, attend, cache, encode, norm  # noqa: F401 (encode: a fixture)


def test_the_workspace_of_attention_does_not_grow_with_the_rows_of_prompts(encode):  # noqa: F811
    # an 8-bit cache's page is 32 KB a key head of 256: a workspace of a few hundred MB is a few long streams'
    asked = [(rows, seqs, heads, kv, dim, dtype, 256) for dim in (64, 128, 256) for dtype in (0, 1) for kv, heads in ((1, 1), (1, 16), (8, 8), (8, 64), (96, 96))
             for seqs in (1, 3, 32) for rows in (1, 100, 2048, 8192, 65536, 262144) if rows >= seqs]
    for a, p in zip(asked, encode([("attend",) + x for x in asked])):
        assert not isinstance(p, str), (a, p)
        assert p[4] <= 600 << 20, (a, p[4] >> 20)
        if a[1] == 1:  # one sequence: units of no more tiles than go at once
            assert p[4] <= 80 << 20, (a, p[4] >> 20)


def test_launches_of_attention_change_with_the_tiles_not_with_a_row(encode):  # noqa: F811
    for heads, kv, dim in ((32, 8, 128), (64, 8, 128), (32, 4, 64), (16, 16, 128)):
        per = 128 * kv // heads     # rows of a wide tile
        rows = [r for tiles in (40, 64, 65, 128, 130) for r in (tiles * per - per + 1, tiles * per - 1, tiles * per)]
        got = encode([("attend", r, 1, heads, kv, dim, 1, 256) for r in rows])
        for i in range(0, len(rows), 3):
            wide = [p for p in got[i:i + 3] if p[0] == 2]     # (40 tiles of 4 key heads of 64 are narrow ones)
            assert len({p[7] for p in wide}) <= 1, ("units aimed at", rows[i:i + 3], got[i:i + 3])
        assert sum(p[0] == 2 for p in got) >= 12


class On:
    """What a planned list looks at of a tensor."""

    def __init__(self, index):
        self.device = torch.device("cuda", index)


@pytest.mark.parametrize("nested", [False, True])
def test_tensors_of_another_gpu_are_refused(nested):
    def ops(index):
        first, op = norm(), attend() if nested else norm()
        first.keep = ()
        if nested:
            op.keep = (cache(), On(0))
            op.keep[0].keep = (On(0), On(index))
        else:
            op.keep = (On(0), None, On(index))
        return D.make_ops([first, op])
    with Session(HOST):
        D.daris_create_partition(8)
        for call in (D.daris_plan_ops, D.daris_run_ops):
            with pytest.raises(D.DarisError) as e:
                call(ops(1), 0)
            assert e.value.code == D.EINVAL and "operator 1" in str(e.value) and "cuda:1" in str(e.value)
            with pytest.raises(D.DarisError) as e:      # tensors of the library's GPU: there is none here
                call(ops(0), 0)
            assert e.value.code == D.ESTATE


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_a_scale_of_scores_that_is_no_number_is_refused(scale):
    with Session(HOST):
        D.daris_create_partition(8)
        op = attend(scale=scale)
        op.keep = ()
        with pytest.raises(D.DarisError) as e:
            D.daris_plan_ops(D.make_ops([op]), 0)
        assert e.value.code == D.EINVAL and "operator 0" in str(e.value) and "scale" in str(e.value)
