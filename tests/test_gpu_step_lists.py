"""daris_run_ops of the C interface, which plans nothing, and lists longer than a queue."""
import pytest
import torch

import paper_2504_08795_amd as D
from step_helpers import E8, F8, Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    yield D.daris_create_partition(256)
    D.daris_shutdown()


def step(dtype):
    """Every operator once, and what it writes."""
    g = torch.Generator().manual_seed(2)
    c = Cache(3, [2000, 70], [1, 1], 2, 64)
    cache = c.gpu(D)
    x, w = torch.randn((2, 512), generator=g).to(dtype).cuda(), torch.ones(512, dtype=dtype, device="cuda")
    codes, scales = torch.randint(0, 256, (512, 256), generator=g, dtype=torch.uint8).cuda(), (torch.rand((512, 4), generator=g) * 0.02).bfloat16().cuda()
    y, ys = torch.zeros((2, 512), dtype=F8, device="cuda"), torch.zeros((2, 4), dtype=E8, device="cuda")
    heads, out, last = torch.zeros((2, 8, 64), dtype=dtype, device="cuda"), torch.zeros((2, 4, 64), dtype=dtype, device="cuda"), torch.zeros((2, 512), dtype=dtype, device="cuda")
    ops = [D.make_norm(x, w, y, 1e-5, scale=ys), D.make_matvec(y, codes, scales, heads.view(2, 512), x_scale=ys), D.make_append(cache, heads[:, 4:6], heads[:, 6:]),
           D.make_attend(cache, heads[:, :4], out, scale=0.125), D.make_matvec(out.view(2, 256), codes[:, :128], scales[:, :2].contiguous(), last)]
    return ops, [y.view(torch.uint8), heads, out, last] + [t.view(torch.uint8) for t in c.on_gpu[:4]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lists_that_are_not_planned_give_the_same(part, dtype):
    ops, outs = step(dtype)
    D.daris_run_ops(D.make_ops(ops), part)
    planned = [t.clone() for t in outs]
    assert all(bool(t.any()) for t in planned)
    for t in outs[:4]:
        t.zero_()
    for _ in range(3):
        listed = D.make_ops(ops)
        assert D.lib().daris_run_ops(listed.array, len(listed), part) == D.OK
        assert not listed.plans
        for a, b in zip(outs, planned):
            assert torch.equal(a, b)


@pytest.mark.parametrize("planned", [False, True])
def test_lists_longer_than_a_queue(part, planned):
    # 3000 norms, each of what the one in front of it left, with 0.5 added: sum counts them
    w = torch.zeros(64, device="cuda")
    x, add, y = (torch.zeros((1, 64), device="cuda") for _ in range(3))
    add += 0.5
    ops = D.make_ops([D.make_norm(x, w, y, 1e-5, res=add, sum=x)] * 3000)
    if planned:
        D.daris_run_ops(ops, part)
    else:
        assert D.lib().daris_run_ops(ops.array, len(ops), part) == D.OK
    assert bool((x == 1500).all())
