"""Lists of operators while tasks have active jobs, on the queue that the jobs use and on another partition's: both give what each gives alone."""
import numpy as np
import pytest
import torch

import paper_2504_08795_amd as D
import workloads as wl
from step_helpers import Cache

pytestmark = pytest.mark.gpu


def operators():
    """A step whose attention and products meet in the workspace, and its outputs."""
    g = torch.Generator().manual_seed(5)
    c = Cache(6, [3000, 70, 500], [1, 1, 1], 2, 64).filled(7)
    x, w = torch.randn((3, 512), generator=g).bfloat16().cuda(), torch.ones(512, dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.randint(0, 256, (512, 256), generator=g, dtype=torch.uint8).cuda(), (torch.rand((512, 4), generator=g) * 0.02).bfloat16().cuda()
    y, q, out = torch.zeros_like(x), torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")
    last = torch.zeros_like(x)
    ops = [D.make_norm(x, w, y, 1e-5), D.make_matvec(y, codes, scales, q.view(3, 512)), D.make_attend(c.gpu(D), q, out, scale=0.125), D.make_matvec(out.view(3, 512), codes, scales, last)]
    return D.make_ops(ops), (y, q, out, last)


@pytest.mark.parametrize("flags", [0, D.SHARED_QUEUE])
def test_operators_and_jobs_do_not_disturb_each_other(flags):
    layers, shp = wl.build_net("resnet18")
    shp = (shp[0], 128, 128)
    weights = wl.make_weights(layers, 3)
    n_out, jobs = layers[-1].c_out, 12
    frames = torch.from_numpy(np.random.default_rng(8).normal(0, 1, (jobs,) + shp).astype(np.float32)).cuda()
    D.daris_init(0, 0, flags)
    try:
        parts = [D.daris_create_partition(128), D.daris_create_partition(128)]
        dnn, keep = D.make_dnn(layers, weights, shp, "fp32")
        tasks = [D.daris_register_task(dnn, 10**9, 10**9, D.HP) for _ in parts]
        for t in tasks:
            D.daris_split_stages(t, 2)
        D.daris_commit()
        want = torch.empty((jobs, n_out), device="cuda")
        for i in range(jobs):
            D.daris_forward(tasks[0], frames[i], want[i], parts[0])
        steps = [operators() for _ in parts]      # of each partition
        alone = []
        for p, (ops, outs) in zip(parts, steps):
            D.daris_run_ops(ops, p)
            alone.append([t.clone() for t in outs])
        beside = 0
        for turn in range(4):
            got = torch.zeros((len(tasks), jobs, n_out), device="cuda")
            torch.cuda.synchronize()
            for i in range(jobs):
                for k, t in enumerate(tasks):
                    D.daris_release_job(t, frames[i], got[k, i])
                for p, (ops, outs), first in zip(parts, steps, alone):
                    for o in outs:
                        o.zero_()
                    D.daris_run_ops(ops, p)
                    stats = [D.daris_get_stats(t) for t in tasks]
                    beside += any(s["completed"] < s["accepted"] for s in stats)
                    for o, f in zip(outs, first):
                        assert torch.equal(o, f), (turn, i, p)
            D.daris_run_until_idle()
            for k in range(len(tasks)):
                assert torch.equal(got[k], want), (turn, k)
        assert beside >= 8, beside                # lists that ended while jobs were still to run
    finally:
        D.daris_shutdown()
