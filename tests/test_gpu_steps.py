"""The operators of a generation step (include/daris_ops.h) against their definitions in 64 bits, at the sizes, layouts and masks where they can go
wrong."""
import pytest
import torch

import paper_2504_08795_amd as D
from step_helpers import BLOCK, DT, E8, F8, PAGE, ROUND, Cache, attend, close, e4m3, e4m3_slack, matvec, norm, scale_exponent, turn_table, turned, two_to

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def part():
    D.daris_init(0, 0, 0)
    p = D.daris_create_partition(256)
    D.daris_create_partition(24)
    yield p
    D.daris_shutdown()


def rand(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def run(part, *ops):
    D.daris_run_ops(D.make_ops(list(ops)), part)


# ---- norm ---------------------------------------------------------------------------------------------------------------------


def norm_case(part, rows, width, dtype, res, group, skew=0, seed=1, x=None, eps=1e-5):
    dt = DT[dtype]
    x = rand((rows, width + skew), dt, seed, 3.0)[:, skew:] if x is None else x
    r = rand((rows, width), dt, seed + 1) if res else None
    w = rand((width,), dt, seed + 2, 0.3) + 1
    wide = torch.zeros((rows, width + skew), dtype=dt, device="cuda")
    wide[:, skew:] = x.cuda()
    xd, rd, wd = wide[:, skew:], r.cuda() if res else None, w.cuda()
    sd = torch.full((rows, width + skew), 7.0, dtype=dt, device="cuda")[:, skew:] if res else None
    y = torch.zeros((rows, width + skew), dtype=F8 if group else dt, device="cuda")[:, skew:]
    sc = torch.zeros((rows, width // group), dtype=torch.uint8, device="cuda").view(E8) if group else None
    run(part, D.make_norm(xd, wd, y, eps, res=rd, sum=sd, scale=sc))
    h, want = norm(x, r, w, eps)
    # the sum of n squares in fp32 (a tree: far below n roundings), its root, two products
    slack = want.abs() * (2.0 ** -20 + ROUND[dtype]) + 1e-38
    if res:
        close(sd, h, h.abs() * (ROUND[dtype] + 2.0 ** -24) + 1e-38, "sum")
    if not group:
        close(y, want, slack, "y")
        return
    most = want.view(rows, -1, group).abs().amax(2)
    e = scale_exponent(most)
    got = sc.cpu().view(torch.uint8).double() - 127
    edge = ((most / (448 * torch.exp2(e)) - 1).abs() < 1e-5) | ((most / (224 * torch.exp2(e)) - 1).abs() < 1e-5)     # either scale is right there
    assert bool(((got == e) | (edge & ((got - e).abs() <= 1))).all())
    s = torch.exp2(got).repeat_interleave(group, 1)
    close(y.cpu().double() * s, want, e4m3_slack(want, s), "codes")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,width,res,skew", [(1, 1, False, 0), (3, 7, True, 0), (2, 64, True, 0), (5, 513, False, 3), (130, 512, True, 0), (1, 4096, True, 0),
                                                 (2, 2050, True, 2), (3, 8192, False, 8), (2, 9000, True, 0), (1, 70000, True, 0), (2, 33333, False, 1)])
def test_norm(part, dtype, rows, width, res, skew):
    norm_case(part, rows, width, dtype, res, 0, skew)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,width,group,skew", [(1, 32, 32, 0), (4, 4096, 128, 0), (3, 192, 64, 0), (33, 96, 32, 1), (2, 1664, 128, 5), (1, 65664, 128, 0), (2, 8320, 64, 0)])
def test_norm_in_eight_bits(part, dtype, rows, width, group, skew):
    norm_case(part, rows, width, dtype, rows % 2 == 0, group, skew)


def test_norm_in_place_and_rows_without_a_number(part):
    x = rand((4, 256), torch.float32, 5)
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 9] = float("inf")
    w = torch.ones(256)
    h, want = norm(x, None, w, 1e-5)
    want[3] = 0                                            # the mean is infinite: what is finite becomes 0, the infinity NaN
    want[3, 9] = float("nan")
    xd = x.cuda()
    run(part, D.make_norm(xd, w.cuda(), xd, 1e-5))          # y on x
    close(xd, want, want.abs().nan_to_num() * 2.0 ** -19 + 1e-38, "in place")
    y, sc = torch.zeros((4, 256), dtype=F8, device="cuda"), torch.zeros((4, 8), dtype=E8, device="cuda")
    run(part, D.make_norm(x.cuda(), w.cuda(), y, 1e-5, scale=sc))
    y, sc = y.cpu().float(), sc.cpu().view(torch.uint8)
    assert bool((sc[1] == 27).all() and (y[1] == 0).all() and torch.isnan(y[2]).all() and torch.isnan(y[3, 9]) and (y[3, :9] == 0).all())
    # the sum may lie on the residual
    r = rand((4, 256), torch.float32, 6)
    rd, out = r.cuda(), torch.empty((4, 256), device="cuda")
    x2 = rand((4, 256), torch.float32, 7)
    run(part, D.make_norm(x2.cuda(), w.cuda(), out, 0.0, res=rd, sum=rd))
    h, want = norm(x2, r, w, 0.0)
    close(rd, h, h.abs() * 2.0 ** -23, "sum in place")
    close(out, want, want.abs() * 2.0 ** -19, "y")


# ---- append ---------------------------------------------------------------------------------------------------------------------


def append_case(part, seed, before, rows, kv, dim, heads, dtype, rot, pairs, edit=None, positions=None, in_place=False, magnitude=1.0, packed=True):
    c = Cache(seed, before, rows, kv, dim)
    if edit:
        edit(c)
    n, dt = sum(rows), DT[dtype]
    qkv = rand((n, heads + 2 * kv, dim), dt, seed + 1, 1.5 * magnitude)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    table = turn_table(positions if positions is not None else max(b + r for b, r in zip(before, rows)) + 1, rot) if rot else None
    old = {m: getattr(c, m).clone() for m in ("k", "v", "k_scale", "v_scale")}
    cache = c.gpu(D)
    g = qkv.cuda()
    gq, gk, gv = g[:, :heads], g[:, heads:heads + kv], g[:, heads + kv:]
    if not packed:
        gk, gv = gk.clone(), gv.clone()
    out = gq if in_place else torch.full((n, heads, dim), 7.0, dtype=dt, device="cuda")
    run(part, D.make_append(cache, gk, gv, row_start=None if all(r == 1 for r in rows) and seed % 2 else c.start.cuda(), q=gq, q_out=out,
                            turn=table.cuda() if rot else None, rot_dim=rot, pairs=pairs))
    got = {m: t.cpu() for m, t in zip(("k", "v", "k_scale", "v_scale"), c.on_gpu)}
    nan_row = torch.full((rot,), float("nan"))
    untouched = {m: torch.ones(old[m].shape, dtype=torch.bool) for m in old}
    for s, (b, r) in enumerate(zip(before, rows)):
        for i in range(r):
            row, pos = int(c.start[s]) + i, b + i
            at = (table[pos] if 0 <= pos < len(table) else nan_row) if rot else None
            want = turned(q[row].double(), at, rot, pairs) if rot else q[row].double()
            close(out[row], want, want.abs().nan_to_num() * ROUND[dtype] + q[row].double().abs().nan_to_num().amax() * 2.0 ** -22, f"query row {row}")
        for first in range(max(0, b) // BLOCK * BLOCK, b + r if r else 0, BLOCK):
            page = int(c.pages[s, first // PAGE]) if first // PAGE < c.pages.shape[1] else -1
            if not 0 <= page < c.k.shape[0]:
                continue
            part_ = first % PAGE // BLOCK
            held, end = max(0, b - first), min(BLOCK, b + r - first)
            lo = first % PAGE
            for name, src in (("k", k), ("v", v)):
                new = torch.stack([(turned(src[int(c.start[s]) + t - b].double(), table[t] if 0 <= t < len(table) else nan_row, rot, pairs)
                                    if rot and name == "k" else src[int(c.start[s]) + t - b].double()) for t in range(max(first + held, b), first + end)], 1)
                codes = (lambda z: z[name][page, :, lo:lo + BLOCK] if name == "k" else z[name][page, :, :, lo:lo + BLOCK].transpose(1, 2))
                was, now = codes(old).double(), codes(got).double()
                s_old = two_to(old[name + "_scale"])[page, :, part_]
                s_new = two_to(got[name + "_scale"])[page, :, part_]
                most = torch.where(torch.isfinite(new), new.abs(), 0.0).amax((1, 2))
                e = torch.exp2(scale_exponent(most))
                if held:
                    e = torch.maximum(e, s_old)
                near = ((most / (448 * e) - 1).abs() < 1e-5) | ((most / (224 * e) - 1).abs() < 1e-5)
                assert bool(((s_new == e) | near).all()), (name, s, first, s_new, e)
                first_new = max(held, b - first if b > first else held)
                want = torch.where(torch.isfinite(new), new, float("nan"))
                close(now[:, first_new:end] * s_new[:, None, None], want, e4m3_slack(want.nan_to_num(), s_new[:, None, None]), f"new {name} of sequence {s} from {first}")
                if held:
                    kept = e4m3(was[:, :held] * (s_old / s_new)[:, None, None])
                    close(now[:, :held], kept, 0.0, f"earlier {name} of sequence {s} from {first}")
                u = untouched[name][page, :, lo:lo + end] if name == "k" else untouched[name][page, :, :, lo:lo + end]
                u[...] = False
                untouched[name + "_scale"][page, :, part_] = False
    for m in old:
        assert torch.equal(got[m].view(torch.uint8)[untouched[m]], old[m].view(torch.uint8)[untouched[m]]), f"{m} changed where nothing was written"


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,pairs", [("bf16", False), ("fp32", True)])
def test_append_one_token_to_each_sequence(part, dim, dtype, pairs):
    before = [0, 1, 15, 16, 63, 64, 200]
    append_case(part, 10 + dim, before, [1] * 7, 2, dim, 6, dtype, dim, pairs)
    append_case(part, 11 + dim, before, [1] * 7, 3, dim, 3, dtype, dim // 2, not pairs, in_place=True)


@pytest.mark.parametrize("dtype,rot,pairs", [("bf16", 64, False), ("fp32", 32, True), ("fp32", 0, False), ("bf16", 2, True)])
def test_append_prompts_of_unequal_lengths(part, dtype, rot, pairs):
    append_case(part, 30 + rot, [0, 5, 100, 0, 17, 64], [70, 0, 3, 16, 1, 130], 2, 64, 5, dtype, rot, pairs)


def test_append_lets_scales_grow_and_keeps_what_is_larger(part):
    for magnitude in (1e-3, 1.0, 1e4):
        append_case(part, 50, [3, 20, 40], [2, 30, 1], 2, 64, 2, "fp32", 64, False, magnitude=magnitude)


def test_append_leaves_out_pages_that_are_not_there(part):
    def edit(c):
        c.pages[0, 1] = -1
        c.pages[1, 0] = 10 ** 6
        c.pages[2, 1] = -(2 ** 31)
    append_case(part, 60, [60, 0, 100], [10, 3, 1], 2, 64, 2, "bf16", 64, False, edit=edit)
    append_case(part, 61, [-3, -5], [10, 2], 1, 128, 2, "fp32", 0, False)              # places in front of the first are none


def test_append_makes_positions_outside_the_table_and_numbers_that_are_none_nan(part):
    append_case(part, 70, [6], [5], 1, 64, 2, "fp32", 64, False, positions=9)
    c = Cache(71, [2], [1], 1, 64)
    x = rand((1, 1, 64), torch.float32, 72)
    x[0, 0, 3], x[0, 0, 5], x[0, 0, 9] = float("inf"), float("nan"), -float("inf")
    cache, xd = c.gpu(D), x.cuda()
    run(part, D.make_append(cache, xd, xd, row_start=c.start.cuda()))
    page = int(c.pages[0, 0])
    k, v = c.on_gpu[0][page, 0, 2].cpu().float(), c.on_gpu[1][page, 0, :, 2].cpu().float()
    for y in (k, v):
        assert torch.isnan(y).nonzero().flatten().tolist() == [3, 5, 9]
    fine = torch.where(torch.isfinite(x[0, 0]), x[0, 0], 0.0).double()
    s = float(two_to(c.on_gpu[2].cpu())[page, 0, 0])
    close(torch.nan_to_num(k).double() * s, fine, e4m3_slack(fine, torch.tensor(s)), "finite ones")


# ---- attend ---------------------------------------------------------------------------------------------------------------------


def attend_case(part, seed, before, rows, kv, group, dim, dtype, window=0, edit=None, scale=None, strided=False, entries=1, q_scale=1.0, gpu_start=True):
    c = Cache(seed, before, rows, kv, dim, extra_entries=entries).filled(seed + 1)
    if edit:
        edit(c)
    n, heads, dt = sum(rows), kv * group, DT[dtype]
    q = rand((n, heads, dim), dt, seed + 2, q_scale)
    scale = dim ** -0.5 / 4 if scale is None else scale
    out = torch.full((n, heads, dim + 3), 7.0, dtype=dt, device="cuda")[..., 1:dim + 1] if strided else torch.full((n, heads, dim), 7.0, dtype=dt, device="cuda")
    gq = torch.cat([q, q[..., :5]], 2).cuda()[..., :dim] if strided else q.cuda()
    op = D.make_attend(c.gpu(D), gq, out, row_start=c.start.cuda() if gpu_start else None, scale=scale, window=window)
    run(part, op)
    want, slack = attend(c, q, scale, window, dtype)
    close(out, want, slack, "out")
    first = out.clone()
    run(part, op)
    assert torch.equal(first.nan_to_num(5.0), out.nan_to_num(5.0)), "another run, other bits"
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kv,group", [(1, 1), (2, 4), (3, 7), (1, 16)])
def test_attend_one_token_of_each_sequence(part, dtype, dim, kv, group):
    attend_case(part, 100 + dim + group, [0, 62, 63, 64, 300, 5, 127, 16], [1] * 8, kv, group, dim, dtype, gpu_start=dim != 128)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [0, 1, 40, 64, 1000])
def test_attend_drafts_and_windows(part, dtype, window):
    attend_case(part, 200 + window, [100, 0, 250, 63, 7], [5, 3, 1, 4, 0], 2, 3, 64, dtype, window)
    attend_case(part, 201 + window, [300, 20], [2, 21], 1, 5, 128, dtype, window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 70])
def test_attend_chunks_of_a_prompt(part, dtype, dim, window):
    attend_case(part, 300 + dim, [130, 0], [70, 33], 1, 3, dim, dtype, window)          # 103 rows x 3 columns in two sequences: wide tiles, the last in part
    attend_case(part, 301 + dim, [0], [150], 2, 1, dim, dtype, window)


def test_attend_long_contexts_in_many_units(part):
    attend_case(part, 400, [9000], [1], 1, 2, 64, "bf16")
    attend_case(part, 401, [5000, 64], [1, 1], 1, 4, 128, "fp32", entries=100)          # a table far wider than the lengths
    attend_case(part, 402, [4000], [65], 1, 1, 64, "bf16")                              # wide, cut into units
    attend_case(part, 403, [4000], [65], 1, 1, 64, "fp32", window=900)


def test_attend_more_sequences_than_a_wave_has_lanes(part):
    before = [(37 * i) % 150 for i in range(150)]
    attend_case(part, 410, before, [1] * 150, 1, 2, 64, "bf16", gpu_start=False)
    attend_case(part, 411, before, [i % 3 for i in range(150)], 1, 2, 64, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [40, 3, 30, 90]])
def test_attend_nothing_and_pages_that_are_not_there(part, dtype, rows):
    def edit(c):
        c.pages[1, 0] = -1
        c.pages[2, 1] = 12345678
        c.pages[3, :] = -7
    out = attend_case(part, 420, [-200, 100, 200, 70], rows, 1, 2, 64, dtype, edit=edit)
    assert bool((out[: rows[0]] == 0).all()) and bool((out[sum(rows[:3]):] == 0).all())
    attend_case(part, 421, [-2, 0], [5, 2], 1, 2, 64, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,window", [([6], 0), ([80], 0), ([6], 4), ([80], 20)])
def test_attend_nan_only_where_it_is_seen(part, dtype, rows, window):
    before = 50

    def edit(c):
        for t, d in ((3, 1), (53, 2), (before + rows[0] - 1, 7)):          # values: an early token, a middle one, the last
            c.v.view(torch.uint8)[int(c.pages[0, t // PAGE]), 0, d, t % PAGE] = 0x7F
        t = before + rows[0] - 2                                           # a key that only the last two rows see
        c.k.view(torch.uint8)[int(c.pages[0, t // PAGE]), 0, t % PAGE, 11] = 0xFF
    out = attend_case(part, 430, [before], rows, 1, 2, 64, dtype, window=window, edit=edit)
    assert bool(torch.isnan(out[-2:]).all()) and not bool(torch.isnan(out[0, :, 7]).any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("before,rows,group", [([200], [1], 2), ([200, 64, 3000], [1, 1, 1], 4), ([200, 90], [7, 30], 3), ([140], [80], 2)])
def test_attend_nan_on_pages_that_every_row_sees(part, dtype, dim, before, rows, group):
    def edit(c):
        c.v.view(torch.uint8)[int(c.pages[0, 0]), 0, 1, 3] = 0x7F
        c.v.view(torch.uint8)[int(c.pages[0, 1]), 0, dim - 2, 63] = 0xFF
        if len(before) > 2:
            c.k.view(torch.uint8)[int(c.pages[2, 20]), 0, 5, 11] = 0x7F
    out = attend_case(part, 435, before, rows, 1, group, dim, dtype, edit=edit)
    gone = torch.isnan(out[: rows[0]])
    assert bool(gone[..., 1].all() and gone[..., dim - 2].all()) and int(gone.sum()) == 2 * rows[0] * group
    assert bool(torch.isnan(out[-1]).all()) if len(before) > 2 else True


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_sizes_of_queries_and_scales(part, dtype):
    def wild(c):
        u = c.v_scale.view(torch.uint8)
        u[u != 0xFE] = torch.randint(60, 190, (int((u != 0xFE).sum()),), generator=torch.Generator().manual_seed(3), dtype=torch.uint8)
    attend_case(part, 440, [200, 90], [1, 2], 1, 3, 64, dtype, edit=wild)
    attend_case(part, 441, [200], [3], 1, 3, 64, dtype, q_scale=1e-30)
    attend_case(part, 442, [200], [3], 1, 3, 64, dtype, q_scale=1e6, scale=1e-6)
    attend_case(part, 443, [200], [3], 1, 3, 64, dtype, scale=0.0)
    attend_case(part, 444, [200], [70], 1, 1, 64, dtype, scale=-0.05)
    attend_case(part, 445, [100, 30], [1, 40], 1, 3, 64, dtype, strided=True)
    attend_case(part, 446, [100], [100], 1, 1, 64, dtype, strided=True)


# ---- 4-bit products -----------------------------------------------------------------------------------------------------------


def matvec_case(part, rows, n, k, group, dtype, codes=False, gate=False, skew=0, seed=1, edit=None):
    dt = DT[dtype]
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8)
    ws = (torch.rand((n, k // group), generator=g) * 0.05).bfloat16()
    x = rand((rows, k), dt, seed + 1)
    if edit:
        edit(x)
    wide = torch.zeros((n, k // 2 + 16 * (skew > 0)), dtype=torch.uint8, device="cuda")
    wide[:, : k // 2] = w.cuda()
    xs = None
    if codes:
        v = x.double().view(rows, -1, group)
        e = scale_exponent(v.abs().amax(2))
        xs = (e + 127).to(torch.uint8).view(E8)
        x = (v / torch.exp2(e)[:, :, None]).float().to(F8).view(rows, k)
        exact = (x.double().view(rows, -1, group) * torch.exp2(e)[:, :, None]).view(rows, k)
    else:
        exact = x.double()
    xd = torch.cat([x.view(torch.uint8) if codes else x, (x.view(torch.uint8) if codes else x)[:, :skew]], 1).cuda()
    xd = (xd.view(F8) if codes else xd)[:, skew:k + skew] if skew else (xd.view(F8) if codes else xd)
    if skew:
        xd = torch.empty((rows, k + skew), dtype=torch.uint8 if codes else dt, device="cuda")
        xd[:, skew:] = (x.view(torch.uint8) if codes else x).cuda()
        xd = (xd.view(F8) if codes else xd)[:, skew:]
    cols = n // 2 if gate else n
    y = torch.full((rows, cols + skew), 7.0, dtype=dt, device="cuda")[:, skew:]
    run(part, D.make_matvec(xd, wide[:, : k // 2], ws.cuda(), y, x_scale=xs.cuda() if codes else None, gate=gate))
    want, slack = matvec(exact, w, ws, gate, dtype)
    close(y, want, slack, "y")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,n,k,group", [(1, 1, 32, 32), (1, 17, 160, 32), (1, 4096, 4096, 128), (2, 100, 4160, 64), (3, 5000, 256, 128), (16, 330, 1184, 32), (15, 64, 4224, 128),
                                            (1, 300, 25088, 64), (16, 48, 25088, 128), (17, 130, 640, 64), (64, 96, 2080, 32), (70, 200, 4096, 128), (130, 40, 192, 64), (1, 9000, 512, 32)])
def test_matvec(part, dtype, rows, n, k, group):
    matvec_case(part, rows, n, k, group, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,n,k,group", [(1, 4096, 4096, 128), (5, 70, 416, 32), (16, 130, 320, 64), (40, 90, 1280, 128)])
def test_matvec_with_rows_in_eight_bits(part, dtype, rows, n, k, group):
    matvec_case(part, rows, n, k, group, dtype, codes=True)
    matvec_case(part, rows, n, k, group, dtype, codes=True, skew=3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,n,k,group", [(1, 2, 64, 64), (1, 4100, 1024, 128), (7, 34, 96, 32), (33, 130, 512, 128)])
def test_matvec_gated_and_strided(part, dtype, rows, n, k, group):
    matvec_case(part, rows, n, k, group, dtype, gate=True)
    matvec_case(part, rows, n, k, group, dtype, gate=True, skew=1)
    matvec_case(part, rows, n, k, group, dtype, skew=5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_matvec_sizes_of_rows(part, dtype):
    def spread(x):
        x *= torch.exp2(torch.linspace(-60, 60, x.shape[1])).to(x.dtype)
    matvec_case(part, 3, 50, 1024, 64, dtype, edit=spread)
    matvec_case(part, 2, 50, 256, 32, dtype, edit=lambda x: x.mul_(0))
    x = rand((3, 256), DT[dtype], 9)
    x[1, 5] = float("nan")
    x[2, 200] = float("inf")
    w = torch.randint(0, 256, (40, 128), generator=torch.Generator().manual_seed(8), dtype=torch.uint8)
    ws = torch.full((40, 2), 0.5).bfloat16()
    y = torch.empty((3, 40), dtype=DT[dtype], device="cuda")
    run(part, D.make_matvec(x.cuda(), w.cuda(), ws.cuda(), y))
    want, slack = matvec(x[:1].double(), w, ws, False, dtype)
    close(y[:1], want, slack, "the row of numbers")
    assert bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[2]).any())


# ---- lists of operators ---------------------------------------------------------------------------------------------------------


def test_a_list_runs_in_order_on_any_partition_and_twice_gives_the_same(part):
    c = Cache(500, [70, 3], [1, 1], 2, 64)
    x, w = rand((2, 256), torch.bfloat16, 501), torch.ones(256, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(502)
    wq, ws = torch.randint(0, 256, (8 * 64, 128), generator=g, dtype=torch.uint8), (torch.rand((8 * 64, 2), generator=g) * 0.02).bfloat16()
    results = []
    for p in (part, 1, part):
        cache = c.gpu(D)
        y, sc = torch.zeros((2, 256), dtype=F8, device="cuda"), torch.zeros((2, 2), dtype=E8, device="cuda")
        qkv, out = torch.zeros((2, 8 * 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
        heads = qkv.view(2, 8, 64)
        table = turn_table(80, 64).cuda()
        ops = D.make_ops([D.make_norm(x.cuda(), w.cuda(), y, 1e-5, scale=sc), D.make_matvec(y, wq.cuda(), ws.cuda(), qkv, x_scale=sc),
                          D.make_append(cache, heads[:, 4:6], heads[:, 6:], q=heads[:, :4], q_out=heads[:, :4], turn=table, rot_dim=64),
                          D.make_attend(cache, heads[:, :4], out, scale=0.125)])
        D.daris_run_ops(ops, p)
        results.append([t.clone() for t in (y.view(torch.uint8), sc.view(torch.uint8), qkv, out)] + [t.view(torch.uint8).clone() for t in c.on_gpu[:4]])
        D.daris_run_ops(ops, p)
    for other in results[1:]:
        assert torch.equal(results[0][0], other[0]) and torch.equal(results[0][1], other[1])
        close(other[2], results[0][2], results[0][2].double().abs() * 2.0 ** -7 + 1e-4, "qkv")       # (other shares of K on fewer CUs)
    for a, b in zip(results[0], results[2]):
        assert torch.equal(a, b)


def test_operators_wait_for_the_callers_streams_and_run_beside_other_plans(part):
    x, w, y = torch.zeros((64, 4096), device="cuda"), torch.ones(4096, device="cuda"), torch.empty((64, 4096), device="cuda")
    ops = D.make_ops([D.make_norm(x, w, y, 1e-5)])
    side = torch.cuda.Stream()
    big = torch.randn((4096, 4096), device="cuda")
    for i in range(5):
        with torch.cuda.stream(side):
            z = big
            for _ in range(4):
                z = (z @ big) * 1e-3
            x.copy_(z[:64] * 0 + i + 1)
        D.daris_run_ops(ops, part)                        # x is written on a stream that has not been waited for
        assert bool(((y - 1).abs() < 1e-4).all()), i
        x.zero_()
        torch.cuda.synchronize()


def test_plans_are_kept_freed_and_gone_after_a_shutdown(part):
    x, w, y = torch.randn((2, 64), device="cuda"), torch.ones(64, device="cuda"), torch.empty((2, 64), device="cuda")
    ops = D.make_ops([D.make_norm(x, w, y, 1e-5)])
    plan = D.daris_plan_ops(ops, part)
    D.daris_run_plan(plan)
    first = y.clone()
    many = [D.daris_plan_ops(ops, part) for _ in range(1500)]      # more than one slab of argument blocks
    D.daris_run_plan(many[-1])
    for p in many:
        D.daris_free_plan(p)
    with pytest.raises(D.DarisError) as e:
        D.daris_run_plan(many[0])
    assert e.value.code == D.binding.ERANGE
    with pytest.raises(D.DarisError):
        D.daris_free_plan(many[0])
    # another plan makes the workspace grow: the first one's launches follow it
    c = Cache(600, [3000], [1], 1, 64).filled(601)
    q, out = rand((1, 2, 64), torch.float32, 602).cuda(), torch.empty((1, 2, 64), device="cuda")
    small = D.make_ops([D.make_attend(c.gpu(D), q, out, scale=0.1)])
    D.daris_run_ops(small, part)
    want = out.clone()
    c2 = Cache(603, [500] * 40, [3] * 40, 2, 256).filled(604)
    q2 = rand((120, 4, 256), torch.float32, 605).cuda()
    D.daris_run_ops(D.make_ops([D.make_attend(c2.gpu(D), q2, torch.empty_like(q2), row_start=c2.start.cuda(), scale=0.1)]), part)
    out.zero_()
    D.daris_run_ops(small, part)
    assert torch.equal(out, want)
    D.daris_shutdown()
    D.daris_init(0, 0, 0)
    assert D.daris_create_partition(256) == part
    D.daris_create_partition(24)
    with pytest.raises(D.DarisError):
        D.daris_run_plan(plan)
    y.zero_()
    D.daris_run_ops(ops, part)                            # planned anew
    assert torch.equal(y, first)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,n,k,group", [(1, 40, 25088, 128), (16, 70, 4224, 64), (33, 34, 3200, 64), (70, 200, 4096, 128), (130, 48, 2112, 32)])
def test_matvec_of_few_outputs_and_a_long_k(part, dtype, rows, n, k, group):
    matvec_case(part, rows, n, k, group, dtype)
    matvec_case(part, rows, n, k, group, dtype, gate=True, skew=1)
    matvec_case(part, rows, n, k, group, dtype, codes=True)
    x = rand((rows, k), DT[dtype], 11).cuda()
    w = torch.randint(0, 256, (n, k // 2), generator=torch.Generator().manual_seed(12), dtype=torch.uint8).cuda()
    ws = torch.full((n, k // group), 0.25, dtype=torch.bfloat16, device="cuda")
    y = [torch.empty((rows, n), dtype=DT[dtype], device="cuda") for _ in range(4)]
    run(part, *[D.make_matvec(x, w, ws, t) for t in y])
    assert all(torch.equal(t, y[0]) for t in y), "another run, other bits"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,window", [(26, 0), (32, 0), (39, 0), (39, 200)])
def test_attend_a_chunk_of_one_sequence_on_few_cus(part, dtype, rows, window):
    # tiles of 128 columns for each of 12 heads on 24 CUs: as many units as go at once, and more
    attend_case(part + 1, 800 + rows, [150], [rows], 12, 16, 64, dtype, window)


def test_operators_without_rows_do_nothing(part):
    e = torch.empty((0, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    c = Cache(700, [3], [0], 1, 64)
    cache = c.gpu(D)
    z = torch.empty((0, 1, 64), device="cuda")
    start = c.start.cuda()
    run(part, D.make_norm(e, w, e, 1e-5), D.make_append(cache, z, z, row_start=start), D.make_attend(cache, z, z, row_start=start),
        D.make_matvec(e, torch.zeros((4, 32), dtype=torch.uint8, device="cuda"), torch.zeros((4, 1), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 4), device="cuda")))
    run(part)
    assert torch.equal(c.on_gpu[0].cpu().view(torch.uint8), c.k.view(torch.uint8))
