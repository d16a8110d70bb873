"""The operators of a generation step on the host: what their descriptors' checks refuse, and that every launch fits what its kernel assumes (LDS, pieces a
thread stages, units and tiles that cover the work).  No GPU."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

import paper_2504_08795_amd as D
from lib_helpers import Session
from paper_2504_08795_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
HOST = D.VIRTUAL_TIME | D.NO_DEVICE
P = 1 << 20      # an address that nothing reads: the checks come before any launch, and there is no device


@pytest.fixture(scope="module")
def encode(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("steps") / "driver")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           "-o", exe, os.path.join(HERE, "host_steps", "driver.cpp")])

    def run(lines):
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, ln)) for ln in lines) + "\n", capture_output=True, text=True, check=True)
        return [ln if ln.startswith("error") else [int(v) for v in ln.split()] for ln in r.stdout.splitlines()]
    return run


def test_matvec_launches_fit_their_kernel(encode):
    rng = random.Random(1)
    asked = [(1, 4096, 4096, 128, 1, 1, 0, 256), (16, 22016, 4096, 128, 1, 0, 1, 256), (1, 4096, 25088, 64, 0, 0, 0, 256), (128, 65536, 65536, 32, 0, 0, 0, 256), (1, 1, 32, 32, 1, 0, 0, 8)]
    while len(asked) < 3000:
        g = rng.choice([32, 64, 128])
        n, codes, dtype = int(2 ** rng.uniform(0, 17)), rng.random() < 0.3, rng.randrange(2)
        asked.append((int(2 ** rng.uniform(0, 10)), n, g * int(2 ** rng.uniform(0, 11)), g, dtype, int(codes), int(n % 2 == 0 and rng.random() < 0.3), rng.choice([8, 24, 128, 256])))
    for a, p in zip(asked, encode([("matvec",) + x for x in asked])):
        rows, n, k, g, dtype, codes, _, n_cu = a
        assert not isinstance(p, str), (a, p)
        kernel, groups, threads, lds, part, counters, cs, log, across, tgs, wgs, shares, each = p
        parts = 2 if not codes and dtype == 0 else 1
        waves, blocks, steps, block_rows = threads // 64, -(-rows // 16), -(-k // 128), min(rows, 16)
        assert kernel == 3 and waves == 16
        assert groups == wgs * blocks * shares and wgs <= max(tgs, 1) and tgs * across * 16 >= n > (tgs - 1) * across * 16, (a, p)
        assert across in (1, 2, 4, 8, 16) and across <= waves and 1 <= cs <= each and cs <= 1 << log < 2 * cs, (a, p)
        assert 1 <= shares and (shares - 1) * each < steps <= shares * each, ("shares of K", a, p)
        if shares > 1:  # one round, no more workgroups than CUs, and a place for each of their numbers
            assert wgs == tgs and groups <= n_cu and counters == wgs * blocks and part == counters * shares * 16 * 16 * across * 4, (a, p)
        else:
            assert part == counters == 0
        assert (16 << log) * block_rows <= (4 if parts == 2 else 8) * threads, ("pieces of x", a, p)
        scales = cs * (128 // g)
        assert -(-scales // 8) * across * 16 <= 2 * threads, ("pieces of scales", a, p)
        chunks = -(-each // cs)
        x = parts * cs * 16 * block_rows * 16 + (0 if not codes and dtype == 1 else cs * (128 // g) * (-(-block_rows // 4) * 4) * 8)
        need = (2 if chunks > 1 else 1) * x + (2 if chunks > 1 or wgs < tgs else 1) * across * 16 * ((scales + 7) // 8 * 8 + 2) * 2 + waves * 16 * 16 * 4
        assert need <= lds <= 160 * 1024, ("LDS", need, a, p)


def test_attend_launches_cover_every_cut(encode):
    """The kernel cuts tiles x pages into units by the lengths it finds; whatever those are, there are enough workgroups and places in the workspace."""
    rng = random.Random(2)
    asked = []
    while len(asked) < 600:
        kv, seqs = rng.choice([1, 2, 8, 12]), int(2 ** rng.uniform(0, 9))
        asked.append((seqs * rng.choice([1, 1, 3, 40]) + rng.randrange(200), seqs, kv * rng.choice([1, 4, 7, 16]), kv, rng.choice([64, 128, 256]), rng.randrange(2), rng.choice([8, 128, 256])))
    for a, p in zip(asked, encode([("attend",) + x for x in asked])):
        n_rows, seqs, heads, kv, dim, dtype, n_cu = a
        kernel, groups, threads, lds, part, counters, group, target, units = p
        cols, most = (16, 256) if kernel == 1 else (128, 16)
        full = 6 if dim == 64 else 3 if dtype == D.BF16 else 8
        assert kernel == (2 if n_rows * group * dim >= 4096 * seqs and n_rows * heads > full * 16 * n_cu and dim < 256 else 1) and threads == 256 and groups == units * kv and lds <= 160 * 1024, (a, p)
        assert counters == (units * kv if target else 0) and part == counters * cols * (dim + 2) * 4, (a, p)
        for _ in range(5):
            cuts = sorted(rng.randrange(n_rows + 1) for _ in range(seqs - 1))
            rows = [y - x for x, y in zip([0] + cuts, cuts + [n_rows])]
            pages = [int(2 ** rng.uniform(0, 11)) if r else 0 for r in rows]
            tiles = [-(-r * group // cols) for r in rows]
            work = sum(t * q for t, q in zip(tiles, pages))
            per = -(-int(work * 1.0001 + 1) // target) if target else max(pages)
            per = max(1, per, -(-max(pages) // most))
            per = (per + 3) // 4 * 4
            # (a unit less: the kernel's own sum is in fp32)
            assert sum(t * max(1, -(-q // per)) if t else 0 for t, q in zip(tiles, pages)) <= units, (a, rows, pages)
            assert not target or max(-(-q // per) for q in pages) <= most


def test_append_launches_have_an_item_for_every_sixteenth(encode):
    rng = random.Random(3)
    for _ in range(50):
        seqs, kv = int(2 ** rng.uniform(0, 8)), rng.choice([1, 3, 8])
        rows = [rng.choice([0, 1, 2, 15, 16, 17, 18, 33, 200]) for _ in range(seqs)]
        n = sum(rows)
        if n == 0:
            continue
        p = encode([("append", n, seqs, 1, kv, 5, 128)])[0]
        _, groups, threads, _, _, _, items, q_items = p
        assert q_items == n * 2 and groups * (threads // 64) >= items + q_items
        start, starts = 0, []
        for s, r in enumerate(rows):
            starts.append(start // 16 + 2 * s)
            start += r
        starts.append(start // 16 + 2 * seqs)
        assert items == starts[-1] * kv
        for s, r in enumerate(rows):
            for first in range(16):      # the place of the first token in its sixteenth
                assert r == 0 or -(-(first + r) // 16) <= starts[s + 1] - starts[s], (r, first)


def test_norm_shapes_hold_a_row(encode):
    for dtype, vec in ((1, 8), (0, 4)):
        for width in (1, 7, 64, 512, 513, 2048, 4096, 8192, 8193, 16384, 32768, 32769, 200000):
            kernel, groups, threads, _, _, _, vectors = encode([("norm", 3, width, 0, dtype, 0, width)])[0]
            nv, t = ((1, 64), (1, 256), (2, 256), (4, 256), (4, 1024), (0, 1024))[kernel]
            assert groups == 3 and threads == t and vectors == -(-width // vec) and (nv == 0 or nv * t >= vectors)


# ---- refusals -------------------------------------------------------------------------------------------------------------------


def norm(**kw):
    return _op(D.STEP_NORM, B.daris_norm(), dict(x=P, weight=P, y=P, x_row=64, y_row=64, rows=2, width=64, dtype=D.FP32, eps=1e-5), kw)


def cache(**kw):
    c = B.daris_cache()
    for n, v in dict(dict(k=P, v=P, k_scale=P, v_scale=P, pages=P, before=P, pages_row=4, n_pages=4, n_seqs=2, kv_heads=2, dim=64), **kw).items():
        setattr(c, n, v)
    return c


def append(c=None, **kw):
    return _op(D.STEP_APPEND, B.daris_append(), dict(cache=c or cache(), k=P, v=P, q=P, q_out=P, turn=P, row_start=P, n_rows=2, q_heads=4, dtype=D.BF16, turn_rows=9, rot_dim=64), kw)


def attend(c=None, **kw):
    return _op(D.STEP_ATTEND, B.daris_attend(), dict(cache=c or cache(), q=P, out=P, row_start=P, n_rows=2, q_heads=4, dtype=D.BF16, scale=1.0), kw)


def matvec(**kw):
    return _op(D.STEP_MATVEC, B.daris_matvec(), dict(x=P, w=P, w_scale=P, y=P, x_row=64, w_row=32, y_row=8, rows=2, n=8, k=64, group=32, dtype=D.FP32), kw)


def _op(kind, value, defaults, changes):
    for n, v in dict(defaults, **changes).items():
        setattr(value, n, v)
    return B._made(kind, value)


WRONG = [
    (norm(dtype=2), "dtype"), (norm(rows=-1), "rows"), (norm(width=0), "width"), (norm(eps=-1.0), "eps"), (norm(eps=float("nan")), "eps"), (norm(x=None), "NULL"), (norm(weight=None), "NULL"),
    (norm(y=None), "NULL"), (norm(x=P + 2), "aligned"), (norm(sum=P + 1), "aligned"), (norm(scale=P, group=48), "group"), (norm(scale=P, group=128), "multiple"), (norm(group=32), "scales"),
    (append(cache(dim=96)), "dim"), (append(cache(kv_heads=0)), "count"), (append(cache(n_seqs=-1)), "count"), (append(cache(pages_row=1 << 25)), "2^30"), (append(cache(pages=None)), "NULL"),
    (append(cache(k=P + 8)), "16 bytes"), (append(cache(v_scale=P + 2)), "4 bytes"), (append(row_start=None, n_rows=3), "without row_start"), (append(k=None), "NULL"), (append(rot_dim=65), "rot_dim"),
    (append(rot_dim=-2), "rot_dim"), (append(turn=None), "table"), (append(q_out=None), "together"), (append(q_heads=0), "query head"), (append(v=P + 1), "aligned"), (append(dtype=-1), "dtype"),
    (append(turn_rows=-1), "turn_rows"),
    (attend(q_heads=5), "key heads"), (attend(q_heads=0), "key heads"), (attend(window=-1), "window"), (attend(q=None), "NULL"), (attend(out=P + 1), "aligned"), (attend(cache(n_pages=-1)), "count"),
    (attend(n_rows=-1), "count"), (attend(cache(before=P + 2)), "4 bytes"),
    (matvec(group=16), "group"), (matvec(k=48), "multiple"), (matvec(n=7, gate=1), "pairs"), (matvec(w=P + 8), "16 bytes"), (matvec(w_row=40), "16 bytes"), (matvec(x=P + 2), "aligned"),
    (matvec(x=None), "NULL"), (matvec(w_scale=P + 1), "aligned"), (matvec(rows=-1), "rows"), (matvec(n=0), "rows"), (matvec(dtype=3), "dtype"), (B.daris_op(7, 0), "no operator"),
    (norm(width=(1 << 30) + 1), "2^30"), (norm(rows=(1 << 31) - 1), "2^30"), (append(n_rows=(1 << 30) + 1), "2^30"), (attend(n_rows=(1 << 31) - 1), "2^30"), (attend(cache(n_seqs=(1 << 31) - 1)), "2^30"),
    (matvec(k=(1 << 31) - 128, group=128), "2^30"), (matvec(n=(1 << 31) - 1), "2^30"), (matvec(rows=(1 << 30) + 1), "2^30"),
]


@pytest.mark.parametrize("i", range(len(WRONG)))
def test_wrong_descriptors_are_refused_and_named(i):
    op, word = WRONG[i]
    op.keep = ()
    with Session(HOST):
        D.daris_create_partition(8)
        good = norm()
        for call in (D.daris_plan_ops, D.daris_run_ops):
            with pytest.raises(D.DarisError) as e:
                call(D.make_ops([good, op]), 0)
            assert e.value.code == D.EINVAL and "operator 1" in str(e.value) and word in str(e.value), str(e.value)


def test_calls_out_of_place():
    ops = D.make_ops([norm()])
    with pytest.raises(D.DarisError) as e:
        D.daris_run_ops(ops, 0)
    assert e.value.code == D.ESTATE
    with Session(HOST):
        D.daris_create_partition(8)
        for p in (-1, 1):
            with pytest.raises(D.DarisError) as e:
                D.daris_run_ops(ops, p)
            assert e.value.code == D.ERANGE
        with pytest.raises(D.DarisError) as e:      # right descriptors, no device
            D.daris_run_ops(ops, 0)
        assert e.value.code == D.ESTATE
        lib = D.lib()
        assert lib.daris_run_ops(None, 1, 0) == D.EINVAL and lib.daris_run_ops(ops.array, -1, 0) == D.EINVAL
        assert lib.daris_run_plan(123456) == D.ERANGE and lib.daris_free_plan(123456) == D.ERANGE


def test_tensors_are_checked_before_they_become_addresses():
    x = torch.zeros((2, 64))
    for call in (lambda: D.make_norm(x, x[0], x, 1e-5), lambda: D.make_matvec(x, x, x, x), lambda: D.make_cache(x, x, x, x, x, x)):
        with pytest.raises(D.DarisError) as e:
            call()
        assert e.value.code == D.EINVAL and "GPU" in str(e.value)
    assert C.sizeof(B.daris_op) == 216
