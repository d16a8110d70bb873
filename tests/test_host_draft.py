"""The operators of a drafted step on the host: what their descriptors' checks refuse, trees as masks, and that every launch covers its work.  No GPU."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_2504_08795_amd as D
from draft_helpers import bits_of, drawn, walk
from lib_helpers import Session
from paper_2504_08795_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
HOST = D.VIRTUAL_TIME | D.NO_DEVICE
P = 1 << 20      # an address that nothing reads: the checks come before any launch, and there is no device


@pytest.fixture(scope="module")
def encode(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("draft") / "driver")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           "-o", exe, os.path.join(HERE, "host_steps", "draft.cpp")])

    def run(*lines):
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, ln)) for ln in lines) + "\n", capture_output=True, text=True, check=True)
        return [ln if ln.startswith("error") else [int(v) for v in ln.split()] for ln in r.stdout.splitlines()]
    return run


def test_descriptors_are_laid_out_as_in_c(encode):
    names = ("op", "tree_append", "tree_attend", "sample", "accept", "keep", "copy")
    want = [C.sizeof(getattr(B, "daris_" + n)) for n in names] + [B.daris_tree_append.tree_words.offset, B.daris_tree_attend.tree_words.offset, B.daris_sample.dtype.offset]
    assert encode(("sizes",))[0] == want


def test_launches_cover_their_work(encode):
    for rows, n, dtype, offset, row in ((1, 50001, 0, 0, 50001), (2, 50001, 0, 0, 50001), (64, 131072, 1, 0, 131072), (3, 7, 1, 2, 8), (5, 512, 0, 16, 516), (1, 1 << 20, 1, 0, 0), (5000, 30000, 1, 0, 30000), (9, 16384, 0, 4, 16385)):
        kernel, groups, threads, lds, part, counters, first, parts, part_chunks, chunks = encode(("sample", rows, n, dtype, offset, row))[0]
        assert kernel == 4 and groups == rows and threads == 1024 and lds <= 80 * 1024 and counters == 0, "two workgroups a CU"
        assert chunks == -(-n // 512) and (parts - 1) * part_chunks < chunks <= parts * part_chunks and part_chunks in (16, 32) and parts <= 128
        assert (first, part) == ((0, 0) if parts == 1 else (rows * parts, rows * 4 * ((chunks + 1) // 2 * 2 + 2 * chunks + 3 * 1024 * parts)))
    for rows, seqs, words in ((26, 1, 1), (3000, 512, 4), (0, 3, 16)):
        assert encode(("accept", rows, seqs, words))[0][:3] == [7, seqs, 64]
    for rows, seqs, kv, dim in ((26, 1, 8, 128), (200, 7, 3, 64), (9, 9, 1, 256)):
        p = encode(("keep", rows, seqs, kv, dim))[0]
        assert p[0] == 5 and p[1] * 4 >= 2 * seqs * kv > (p[1] - 1) * 4 and p[2] == 256
    for n, pages, kv, dim in ((1, 3, 8, 128), (1001, 2003, 8, 128), (7, 9, 1, 64), (2, 5, 12, 256)):
        p = encode(("copy", n, pages, kv, dim))[0]
        assert p[0] == 6 and p[-1] * 16384 >= kv * 64 * dim > (p[-1] - 1) * 16384 and p[1] == 2 * n * p[-1]
    assert "workgroups" in encode(("copy", 1 << 29, 1 << 30, 8, 128))[0]
    p = encode(("append", 1000, 20, 3, 5, 128, 2))[0]
    assert p[0] == 1 and p[-3] == (1000 // 16 + 40) * 3 * 2 and p[-2] == 2000 and p[-1] == 2
    narrow, wide = encode(("attend", 64, 4, 32, 8, 128, 1, 1, 256), ("attend", 64 * 32, 32, 32, 8, 128, 1, 4, 256))
    assert narrow[0] == 2 and wide[0] == 3 and wide[-1] == 4
    for dtype, dim, kernel in ((D.FP32, 64, 3), (D.FP32, 128, 2), (D.BF16, 128, 3), (D.BF16, 256, 2)):
        assert encode(("attend", 64 * 32, 32, 32, 8, dim, dtype, 1, 256))[0][0] == kernel


def test_operators_without_rows_are_no_launches(encode):
    for line in (("sample", 0, 7, 0, 0, 7), ("accept", 0, 0, 1), ("keep", 0, 0, 1, 64), ("copy", 0, 5, 1, 64), ("copy", 3, 0, 1, 64), ("append", 0, 3, 1, 1, 64, 1), ("attend", 0, 3, 1, 1, 64, 1, 1, 8)):
        assert encode(line)[0][1] == 0, line


def cache(**kw):
    c = B.daris_cache()
    for n, v in dict(dict(k=P, v=P, k_scale=P, v_scale=P, pages=P, before=P, pages_row=4, n_pages=4, n_seqs=2, kv_heads=2, dim=64), **kw).items():
        setattr(c, n, v)
    return c


def _op(kind, value, defaults, changes):
    for n, v in dict(defaults, **changes).items():
        setattr(value, n, v)
    op = B._made(kind, value)
    op.keep = ()
    return op


def append(c=None, **kw):
    return _op(D.STEP_TREE_APPEND, B.daris_tree_append(), dict(cache=c or cache(), k=P, v=P, q=P, q_out=P, turn=P, row_start=P, tree=P, n_rows=2, q_heads=4, dtype=D.BF16, turn_rows=9, rot_dim=64, tree_words=1), kw)


def attend(c=None, tree=P, tree_words=1, **kw):
    a = B.daris_attend()
    for n, v in dict(dict(cache=c or cache(), q=P, out=P, row_start=P, n_rows=2, q_heads=4, dtype=D.BF16, scale=1.0), **kw).items():
        setattr(a, n, v)
    return _op(D.STEP_TREE_ATTEND, B.daris_tree_attend(), dict(attend=a, tree=tree, tree_words=tree_words), {})


def sample(**kw):
    return _op(D.STEP_SAMPLE, B.daris_sample(), dict(logits=P, word=P, random=P, logits_row=64, rows=2, n=64, dtype=D.FP32), kw)


def accept(**kw):
    return _op(D.STEP_ACCEPT, B.daris_accept(), dict(tree=P, words=P, answers=P, row_start=P, path=P, count=P, word=P, n_rows=2, n_seqs=2, tree_words=1), kw)


def keep(c=None, **kw):
    return _op(D.STEP_KEEP, B.daris_keep(), dict(cache=c or cache(), path=P, count=P, row_start=P, n_rows=2), kw)


def copy(c=None, **kw):
    return _op(D.STEP_COPY, B.daris_copy(), dict(cache=c or cache(pages=None, before=None), pairs=P, n=2), kw)


BIG = (1 << 30) + 1
WRONG = [
    (append(cache(dim=96)), "dim"), (append(tree=None), "no masks"), (append(tree=P + 4), "8 bytes"), (append(tree_words=0), "0 words"), (append(tree_words=17), "17 words"), (append(k=None), "NULL"),
    (append(rot_dim=65), "rot_dim"), (append(row_start=None, n_rows=3), "without row_start"), (append(n_rows=BIG), "2^30"), (append(dtype=5), "dtype"),
    (attend(tree=None), "no masks"), (attend(tree_words=-1), "-1 words"), (attend(tree=P + 1), "8 bytes"), (attend(q_heads=5), "key heads"), (attend(window=-1), "window"), (attend(cache(before=P + 2)), "4 bytes"),
    (sample(dtype=2), "dtype"), (sample(rows=-1), "rows"), (sample(n=0), "rows"), (sample(n=(1 << 20) + 1), "2^20"), (sample(rows=BIG), "2^30"), (sample(logits=None), "NULL"), (sample(word=None), "NULL"),
    (sample(logits=P + 2), "aligned"), (sample(top_k=P + 1), "aligned"), (sample(chance=P + 2), "aligned"),
    (accept(tree=None), "no masks"), (accept(tree_words=20), "20 words"), (accept(words=None), "NULL"), (accept(count=None), "NULL"), (accept(word=None), "NULL"), (accept(path=P + 1), "4 bytes"),
    (accept(after=P), "without before"), (accept(row_start=None, n_rows=3), "without row_start"), (accept(n_rows=-1), "count"), (accept(n_seqs=BIG), "2^30"),
    (keep(cache(dim=0)), "dim"), (keep(path=None), "NULL"), (keep(count=None), "NULL"), (keep(count=P + 2), "4 bytes"), (keep(cache(k=P + 8)), "16 bytes"), (keep(n_rows=BIG), "2^30"),
    (keep(row_start=None, n_rows=1), "without row_start"),
    (copy(cache(dim=100)), "dim"), (copy(n=-1), "count"), (copy(n=BIG), "2^30"), (copy(pairs=None), "NULL"), (copy(cache(v=P + 8)), "16 bytes"), (copy(cache(k_scale=P + 1)), "4 bytes"), (copy(cache(kv_heads=0)), "count"),
    (copy(pairs=P + 2), "4 bytes"),
]


@pytest.mark.parametrize("i", range(len(WRONG)))
def test_wrong_descriptors_are_refused_and_named(i):
    op, word = WRONG[i]
    with Session(HOST):
        D.daris_create_partition(8)
        good = sample()
        for call in (D.daris_plan_ops, D.daris_run_ops):
            with pytest.raises(D.DarisError) as e:
                call(D.make_ops([good, op]), 0)
            assert e.value.code == D.EINVAL and "operator 1" in str(e.value) and word in str(e.value), str(e.value)


def test_right_descriptors_get_past_the_checks():
    with Session(HOST):
        D.daris_create_partition(8)
        for op in (append(), attend(), sample(), accept(), keep(), copy(), append(n_rows=0, tree=None), sample(rows=0, logits=None), accept(n_rows=0, words=None, path=None, answers=None, tree=None), copy(n=0, pairs=None)):
            with pytest.raises(D.DarisError) as e:      # (no device)
                D.daris_run_ops(D.make_ops([op]), 0)
            assert e.value.code == D.ESTATE, str(e.value)


def test_tensors_are_checked_before_they_become_addresses():
    x, i = torch.zeros((2, 64)), torch.zeros(2, dtype=torch.int32)
    c = B.daris_cache()
    c.n_seqs, c.dim, c.kv_heads = 2, 64, 1
    c.keep = ()
    for call in (lambda: D.make_sample(x, i), lambda: D.make_accept(i, i, i, i, i, i), lambda: D.make_keep(c, i, i), lambda: D.make_copy(c, i.view(1, 2)), lambda: D.make_append(c, x[None], x[None], tree=i),
                 lambda: D.make_attend(c, x[None], x[None], tree=i)):
        with pytest.raises(D.DarisError) as e:
            call()
        assert e.value.code == D.EINVAL and "GPU" in str(e.value)


def test_trees_as_masks():
    m = D.tree_masks([[-1, 0, 0, 1, 3], [], [-1], [-1, -1, 1]])
    assert m.dtype == torch.int64 and [bits_of(r.tolist()) for r in m] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [0], [0], [1], [1, 2]]
    m = D.tree_masks([list(range(-1, 129))], words=4)
    assert m.shape == (130, 4) and bits_of(m[129].tolist()) == list(range(130)) and m[63, 0] == -1
    assert D.tree_masks([[]]).shape == (0, 1)
    for wrong, words in (([[0]], None), ([[-1, 1]], None), ([[-2]], None), ([[-1] * 65], 1), ([[-1] * 1025], None), ([[-1]], 17), ([[-1]], 0)):
        with pytest.raises(D.DarisError) as e:
            D.tree_masks(wrong, words)
        assert e.value.code == D.EINVAL


def test_the_definitions_on_small_cases():
    """The plain forms that GPU results are compared with, on cases worked by hand."""
    x = torch.tensor([0.0, 1.0, 1.0, -1.0])
    e = 2.718281828459045
    total = 1 + 2 * e + 1 / e
    assert drawn(x, 0.0) == (0, pytest.approx(1 / total)) and drawn(x, 0.16)[0] == 1 and drawn(x, 1 / total + 1e-9)[0] == 1 and drawn(x, 0.999)[0] == 3
    assert drawn(x, 0.999, top_k=1) == (1, 1.0) and drawn(x, 0.999, top_k=2) == (2, 0.5) and drawn(x, 0.0, top_k=3)[0] == 0
    assert drawn(x, 0.999, top_p=0.39)[0] == 1 and drawn(x, 0.999, top_p=0.5)[0] == 2 and drawn(x, 0.999, top_p=0.0)[0] == 1
    assert drawn(x, 0.999, min_p=0.5)[0] == 2 and drawn(x, 0.0, min_p=0.3)[0] == 0 and drawn(x, 0.999, min_p=7.0) == (1, 1.0)
    assert drawn(x, 0.999, temperature=0.0) == (1, 1.0) and drawn(torch.full((3,), float("nan")), 0.5) == (-1, 0.0)
    masks = D.tree_masks([[-1, 0, 0, 1, 1, 2]])
    assert walk(masks, [9, 5, 6, 7, 7, 8], [5, 7, 0, 1, 2, 3]) == ([0, 1, 3], 1)     # of equal words the first node
    assert walk(masks, [9, 5, 6, 7, 7, 8], [4, 7, 0, 1, 2, 3]) == ([0], 4) and walk(masks, [9, -1, 6, 7, 7, 8], [-1, 7, 0, 1, 2, 3]) == ([0], -1)
