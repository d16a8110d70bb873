"""ctypes binding of include/daris.h.  Function names and argument order follow the C ABI one to one;
the only additions are `make_dnn` (packs a Python layer table + numpy weights into a `daris_dnn`),
`trace_read_all` (decodes the 32-byte records) and error-code-to-exception conversion."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DARIS_LIB") or os.path.join(_HERE, "libdaris.so")   # DARIS_LIB: another build of the same sources

OK, EINVAL, ENOMEM, EHIP, ESTATE, ERANGE = 0, -1, -2, -3, -4, -5
VIRTUAL_TIME, NO_DEVICE, NO_LAST, NO_PRIOR, NO_FIXED, HP_ADMISSION, KEEP_ACTIVATIONS, WAVE_PRIORITY, SHARED_QUEUE = 1, 2, 4, 8, 16, 32, 64, 128, 256
NO_PAIR, NO_FUSED_INGEST, NO_STAGED_ROWS, NO_SMALL_TILES, NO_FUSED_DW, NO_TALL_TILES, NO_JOIN = 512, 1024, 2048, 4096, 8192, 16384, 32768
LP, HP = 0, 1
FP32, BF16 = 0, 1
ACCEPTED, MIGRATED, REJECT_ADMISSION, REJECT_OVERRUN, QUEUED = 1, 2, 3, 4, 5
T_RELEASE, T_ACCEPT, T_REJECT, T_MIGRATE, T_DISPATCH, T_STAGE_DONE, T_JOB_DONE, T_QUEUED, T_CMD_MIGRATE = range(1, 10)


class DarisError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"daris error {code}: {text}")
        self.code = code


class daris_layer(C.Structure):
    _fields_ = [("op", C.c_int32), ("c_in", C.c_int32), ("c_out", C.c_int32), ("k", C.c_int32), ("stride", C.c_int32),
                ("pad", C.c_int32), ("groups", C.c_int32), ("act", C.c_int32), ("in_from", C.c_int32),
                ("res_from", C.c_int32), ("w", C.POINTER(C.c_float)), ("b", C.POINTER(C.c_float))]


class daris_dnn(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("in_c", C.c_int32), ("in_h", C.c_int32), ("in_w", C.c_int32),
                ("dtype", C.c_int32), ("layers", C.POINTER(daris_layer))]


class daris_task_stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("released", "accepted", "completed", "missed", "rejected_admission",
                                         "rejected_overrun", "resp_min_ns", "resp_max_ns", "resp_sum_ns",
                                         "first_release_ns", "last_finish_ns")] + [("partition", C.c_int32), ("n_stages", C.c_int32)]


TRACE_DTYPE = np.dtype([("seq", "<u8"), ("t_ns", "<i8"), ("type", "u1"), ("level", "u1"), ("stage", "u1"),
                        ("partition", "u1"), ("task", "<u2"), ("stream", "<u2"), ("job", "<u4"), ("aux", "<u4")])
assert TRACE_DTYPE.itemsize == 32

_lib = None

_SIGS = {
    "daris_init": (C.c_int32, [C.c_int, C.c_uint64, C.c_int]),
    "daris_shutdown": (C.c_int32, []),
    "daris_set_timeout": (C.c_int32, [C.c_int64]),
    "daris_set_plan_cus": (C.c_int32, [C.c_int32]),
    "daris_last_error": (C.c_char_p, []),
    "daris_cu_per_partition": (C.c_int32, [C.c_int32] * 4),
    "daris_create_partition": (C.c_int32, [C.c_int]),
    "daris_partition_set_streams": (C.c_int32, [C.c_int32, C.c_int]),
    "daris_partition_get_mask": (C.c_int32, [C.c_int32, C.POINTER(C.c_uint32)]),
    "daris_register_task": (C.c_int32, [C.POINTER(daris_dnn), C.c_int64, C.c_int64, C.c_int]),
    "daris_split_stages": (C.c_int32, [C.c_int32, C.c_int]),
    "daris_get_stage_cuts": (C.c_int32, [C.c_int32, C.POINTER(C.c_int32), C.c_int32]),
    "daris_set_afet": (C.c_int32, [C.c_int32, C.c_int, C.c_int64]),
    "daris_set_window": (C.c_int32, [C.c_int]),
    "daris_set_virtual_time": (C.c_int32, [C.c_int32, C.c_int, C.c_int32, C.c_int64, C.c_int64, C.POINTER(C.c_int64)]),
    "daris_commit": (C.c_int32, []),
    "daris_get_partition": (C.c_int32, [C.c_int32]),
    "daris_release_job": (C.c_int32, [C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.POINTER(C.c_int32)]),
    "daris_migrate": (C.c_int32, [C.c_int32, C.c_int32]),
    "daris_run_until_idle": (C.c_int32, []),
    "daris_task_set_io": (C.c_int32, [C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32]),
    "daris_run_periodic": (C.c_int32, [C.POINTER(C.c_int64), C.POINTER(C.c_int32)]),
    "daris_run_closed_loop": (C.c_int32, [C.POINTER(C.c_int32), C.c_int64]),
    "daris_get_stats": (C.c_int32, [C.c_int32, C.POINTER(daris_task_stats)]),
    "daris_trace_read": (C.c_int64, [C.c_void_p, C.c_int64]),
    "daris_get_mret": (C.c_int64, [C.c_int32, C.c_int]),
    "daris_forward": (C.c_int32, [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32]),
    "daris_forward_static": (C.c_int32, [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32]),
    "daris_read_layer": (C.c_int32, [C.c_int32, C.c_int, C.POINTER(C.c_float), C.c_int64]),
    "daris_profile_layers": (C.c_int32, [C.c_int32, C.c_int32, C.c_int, C.POINTER(C.c_float), C.POINTER(C.c_int32), C.POINTER(C.c_double)]),
    "daris_kernel_name": (C.c_char_p, [C.c_int32]),
    "daris_calibrate_afet": (C.c_int32, [C.c_int32, C.c_int32, C.c_int]),
    "daris_calibrate_afet_loaded": (C.c_int32, [C.c_int32, C.c_int32, C.c_int]),
    "daris_kernel_timing_start": (C.c_int32, [C.c_int, C.c_int]),
    "daris_driver_profile": (C.c_int32, [C.c_int, C.POINTER(C.c_int64)]),
    "daris_get_launch_plan": (C.c_int32, [C.c_int32, C.c_int, C.POINTER(C.c_int64), C.c_int32]),
    "daris_kernel_timing_read": (C.c_int32, [C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "daris_probe_cus": (C.c_int32, [C.c_int32, C.c_int, C.c_int, C.POINTER(C.c_uint32)]),
}
EXPORTS = sorted(_SIGS)


def lib():
    """The loaded shared library; raises if libdaris.so has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise DarisError(ESTATE, f"{LIB_PATH} not built: run `python -m paper_2504_08795_amd.build`")
        # PyTorch owns the device memory the caller passes in, so both must use ONE HIP runtime: import torch first,
        # then libdaris.so binds to the libamdhip64.so.7 that torch has already mapped into the process.
        import torch  # noqa: F401
        _lib = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(_lib, name)
            f.restype, f.argtypes = res, args
    return _lib


def _chk(code):
    if code < 0:
        raise DarisError(code, lib().daris_last_error().decode())
    return code


def _ptr(x):
    """Device pointer of a torch tensor / int address / None."""
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return C.c_void_p(x.data_ptr())
    return C.c_void_p(int(x))


_device = None     # of the last daris_init


def daris_init(device=0, seed=0, flags=0):
    global _device
    code = _chk(lib().daris_init(device, seed, flags))
    _device = device
    return code


def daris_shutdown():
    return _chk(lib().daris_shutdown())


def daris_set_timeout(ns):
    return _chk(lib().daris_set_timeout(int(ns)))


def daris_set_plan_cus(n_cu):
    return _chk(lib().daris_set_plan_cus(int(n_cu)))


def daris_cu_per_partition(os_num, os_den, n_cu_max, n_c):
    return _chk(lib().daris_cu_per_partition(os_num, os_den, n_cu_max, n_c))


def daris_create_partition(n_cu):
    return _chk(lib().daris_create_partition(n_cu))


def daris_partition_set_streams(p, n_s):
    return _chk(lib().daris_partition_set_streams(p, n_s))


def daris_partition_get_mask(p):
    m = (C.c_uint32 * 8)()
    _chk(lib().daris_partition_get_mask(p, m))
    return list(m)


def make_dnn(layers, weights, in_shape, dtype):
    """Build a daris_dnn from records with fields op, c_in, c_out, k, stride, pad, groups, act, in_from, res_from and
    per-layer (w, b) float32 numpy arrays (or (None, None)).  Returns (dnn, keepalive)."""
    arr = (daris_layer * len(layers))()
    keep = [arr]
    fp = C.POINTER(C.c_float)
    for i, L in enumerate(layers):
        w, b = weights[i] if weights is not None else (None, None)
        a = arr[i]
        a.op, a.c_in, a.c_out, a.k, a.stride, a.pad = L.op, L.c_in, L.c_out, L.k, L.stride, L.pad
        a.groups, a.act, a.in_from, a.res_from = L.groups, L.act, L.in_from, L.res_from
        if w is not None:
            w = np.ascontiguousarray(w, np.float32)
            keep.append(w)
            a.w = w.ctypes.data_as(fp)
        if b is not None:
            b = np.ascontiguousarray(b, np.float32)
            keep.append(b)
            a.b = b.ctypes.data_as(fp)
    d = daris_dnn(len(layers), in_shape[0], in_shape[1], in_shape[2], BF16 if dtype in (BF16, "bf16") else FP32, arr)
    return d, keep


def daris_register_task(dnn, period_ns, deadline_ns, priority):
    return _chk(lib().daris_register_task(C.byref(dnn), period_ns, deadline_ns, priority))


def daris_split_stages(t, k):
    return _chk(lib().daris_split_stages(t, k))


def daris_get_stage_cuts(t):
    buf = (C.c_int32 * 256)()
    n = _chk(lib().daris_get_stage_cuts(t, buf, 256))
    return list(buf[:n])


PLAN_FIELDS = ("kernel_id", "dense_conv", "rows", "M", "N", "K", "Kpad", "tn", "nw", "S", "sz", "sw", "splitk", "MT", "NTn", "G", "xmode",
               "grid_x", "grid_y", "grid_z", "threads", "ws_bytes", "pair_with", "pair_lead", "out_slot", "in_slot", "res_slot", "gather")
# values of "gather": how a convolution's waves come by their pixels
GATHER_ALIGNED, GATHER_GENERAL, GATHER_INPUT, GATHER_ROWS, GATHER_DEPTHWISE, GATHER_TAPS, GATHER_IMAGE = range(7)


def daris_get_launch_plan(t, layer):
    buf = (C.c_int64 * 28)()
    _chk(lib().daris_get_launch_plan(t, layer, buf, 28))
    return dict(zip(PLAN_FIELDS, (int(v) for v in buf)))


def daris_set_afet(t, stage, ns):
    return _chk(lib().daris_set_afet(t, stage, int(ns)))


def daris_set_window(ws):
    return _chk(lib().daris_set_window(ws))


def daris_set_virtual_time(t, stage, p, job_lo, job_hi, et_ns):
    a = np.ascontiguousarray(et_ns, np.int64)
    assert a.size == job_hi - job_lo
    return _chk(lib().daris_set_virtual_time(t, stage, p, job_lo, job_hi, a.ctypes.data_as(C.POINTER(C.c_int64))))


def daris_commit():
    return _chk(lib().daris_commit())


def daris_get_partition(t):
    return _chk(lib().daris_get_partition(t))


def daris_release_job(t, d_input, d_logits, release_ns=-1):
    dec = C.c_int32(0)
    _chk(lib().daris_release_job(t, _ptr(d_input), _ptr(d_logits), int(release_ns), C.byref(dec)))
    return dec.value


def daris_migrate(t, p):
    return _chk(lib().daris_migrate(t, p))


def daris_run_until_idle():
    return _chk(lib().daris_run_until_idle())


def daris_task_set_io(t, d_inputs, n_inputs, d_logits, n_slots):
    return _chk(lib().daris_task_set_io(t, _ptr(d_inputs), n_inputs, _ptr(d_logits), n_slots))


def daris_run_periodic(phase_ns, n_jobs):
    n = np.ascontiguousarray(n_jobs, np.int32)
    ph = None if phase_ns is None else np.ascontiguousarray(phase_ns, np.int64)
    return _chk(lib().daris_run_periodic(None if ph is None else ph.ctypes.data_as(C.POINTER(C.c_int64)),
                                         n.ctypes.data_as(C.POINTER(C.c_int32))))


def daris_run_closed_loop(n_jobs, total_jobs=0):
    n = np.ascontiguousarray(n_jobs, np.int32)
    return _chk(lib().daris_run_closed_loop(n.ctypes.data_as(C.POINTER(C.c_int32)), int(total_jobs)))


def daris_get_stats(t):
    s = daris_task_stats()
    _chk(lib().daris_get_stats(t, C.byref(s)))
    return {n: getattr(s, n) for n, _ in daris_task_stats._fields_}


def daris_trace_read(max_records=1 << 16):
    buf = np.empty(max_records, TRACE_DTYPE)
    n = _chk(lib().daris_trace_read(buf.ctypes.data_as(C.c_void_p), buf.nbytes))
    return buf[: n // 32]


def trace_read_all():
    """All unread trace records as a list of tuples (seq, t, type, level, stage, partition, task, stream, job, aux)."""
    out = []
    while True:
        chunk = daris_trace_read()
        if len(chunk) == 0:
            return out
        out += [tuple(int(v) for v in r) for r in chunk.tolist()]


def daris_get_mret(t, stage):
    return _chk(lib().daris_get_mret(t, stage))


def daris_forward(t, d_input, d_logits, p=0):
    return _chk(lib().daris_forward(t, _ptr(d_input), _ptr(d_logits), p))


def daris_forward_static(t, d_input, d_logits, p=0):
    return _chk(lib().daris_forward_static(t, _ptr(d_input), _ptr(d_logits), p))


def daris_read_layer(t, layer, n_elems):
    out = np.empty(n_elems, np.float32)
    _chk(lib().daris_read_layer(t, layer, out.ctypes.data_as(C.POINTER(C.c_float)), n_elems))
    return out


def daris_profile_layers(t, p, reps, n_layers):
    ms = np.zeros(n_layers, np.float32)
    kid = np.zeros(n_layers, np.int32)
    fl = np.zeros(n_layers, np.float64)
    _chk(lib().daris_profile_layers(t, p, reps, ms.ctypes.data_as(C.POINTER(C.c_float)), kid.ctypes.data_as(C.POINTER(C.c_int32)),
                                    fl.ctypes.data_as(C.POINTER(C.c_double))))
    return ms, kid, fl


def daris_kernel_name(kernel_id):
    return lib().daris_kernel_name(int(kernel_id)).decode()


def daris_kernel_timing_start(every, max_samples):
    return _chk(lib().daris_kernel_timing_start(every, max_samples))


def daris_kernel_timing_read():
    """({kernel name: (launches, total_ms, total_flops)}, empty_pair_ms) of the sampled launches since daris_kernel_timing_start."""
    n, ms, fl = np.zeros(64, np.int64), np.zeros(64, np.float64), np.zeros(64, np.float64)
    ov = C.c_double(0.0)
    k = _chk(lib().daris_kernel_timing_read(64, n.ctypes.data_as(C.POINTER(C.c_int64)), ms.ctypes.data_as(C.POINTER(C.c_double)),
                                            fl.ctypes.data_as(C.POINTER(C.c_double)), C.byref(ov)))
    return {daris_kernel_name(i): (int(n[i]), float(ms[i]), float(fl[i])) for i in range(k) if n[i] > 0}, ov.value


def daris_driver_profile(enable):
    """Totals since the last call (dict, ns) of where the stages' wall time went; switches the gathering on or off."""
    out = np.zeros(8, np.int64)
    _chk(lib().daris_driver_profile(int(bool(enable)), out.ctypes.data_as(C.POINTER(C.c_int64))))
    keys = ("stages", "enqueue_ns", "wait_ns", "lock_ns", "sched_ns", "gpu_ns", "handover_ns")
    return {k: int(out[i]) for i, k in enumerate(keys)}


def daris_calibrate_afet(t, p, reps=5):
    return _chk(lib().daris_calibrate_afet(t, p, reps))


def daris_calibrate_afet_loaded(t, p, reps=5):
    return _chk(lib().daris_calibrate_afet_loaded(t, p, reps))


def daris_probe_cus(p, n_groups=2048, spin=2000):
    """(xcc_id, hw_id) per workgroup of a probe launch on stream 0 of partition p."""
    out = np.zeros(2 * n_groups, np.uint32)
    _chk(lib().daris_probe_cus(p, n_groups, spin, out.ctypes.data_as(C.POINTER(C.c_uint32))))
    return out.reshape(n_groups, 2)


# ---- operators of a generation step (include/daris_ops.h) ------------------------------------------------------------------

STEP_NORM, STEP_APPEND, STEP_ATTEND, STEP_MATVEC, STEP_TREE_APPEND, STEP_TREE_ATTEND, STEP_SAMPLE = range(7)
STEP_ACCEPT, STEP_KEEP, STEP_COPY = range(8, 11)
PAGE_TOKENS, SCALE_TOKENS, TREE_WORDS, SAMPLE_WORDS = 64, 16, 16, 1 << 20


def _struct(name, *fields):
    return type(name, (C.Structure,), {"_fields_": [(f, t) for t, fs in fields for f in fs.split()]})


_P, _L, _I, _F = C.c_void_p, C.c_int64, C.c_int32, C.c_float
daris_norm = _struct("daris_norm", (_P, "x res weight sum y scale"), (_L, "x_row res_row sum_row y_row"), (_I, "rows width group dtype"), (_F, "eps"))
daris_cache = _struct("daris_cache", (_P, "k v k_scale v_scale pages before"), (_L, "pages_row"), (_I, "n_pages n_seqs kv_heads dim"))
daris_append = _struct("daris_append", (daris_cache, "cache"), (_P, "k v q q_out turn row_start"),
                       (_L, "k_row k_head v_row v_head q_row q_head qo_row qo_head"), (_I, "n_rows q_heads dtype turn_rows rot_dim pairs"))
daris_attend = _struct("daris_attend", (daris_cache, "cache"), (_P, "q out row_start"), (_L, "q_row q_head out_row out_head"),
                       (_I, "n_rows q_heads dtype window"), (_F, "scale"))
daris_matvec = _struct("daris_matvec", (_P, "x x_scale w w_scale y"), (_L, "x_row w_row y_row"), (_I, "rows n k group dtype gate"))

daris_tree_append = _struct("daris_tree_append", (daris_cache, "cache"), (_P, "k v q q_out turn row_start tree"), (_L, "kv_row kv_head q_row q_head qo_row qo_head"),
                            (_I, "n_rows q_heads dtype turn_rows rot_dim pairs tree_words"))
daris_tree_attend = _struct("daris_tree_attend", (daris_attend, "attend"), (_P, "tree"), (_I, "tree_words"))
daris_sample = _struct("daris_sample", (_P, "logits temperature top_k top_p min_p random word chance"), (_L, "logits_row"), (_I, "rows n dtype"))
daris_accept = _struct("daris_accept", (_P, "tree words answers row_start before path count word after"), (_I, "n_rows n_seqs tree_words"))
daris_keep = _struct("daris_keep", (daris_cache, "cache"), (_P, "path count row_start"), (_I, "n_rows"))
daris_copy = _struct("daris_copy", (daris_cache, "cache"), (_P, "pairs"), (_I, "n"))
_KINDS = {STEP_NORM: "norm", STEP_APPEND: "append", STEP_ATTEND: "attend", STEP_MATVEC: "matvec", STEP_TREE_APPEND: "tree_append", STEP_TREE_ATTEND: "tree_attend",
          STEP_SAMPLE: "sample", STEP_ACCEPT: "accept", STEP_KEEP: "keep", STEP_COPY: "copy"}


class _step(C.Union):
    _fields_ = [(name, globals()["daris_" + name]) for name in _KINDS.values()]


class daris_op(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("u", _step)]


_SIGS.update({
    "daris_run_ops": (C.c_int32, [C.POINTER(daris_op), C.c_int32, C.c_int32]),
    "daris_plan_ops": (C.c_int32, [C.POINTER(daris_op), C.c_int32, C.c_int32]),
    "daris_run_plan": (C.c_int32, [C.c_int32]),
    "daris_free_plan": (C.c_int32, [C.c_int32]),
})
EXPORTS = sorted(_SIGS)


def _need(ok, text):
    if not ok:
        raise DarisError(EINVAL, text)


def _tensor(name, t, dims, dtypes):
    """Checks what a descriptor cannot say: a GPU tensor of one of `dtypes` with `dims` dimensions, the last one's elements side by side."""
    _need(hasattr(t, "data_ptr") and t.is_cuda, f"{name} is no GPU tensor")
    _need(t.dim() == dims, f"{name} has {t.dim()} dimensions, not {dims}")
    _need(str(t.dtype)[6:] in dtypes, f"{name} is of {t.dtype}, not {' or '.join(dtypes)}")
    _need(t.shape[-1] <= 1 or t.stride(-1) == 1, f"{name}'s last dimension is strided")
    return t


def _dense(name, t, shape, dtypes):
    _tensor(name, t, len(shape), dtypes)
    _need(tuple(t.shape) == tuple(shape), f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    _need(t.is_contiguous(), f"{name} is not contiguous")
    return t


_ACT = ("bfloat16", "float32")
_F8 = ("float8_e4m3fn",)
_E8 = ("float8_e8m0fnu", "uint8")


def _like(name, t, x):
    _need(t.dtype == x.dtype, f"{name} is of {t.dtype}, not {x.dtype}")
    return t


def _dtype(t):
    return BF16 if str(t.dtype) == "torch.bfloat16" else FP32


def _at(t):
    return t.data_ptr() if t is not None else None


def _made(kind, value, *keep):
    op = daris_op(kind, 0)
    setattr(op.u, _KINDS[kind], value)
    op.keep = keep      # the buffers live as long as their descriptor
    return op


def make_norm(x, weight, y, eps, res=None, sum=None, scale=None):
    """y = norm(x + res) * weight for tensors [rows][width] (see daris_norm); y in float8_e4m3fn with scale [rows][width / group]."""
    _tensor("x", x, 2, _ACT)
    rows, width = x.shape
    _like("weight", _dense("weight", weight, (width,), _ACT), x)
    for name, t in (("res", res), ("sum", sum)):
        if t is not None:
            _need(tuple(_like(name, _tensor(name, t, 2, _ACT), x).shape) == (rows, width), f"{name} is {tuple(t.shape)}, not {(rows, width)}")
    _tensor("y", y, 2, _F8 if scale is not None else _ACT)
    _need(tuple(y.shape) == (rows, width), f"y is {tuple(y.shape)}, not {(rows, width)}")
    group = 0
    if scale is None:
        _like("y", y, x)
    else:
        _tensor("scale", scale, 2, _E8)
        _need(scale.shape[1] > 0 and width % scale.shape[1] == 0, f"{scale.shape[1]} scales for rows of {width}")
        group = width // scale.shape[1]
        _dense("scale", scale, (rows, width // group), _E8)
    return _made(STEP_NORM, daris_norm(_at(x), _at(res), _at(weight), _at(sum), _at(y), _at(scale), x.stride(0), res.stride(0) if res is not None else 0,
                                       sum.stride(0) if sum is not None else 0, y.stride(0), rows, width, group, _dtype(x), eps), x, weight, y, res, sum, scale)


def make_cache(k, v, k_scale, v_scale, pages, before):
    """A paged cache (see daris_cache): k [pages][heads][64][dim] and v [pages][heads][dim][64] in float8_e4m3fn, scales [pages][heads][4],
    pages int32 [sequences][entries], before int32 [sequences]."""
    _tensor("k", k, 4, _F8)
    n, h, _, d = k.shape
    _dense("k", k, (n, h, PAGE_TOKENS, d), _F8)
    _dense("v", v, (n, h, d, PAGE_TOKENS), _F8)
    _dense("k_scale", k_scale, (n, h, PAGE_TOKENS // SCALE_TOKENS), _E8)
    _dense("v_scale", v_scale, (n, h, PAGE_TOKENS // SCALE_TOKENS), _E8)
    _tensor("pages", pages, 2, ("int32",))
    _dense("before", before, (pages.shape[0],), ("int32",))
    _need(pages.shape[0] <= 1 or pages.stride(0) == pages.shape[1], "pages is not contiguous")
    c = daris_cache(_at(k), _at(v), _at(k_scale), _at(v_scale), _at(pages), _at(before), pages.shape[1], n, pages.shape[0], h, d)
    c.keep = (k, v, k_scale, v_scale, pages, before)
    return c


def _rows(cache, name, t, row_start, heads=None):
    _tensor(name, t, 3, _ACT)
    _need(t.shape[2] == cache.dim, f"{name} has heads of {t.shape[2]}, the cache of {cache.dim}")
    _need(heads is None or t.shape[1] == heads, f"{name} has {t.shape[1]} heads, not {heads}")
    if row_start is not None:
        _dense("row_start", row_start, (cache.n_seqs + 1,), ("int32",))
    return t


def _tree(t, rows):
    _tensor("tree", t, 2, ("int64", "uint64"))
    _need(1 <= t.shape[1] <= TREE_WORDS, f"masks of {t.shape[1]} words, not 1 to {TREE_WORDS}")
    return _dense("tree", t, (rows, t.shape[1]), ("int64", "uint64"))


def tree_masks(parents, words=None):
    """Masks [rows][words] (an int64 tensor of the CPU) of trees: parents[s][i] is the node of sequence s above node i, which lies in front of it, or -1 for
    one that hangs on the cached tokens.  A node's mask has the bits of itself and of all nodes above it."""
    import torch
    most = max([len(p) for p in parents] + [1])
    words = -(-most // 64) if words is None else words
    _need(most <= 64 * words and 1 <= words <= TREE_WORDS, f"trees of up to {most} nodes in {words} words of 64, {TREE_WORDS} words at most")
    out = np.zeros((sum(len(p) for p in parents), words), np.uint64)
    at = 0
    for s, p in enumerate(parents):
        for i, above in enumerate(p):
            _need(-1 <= above < i, f"node {i} of sequence {s} is below node {above}")
            if above >= 0:
                out[at + i] = out[at + above]
            out[at + i, i // 64] |= np.uint64(1 << (i % 64))
        at += len(p)
    return torch.from_numpy(out.view(np.int64))


def make_append(cache, k, v, row_start=None, q=None, q_out=None, turn=None, rot_dim=0, pairs=False, tree=None):
    """Appends rows k, v [rows][heads][dim] to the cache, keys and q -> q_out turned by turn [positions][rot_dim] (see daris_append); tree: masks
    [rows][words] of rows that are nodes of trees (see daris_tree_append)."""
    _rows(cache, "k", k, row_start, cache.kv_heads)
    _like("v", _rows(cache, "v", v, row_start, cache.kv_heads), k)
    _need(v.shape[0] == k.shape[0], f"{v.shape[0]} rows of v, {k.shape[0]} of k")
    _need((q is None) == (q_out is None), "q and q_out go together")
    for name, t in (("q", q), ("q_out", q_out)):
        if t is not None:
            _need(_like(name, _rows(cache, name, t, row_start, q.shape[1]), k).shape[0] == k.shape[0], f"{t.shape[0]} rows of {name}, {k.shape[0]} of k")
    if turn is not None:
        _dense("turn", turn, (turn.shape[0], rot_dim), ("float32",))
    _need(turn is not None or rot_dim == 0, "no table of angles")
    z = (0, 0, 0)
    a = daris_append(cache, _at(k), _at(v), _at(q), _at(q_out), _at(turn), _at(row_start), *k.stride()[:2], *v.stride()[:2], *(q.stride() if q is not None else z)[:2],
                     *(q_out.stride() if q is not None else z)[:2], k.shape[0], q.shape[1] if q is not None else 0, _dtype(k), turn.shape[0] if turn is not None else 0, rot_dim, int(pairs))
    if tree is None:
        return _made(STEP_APPEND, a, cache, k, v, q, q_out, turn, row_start)
    _tree(tree, k.shape[0])
    _need(all(k.shape[d] <= 1 or k.stride(d) == v.stride(d) for d in (0, 1)), f"with a tree, k and v lie alike: their distances are {k.stride()[:2]} and {v.stride()[:2]}")
    t = daris_tree_append(cache, a.k, a.v, a.q, a.q_out, a.turn, a.row_start, _at(tree), a.k_row, a.k_head, a.q_row, a.q_head, a.qo_row, a.qo_head,
                          a.n_rows, a.q_heads, a.dtype, a.turn_rows, a.rot_dim, a.pairs, tree.shape[1])
    return _made(STEP_TREE_APPEND, t, cache, k, v, q, q_out, turn, row_start, tree)


def make_attend(cache, q, out, row_start=None, scale=1.0, window=0, tree=None):
    """out = attention of q [rows][heads][dim] over the cache (see daris_attend); tree: masks [rows][words] of rows that are nodes of trees (see daris_tree_attend)."""
    _rows(cache, "q", q, row_start)
    _need(_like("out", _rows(cache, "out", out, row_start, q.shape[1]), q).shape[0] == q.shape[0], f"{out.shape[0]} rows of out, {q.shape[0]} of q")
    a = daris_attend(cache, _at(q), _at(out), _at(row_start), *q.stride()[:2], *out.stride()[:2], q.shape[0], q.shape[1], _dtype(q), window, scale)
    if tree is None:
        return _made(STEP_ATTEND, a, cache, q, out, row_start)
    _tree(tree, q.shape[0])
    return _made(STEP_TREE_ATTEND, daris_tree_attend(a, _at(tree), tree.shape[1]), cache, q, out, row_start, tree)


def make_sample(logits, word, random=None, temperature=None, top_k=None, top_p=None, min_p=None, chance=None):
    """word [rows] (int32) drawn from logits [rows][n] by random [rows] (see daris_sample); temperature, top_p, min_p, chance [rows] of float32, top_k of int32."""
    _tensor("logits", logits, 2, _ACT)
    rows, n = logits.shape
    _dense("word", word, (rows,), ("int32",))
    for name, t in (("random", random), ("temperature", temperature), ("top_p", top_p), ("min_p", min_p), ("chance", chance)):
        if t is not None:
            _dense(name, t, (rows,), ("float32",))
    if top_k is not None:
        _dense("top_k", top_k, (rows,), ("int32",))
    a = daris_sample(_at(logits), _at(temperature), _at(top_k), _at(top_p), _at(min_p), _at(random), _at(word), _at(chance), logits.stride(0), rows, n, _dtype(logits))
    return _made(STEP_SAMPLE, a, logits, word, random, temperature, top_k, top_p, min_p, chance)


def make_accept(tree, words, answers, path, count, word, row_start=None, before=None, after=None):
    """Walks down the trees of masks tree [rows][words]: path [rows], count and word [sequences] from words and answers [rows], all int32 (see daris_accept);
    after = before + count [sequences]."""
    rows = _tensor("words", words, 1, ("int32",)).shape[0]
    _dense("words", words, (rows,), ("int32",))
    _tree(tree, rows)
    _dense("answers", answers, (rows,), ("int32",))
    _dense("path", path, (rows,), ("int32",))
    seqs = _tensor("count", count, 1, ("int32",)).shape[0]
    _dense("count", count, (seqs,), ("int32",))
    for name, t in (("word", word), ("before", before), ("after", after)):
        if t is not None or name == "word":
            _dense(name, t, (seqs,), ("int32",))
    if row_start is not None:
        _dense("row_start", row_start, (seqs + 1,), ("int32",))
    a = daris_accept(_at(tree), _at(words), _at(answers), _at(row_start), _at(before), _at(path), _at(count), _at(word), _at(after), rows, seqs, tree.shape[1])
    return _made(STEP_ACCEPT, a, tree, words, answers, path, count, word, row_start, before, after)


def make_keep(cache, path, count, row_start=None):
    """Keeps the tokens of the nodes path [rows] (count [sequences] of each sequence), int32, one behind the other in the cache (see daris_keep)."""
    _dense("path", path, (_tensor("path", path, 1, ("int32",)).shape[0],), ("int32",))
    _dense("count", count, (cache.n_seqs,), ("int32",))
    if row_start is not None:
        _dense("row_start", row_start, (cache.n_seqs + 1,), ("int32",))
    return _made(STEP_KEEP, daris_keep(cache, _at(path), _at(count), _at(row_start), path.shape[0]), cache, path, count, row_start)


def make_copy(cache, pairs):
    """Copies pages pairs[i][0] of the cache over pages pairs[i][1], pairs [n][2] of int32 (see daris_copy)."""
    _dense("pairs", pairs, (_tensor("pairs", pairs, 2, ("int32",)).shape[0], 2), ("int32",))
    return _made(STEP_COPY, daris_copy(cache, _at(pairs), pairs.shape[0]), cache, pairs)


def make_matvec(x, w, w_scale, y, x_scale=None, gate=False):
    """y [rows][n] = x [rows][k] times 4-bit weights w [n][k / 2] (uint8) with scales w_scale [n][k / group] (bfloat16); x in float8_e4m3fn with
    x_scale [rows][k / group]; gate: y [rows][n / 2] (see daris_matvec)."""
    _tensor("x", x, 2, _F8 if x_scale is not None else _ACT)
    _tensor("w", w, 2, ("uint8",))
    rows, k = x.shape
    n = w.shape[0]
    _need(k == 2 * w.shape[1], f"x has {k} channels, w {2 * w.shape[1]}")
    _tensor("w_scale", w_scale, 2, ("bfloat16",))
    _need(w_scale.shape[1] > 0 and k % w_scale.shape[1] == 0, f"{w_scale.shape[1]} scales for {k} channels")
    group = k // w_scale.shape[1]
    _dense("w_scale", w_scale, (n, k // group), ("bfloat16",))
    if x_scale is not None:
        _dense("x_scale", x_scale, (rows, k // group), _E8)
    _tensor("y", y, 2, _ACT)
    _need(x_scale is not None or y.dtype == x.dtype, f"y is of {y.dtype}, not {x.dtype}")
    _need(tuple(y.shape) == (rows, n // 2 if gate else n), f"y is {tuple(y.shape)}, not {(rows, n // 2 if gate else n)}")
    a = daris_matvec(_at(x), _at(x_scale), _at(w), _at(w_scale), _at(y), x.stride(0), w.stride(0), y.stride(0), rows, n, k, group, _dtype(y), int(gate))
    return _made(STEP_MATVEC, a, x, w, w_scale, y, x_scale)


class Ops:
    """Operators in the order in which they run; holds their buffers, and their plan on each partition that has run them."""

    def __init__(self, ops):
        self.array = (daris_op * len(ops))(*ops)
        self.keep = tuple(o.keep for o in ops)
        self.plans = {}

    def __len__(self):
        return len(self.array)

    def __del__(self):
        if _lib is not None:
            for plan in self.plans.values():
                _lib.daris_free_plan(plan)


def make_ops(ops):
    """Operators in the order in which they run, as daris_run_ops takes them; a program keeps it from step to step."""
    return Ops(ops)


def _kept(things):
    for t in things:
        if hasattr(t, "device"):
            yield t
        elif hasattr(t, "keep"):
            yield from _kept(t.keep)


def daris_plan_ops(ops, p=0):
    for i, things in enumerate(ops.keep):
        for t in _kept(things):
            _need(_device is None or t.device.index == _device, f"operator {i}: a tensor is on {t.device}, the library on device {_device}")
    return _chk(lib().daris_plan_ops(ops.array, len(ops), p))


def daris_run_plan(plan):
    return _chk(lib().daris_run_plan(plan))


def daris_free_plan(plan):
    return _chk(lib().daris_free_plan(plan))


def daris_run_ops(ops, p=0):
    """Runs what make_ops made on partition p and waits for it: planned by the first run there (and by the first after a daris_shutdown)."""
    plan = ops.plans.get(p)
    if plan is not None:
        code = lib().daris_run_plan(plan)
        if code != ERANGE:
            return _chk(code)
    ops.plans[p] = plan = daris_plan_ops(ops, p)
    return daris_run_plan(plan)
