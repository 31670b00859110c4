"""Python binding of libnopfs.so (argument marshalling only).

Every computation runs in the library's HIP kernels; this module only turns
torch tensors (device memory) and torch's current stream into the C ABI's
pointers. It raises ``NopfsError`` for a non-zero status and ``RuntimeError``
if the compiled library is missing: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch  # loads the HIP runtime before the library does

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libnopfs.so")

NOPFS_OK, NOPFS_EINVAL, NOPFS_ERANGE, NOPFS_ENOMEM, NOPFS_EDEVICE = 0, -1, -2, -3, -4


class NopfsError(RuntimeError):
    def __init__(self, code: int, what: str, detail: str):
        super().__init__(f"{what}: status {code} ({detail})")
        self.code = code


class _Job(ctypes.Structure):
    _fields_ = [("F", ctypes.c_int64), ("E", ctypes.c_int32),
                ("N", ctypes.c_int32), ("B", ctypes.c_int32),
                ("drop_last", ctypes.c_int32), ("seed", ctypes.c_uint64)]


@dataclass(frozen=True)
class Job:
    """A training job as the paper states it: F samples, E epochs, N workers,
    per-worker batch B, drop_last, shuffle seed."""
    F: int
    E: int
    N: int
    B: int
    drop_last: int = 1
    seed: int = 42

    def c(self) -> _Job:
        return _Job(int(self.F), int(self.E), int(self.N), int(self.B),
                    int(self.drop_last), int(self.seed) & ((1 << 64) - 1))

    def epochs(self, e_begin: int, e_end: int) -> "Job":
        """The shape of epochs [e_begin, e_end) of this job: what
        access_streams_range writes, and what the stats, next-use and plan
        calls take for those epochs' streams. (Its own access_streams would
        draw epochs 0.., not e_begin..: use access_streams_range.)"""
        return Job(self.F, int(e_end) - int(e_begin), self.N, self.B, self.drop_last, self.seed)


class Model(ctypes.Structure):
    """Parameters of the performance model (nopfs_model): bytes, bytes/s,
    seconds; r and p per cache tier."""
    _fields_ = [("c", ctypes.c_double), ("beta", ctypes.c_double), ("b_c", ctypes.c_double),
                ("pfs_t", ctypes.c_double), ("pfs_gamma", ctypes.c_double),
                ("w0", ctypes.c_double), ("p0", ctypes.c_double),
                ("J", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("r", ctypes.c_double * 32), ("p", ctypes.c_double * 32)]


def make_model(c, beta, b_c, pfs_t, pfs_gamma, w0, p0, r, p) -> Model:
    m = Model()
    m.c, m.beta, m.b_c = float(c), float(beta), float(b_c)
    m.pfs_t, m.pfs_gamma, m.w0, m.p0 = float(pfs_t), float(pfs_gamma), float(w0), float(p0)
    m.J = len(r)
    for j, (rj, pj) in enumerate(zip(list(r)[:32], list(p)[:32])):
        m.r[j], m.p[j] = float(rj), float(pj)
    return m


class _Batch(ctypes.Structure):
    _fields_ = ([(x, ctypes.c_int64) for x in ("F", "ids_stride", "free_stride")]
                + [(x, ctypes.c_int32) for x in ("G", "n", "blocks", "block", "width", "cap")]
                + [("scratch", ctypes.c_void_p), ("scratch_bytes", ctypes.c_int64)])


class _Attention(ctypes.Structure):
    # a stride[2] of the C struct is a pair of fields here: token, head
    _fields_ = ([("T", ctypes.c_int64)]
                + [(x, ctypes.c_int32) for x in ("n", "heads", "kv_heads", "width", "dtype")]
                + [("scale", ctypes.c_float)]
                + [(f"{x}_{y}", ctypes.c_int64)
                   for x in ("q", "k", "v", "o", "do", "dq", "dk", "dv") for y in ("token", "head")]
                + [("scratch", ctypes.c_void_p), ("scratch_bytes", ctypes.c_int64)])


class _Distill(ctypes.Structure):
    _fields_ = ([(x, ctypes.c_int64) for x in ("T", "V", "logits_stride", "grad_stride",
                                               "index_stride", "teacher_stride")]
                + [(x, ctypes.c_int32) for x in ("K", "dtype", "teacher_dtype")]
                + [("tau", ctypes.c_float)])


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the compiled library (fails loudly if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python paper_2101_08734_amd/build.py` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        P, I64, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        jp = ctypes.POINTER(_Job)
        sig = {
            "nopfs_stream_shape": [jp, P, P, P],
            "nopfs_access_streams": [jp, P, P],
            "nopfs_access_stats": [jp, P, P, P, P],
            "nopfs_reuse_next": [jp, P, P, P],
            "nopfs_tier_plan": [jp, P, P, P, P, I32, P, P, P],
            "nopfs_plan_job": [jp, P, P, I32, P, P, P, P, P, P, P],
            "nopfs_plan_job_noalloc": [jp, P, P, I32, P, P, P, P, P, P, P],
            "nopfs_prefetch_order": [jp, P, P, I32, P, P, P],
            "nopfs_staging_schedule": [jp, P, P, I64, P, P],
            "nopfs_fetch_model": [jp, P, P, P, ctypes.POINTER(Model), P, P, P],
            "nopfs_buffer_sim": [jp, P, P, P, I64, P, P, P],
            "nopfs_access_streams_range": [jp, ctypes.c_int32, ctypes.c_int32, P, P],
            "nopfs_policy_sim": [jp, P, P, P, P, ctypes.POINTER(Model), ctypes.c_int32, P, P, P, P],
            "nopfs_batch_tables": [ctypes.POINTER(_Batch)] + [P] * 10,
            "nopfs_batch_tables_scratch": [ctypes.POINTER(_Batch), P],
            "nopfs_packed_attention_scratch": [ctypes.POINTER(_Attention), ctypes.c_int32, P],
            "nopfs_packed_attention": [ctypes.POINTER(_Attention)] + [P] * 7,
            "nopfs_packed_attention_grad": [ctypes.POINTER(_Attention)] + [P] * 11,
            "nopfs_topk_distill": [ctypes.POINTER(_Distill)] + [P] * 7,
            "nopfs_profile_enable": [ctypes.c_int],
            "nopfs_profile_query": [ctypes.c_int, ctypes.POINTER(ctypes.c_char_p),
                                    ctypes.POINTER(I64), ctypes.POINTER(ctypes.c_double)],
            "nopfs_calibration_copy": [P, P, I64, P],
            "nopfs_scratch_release": [P],
            "nopfs_debug_set": [ctypes.c_int, I64],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        L.nopfs_strerror.argtypes = [ctypes.c_int]
        L.nopfs_strerror.restype = ctypes.c_char_p
        L.nopfs_last_error.argtypes = []
        L.nopfs_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


EXPORTED = ("nopfs_stream_shape", "nopfs_access_streams", "nopfs_access_streams_range",
            "nopfs_access_stats",
            "nopfs_reuse_next", "nopfs_tier_plan", "nopfs_plan_job", "nopfs_plan_job_noalloc",
            "nopfs_prefetch_order",
            "nopfs_staging_schedule", "nopfs_fetch_model", "nopfs_buffer_sim", "nopfs_policy_sim",
            "nopfs_batch_tables", "nopfs_packed_attention", "nopfs_packed_attention_grad",
            "nopfs_batch_tables_scratch", "nopfs_packed_attention_scratch",
            "nopfs_topk_distill", "nopfs_strerror",
            "nopfs_last_error", "nopfs_profile_enable", "nopfs_profile_query",
            "nopfs_calibration_copy", "nopfs_scratch_release", "nopfs_debug_set")


def _check(rc: int, what: str):
    if rc != NOPFS_OK:
        L = lib()
        detail = L.nopfs_last_error().decode() or L.nopfs_strerror(rc).decode()
        raise NopfsError(rc, what, detail)


def _ptr(t) -> ctypes.c_void_p:
    if t is None:
        return ctypes.c_void_p(0)
    if isinstance(t, int):
        return ctypes.c_void_p(t)
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _device_tensor(t, dtype, shape, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t


def stream_shape(job: Job):
    """(T, M_max, [M_i]) on the host; no GPU needed."""
    T = ctypes.c_int64()
    M = ctypes.c_int64()
    Mw = (ctypes.c_int64 * int(job.N))()
    j = job.c()
    _check(lib().nopfs_stream_shape(ctypes.byref(j), ctypes.byref(T), ctypes.byref(M), Mw),
           "nopfs_stream_shape")
    return T.value, M.value, list(Mw)


def access_streams(job: Job, R=None, stream=None):
    _, M, _ = stream_shape(job)
    if R is None:
        R = torch.empty((job.N, M), dtype=torch.int32, device="cuda")
    _device_tensor(R, torch.int32, (job.N, M), "R")
    j = job.c()
    _check(lib().nopfs_access_streams(ctypes.byref(j), _ptr(R), _stream(stream)),
           "nopfs_access_streams")
    return R


def access_stats(job: Job, R, count=None, first=None, stream=None):
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    if count is None:
        count = torch.empty((job.N, job.F), dtype=torch.uint8, device="cuda")
    if first is None:
        first = torch.empty((job.N, job.F), dtype=torch.int32, device="cuda")
    _device_tensor(count, torch.uint8, (job.N, job.F), "count")
    _device_tensor(first, torch.int32, (job.N, job.F), "first")
    j = job.c()
    _check(lib().nopfs_access_stats(ctypes.byref(j), _ptr(R), _ptr(count), _ptr(first),
                                    _stream(stream)), "nopfs_access_stats")
    return count, first


def access_streams_range(job: Job, e_begin: int, e_end: int, R=None, stream=None):
    """Streams of epochs [e_begin, e_end) (nopfs_access_streams_range), shaped
    as the streams of job.epochs(e_begin, e_end)."""
    sub = job.epochs(e_begin, e_end)
    M = stream_shape(sub)[1] if e_end > e_begin else 0
    if R is None:
        R = torch.empty((job.N, M), dtype=torch.int32, device="cuda")
    _device_tensor(R, torch.int32, (job.N, M), "R")
    j = job.c()
    _check(lib().nopfs_access_streams_range(ctypes.byref(j), int(e_begin), int(e_end), _ptr(R),
                                            _stream(stream)), "nopfs_access_streams_range")
    return R


def reuse_next(job: Job, R, next=None, stream=None):
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    if next is None:
        next = torch.empty((job.N, M), dtype=torch.int32, device="cuda")
    _device_tensor(next, torch.int32, (job.N, M), "next")
    j = job.c()
    _check(lib().nopfs_reuse_next(ctypes.byref(j), _ptr(R), _ptr(next), _stream(stream)),
           "nopfs_reuse_next")
    return next


def tier_plan(job: Job, count, first, sizes, caps, tier=None, used=None, stream=None):
    """caps: host sequence of per-worker tier capacities (bytes), fastest first."""
    _device_tensor(count, torch.uint8, (job.N, job.F), "count")
    _device_tensor(first, torch.int32, (job.N, job.F), "first")
    _device_tensor(sizes, torch.int64, (job.F,), "sizes")
    caps_list = [int(c) for c in caps]
    J = len(caps_list)
    caps_host = (ctypes.c_int64 * max(J, 1))(*caps_list)
    if tier is None:
        tier = torch.empty((job.N, job.F), dtype=torch.int8, device="cuda")
    if used is None:
        used = torch.empty((job.N, max(J, 1)), dtype=torch.int64, device="cuda")
    _device_tensor(tier, torch.int8, (job.N, job.F), "tier")
    _device_tensor(used, torch.int64, (job.N, max(J, 1)), "used")
    j = job.c()
    _check(lib().nopfs_tier_plan(ctypes.byref(j), _ptr(count), _ptr(first), _ptr(sizes),
                                 ctypes.cast(caps_host, ctypes.c_void_p), J, _ptr(tier),
                                 _ptr(used), _stream(stream)), "nopfs_tier_plan")
    return tier, used


def plan_job(job: Job, sizes, caps, out=None, stream=None):
    """The whole path in one library call (nopfs_plan_job); the same outputs
    as plan(). `out` may hold preallocated R, count, first, next, tier, used."""
    return _plan_job("nopfs_plan_job", job, sizes, caps, out, stream)


def plan_job_noalloc(job: Job, sizes, caps, out, stream=None):
    """nopfs_plan_job_noalloc: plan_job with the library's fixed per-device
    scratch array, no device allocation by the library. `out` must hold all
    six preallocated outputs."""
    for name in ("R", "count", "first", "next", "tier", "used"):
        if out.get(name) is None:
            raise ValueError(f"plan_job_noalloc needs a preallocated {name}")
    return _plan_job("nopfs_plan_job_noalloc", job, sizes, caps, out, stream)


def _plan_job(fn, job: Job, sizes, caps, out, stream):
    _, M, _ = stream_shape(job)
    _device_tensor(sizes, torch.int64, (job.F,), "sizes")
    caps_list = [int(c) for c in caps]
    J = len(caps_list)
    caps_host = (ctypes.c_int64 * max(J, 1))(*caps_list)
    shapes = dict(R=((job.N, M), torch.int32), count=((job.N, job.F), torch.uint8),
                  first=((job.N, job.F), torch.int32), next=((job.N, M), torch.int32),
                  tier=((job.N, job.F), torch.int8), used=((job.N, max(J, 1)), torch.int64))
    o = dict(out or {})
    for name, (shape, dt) in shapes.items():
        if o.get(name) is None:
            o[name] = torch.empty(shape, dtype=dt, device="cuda")
        _device_tensor(o[name], dt, shape, name)
    j = job.c()
    _check(getattr(lib(), fn)(ctypes.byref(j), _ptr(sizes), ctypes.cast(caps_host, ctypes.c_void_p),
                              J, _ptr(o["R"]), _ptr(o["count"]), _ptr(o["first"]), _ptr(o["next"]),
                              _ptr(o["tier"]), _ptr(o["used"]), _stream(stream)), fn)
    return o


def prefetch_order(job: Job, R, tier, J, order=None, qlen=None, stream=None):
    """Per-tier prefetch queues (nopfs_prefetch_order): order [N][M_max] int32
    (tier 0's queue, tier 1's, ..., then -1) and qlen [N][J] int64."""
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    _device_tensor(tier, torch.int8, (job.N, job.F), "tier")
    J = int(J)
    if order is None:
        order = torch.empty((job.N, M), dtype=torch.int32, device="cuda")
    if qlen is None:
        qlen = torch.empty((job.N, max(J, 1)), dtype=torch.int64, device="cuda")
    _device_tensor(order, torch.int32, (job.N, M), "order")
    _device_tensor(qlen, torch.int64, (job.N, max(J, 1)), "qlen")
    j = job.c()
    _check(lib().nopfs_prefetch_order(ctypes.byref(j), _ptr(R), _ptr(tier), J,
                                      _ptr(order), _ptr(qlen), _stream(stream)),
           "nopfs_prefetch_order")
    return order, qlen


def staging_schedule(job: Job, R, sizes, d0, fill=None, stream=None):
    """Staging-buffer schedule (nopfs_staging_schedule): fill [N][M_max] int32,
    the first stream position from which each read's sample may be staged
    into a buffer of d0 bytes (-1 in padding)."""
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    _device_tensor(sizes, torch.int64, (job.F,), "sizes")
    if fill is None:
        fill = torch.empty((job.N, M), dtype=torch.int32, device="cuda")
    _device_tensor(fill, torch.int32, (job.N, M), "fill")
    j = job.c()
    _check(lib().nopfs_staging_schedule(ctypes.byref(j), _ptr(R), _ptr(sizes), int(d0), _ptr(fill),
                                        _stream(stream)), "nopfs_staging_schedule")
    return fill


def fetch_model(job: Job, R, tier, sizes, model: Model, src=None, t=None, stream=None):
    """Fetch source and consumption time of every read under the performance
    model (nopfs_fetch_model): src [N][M_max] int16 (0 PFS, 128 + j another
    worker's tier j, 256 + j own tier j, -1 padding), t [N][M_max] float64
    seconds (-1 padding)."""
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    _device_tensor(tier, torch.int8, (job.N, job.F), "tier")
    _device_tensor(sizes, torch.int64, (job.F,), "sizes")
    if src is None:
        src = torch.empty((job.N, M), dtype=torch.int16, device="cuda")
    if t is None:
        t = torch.empty((job.N, M), dtype=torch.float64, device="cuda")
    _device_tensor(src, torch.int16, (job.N, M), "src")
    _device_tensor(t, torch.float64, (job.N, M), "t")
    j = job.c()
    _check(lib().nopfs_fetch_model(ctypes.byref(j), _ptr(R), _ptr(tier), _ptr(sizes),
                                   ctypes.byref(model), _ptr(src), _ptr(t), _stream(stream)),
           "nopfs_fetch_model")
    return src, t


def buffer_sim(job: Job, R, next, sizes, d0, hit=None, hits=None, stream=None):
    """Clairvoyant buffer of d0 bytes per worker (nopfs_buffer_sim): hit
    [N][M_max] int8 (1 hit, 0 miss, -1 padding), hits [N][2] int64 (hits, hit
    bytes)."""
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    _device_tensor(next, torch.int32, (job.N, M), "next")
    _device_tensor(sizes, torch.int64, (job.F,), "sizes")
    if hit is None:
        hit = torch.empty((job.N, M), dtype=torch.int8, device="cuda")
    if hits is None:
        hits = torch.empty((job.N, 2), dtype=torch.int64, device="cuda")
    _device_tensor(hit, torch.int8, (job.N, M), "hit")
    _device_tensor(hits, torch.int64, (job.N, 2), "hits")
    j = job.c()
    _check(lib().nopfs_buffer_sim(ctypes.byref(j), _ptr(R), _ptr(next), _ptr(sizes), int(d0),
                                  _ptr(hit), _ptr(hits), _stream(stream)), "nopfs_buffer_sim")
    return hit, hits


POLICY_PERFECT, POLICY_NAIVE, POLICY_STAGING, POLICY_NOPFS = 0, 1, 2, 3


def policy_sim(job: Job, R, sizes, model, policy, src=None, fill=None, t=None, finish=None,
               io=None, stream=None):
    """Simulated training time under a data-loading policy (nopfs_policy_sim):
    t [N][M_max] float64 consumption times (-1 padding), finish [N], io
    [N][1 + 2J] fetch time by source class."""
    _, M, _ = stream_shape(job)
    _device_tensor(R, torch.int32, (job.N, M), "R")
    _device_tensor(sizes, torch.int64, (job.F,), "sizes")
    if src is not None:
        _device_tensor(src, torch.int16, (job.N, M), "src")
    if fill is not None:
        _device_tensor(fill, torch.int32, (job.N, M), "fill")
    K = 1 + 2 * model.J
    if t is None:
        t = torch.empty((job.N, M), dtype=torch.float64, device="cuda")
    if finish is None:
        finish = torch.empty(job.N, dtype=torch.float64, device="cuda")
    if io is None:
        io = torch.empty((job.N, K), dtype=torch.float64, device="cuda")
    _device_tensor(t, torch.float64, (job.N, M), "t")
    _device_tensor(finish, torch.float64, (job.N,), "finish")
    _device_tensor(io, torch.float64, (job.N, K), "io")
    j = job.c()
    _check(lib().nopfs_policy_sim(ctypes.byref(j), _ptr(R), _ptr(sizes),
                                  None if src is None else _ptr(src),
                                  None if fill is None else _ptr(fill), ctypes.byref(model),
                                  int(policy), _ptr(t), _ptr(finish), _ptr(io), _stream(stream)),
           "nopfs_policy_sim")
    return t, finish, io


def plan(job: Job, sizes, caps, stream=None):
    """The whole path: streams, stats, next use, tier plan (all on device)."""
    R = access_streams(job, stream=stream)
    count, first = access_stats(job, R, stream=stream)
    nxt = reuse_next(job, R, stream=stream)
    tier, used = tier_plan(job, count, first, sizes, caps, stream=stream)
    return dict(R=R, count=count, first=first, next=nxt, tier=tier, used=used)


# -- a training step on the reads that come next ------------------------------------
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}  # NOPFS_BF16, _FP16, _FP32


def _step_tensor(t, name, dtypes, ndim, device):
    """A device tensor of one of these types and this many dimensions, adjacent
    along the last one, on the current device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be of type " + " or ".join(str(d) for d in dtypes))
    if t.dim() != ndim or (t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{name} must have {ndim} dimensions, the last one adjacent in memory")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on device {device}, where the call runs")
    return t


def _step_shape(t, name, shape):
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")


def _dense(t, name):
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _step_dense(t, name, dtype, shape, device):
    """A contiguous device tensor of this type and shape on the current device:
    one test where it is one, the reason where it is not."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape
            and t.is_contiguous() and t.get_device() == device):
        return t
    _step_shape(_step_tensor(t, name, (dtype,), len(shape), device), name, shape)
    return _dense(t, name)


# The current stream's handle without the object around it, which takes 1 us to
# make, a tenth of a small call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def _step_stream(stream, device, tensors):
    """The stream's handle. Where it is not the current one, the allocator is
    told that the call's tensors are in use there."""
    if stream is None:
        return _raw_stream(device)
    if stream.cuda_stream != _raw_stream(device):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    return stream.cuda_stream


# Whether the current stream is being captured into a graph.
_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None) or torch.cuda.is_current_stream_capturing


def _step_scratch(desc, device, stream, size, *args):
    """Scratch for a call that is being captured into a graph, from torch's
    allocator, which keeps it as long as the graph (elsewhere the library has its
    own). The function `size` tells how much. The current stream is asked: a call
    captured on another one while the current one is not is refused."""
    if stream is not None and stream.cuda_stream != _raw_stream(device):
        with torch.cuda.stream(stream):
            return _step_scratch(desc, device, None, size, *args)
    need = ctypes.c_int64()
    _check(getattr(lib(), size)(ctypes.byref(desc), *args, ctypes.byref(need)), size)
    t = torch.empty(need.value, dtype=torch.uint8, device=device)
    desc.scratch, desc.scratch_bytes = t.data_ptr(), need.value
    return t


def _row_stride(t):
    """Elements from row to row; a single row's stride says nothing."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


_I32 = (torch.int32,)


def batch_tables(ids, tokens, free, block: int, width: int, cap: int, out=None, stream=None):
    """Block tables and slot maps of the next reads (nopfs_batch_tables), from
    their lengths in tokens.

    ids [G][n] int32, the reads of G workers (columns of the streams R, say);
    tokens [F] int32, every sample's length. With ids None, tokens [G][n] holds
    the reads' lengths. free [G][blocks] int32, each worker's free blocks of
    `block` tokens. Returns start [G][n+1], table [G][n][width], row and pos
    [G][cap], used [G][3] (reads, tokens, blocks) as int32 and slot [G][cap] as
    int64; `out` may hold any of them preallocated."""
    dev = torch.cuda.current_device()
    free = _step_tensor(free, "free", _I32, 2, dev)
    if ids is None:
        lead, F = _step_tensor(tokens, "tokens", _I32, 2, dev), 0
    else:
        lead = _step_tensor(ids, "ids", _I32, 2, dev)
        F = _dense(_step_tensor(tokens, "tokens", _I32, 1, dev), "tokens").shape[0]
    G, n = lead.shape
    block, width, cap = int(block), int(width), int(cap)
    if free.shape[0] != G:
        raise ValueError(f"free must have {G} rows")
    if not (0 < block < 2**31 and 0 < width < 2**31 and 0 <= cap < 2**31):
        raise ValueError("block and width must be positive, cap not negative, all below 2^31")
    o = dict(out) if out else {}
    for name, shape, dt in (("start", (G, n + 1), torch.int32), ("table", (G, n, width), torch.int32),
                            ("slot", (G, cap), torch.int64), ("row", (G, cap), torch.int32),
                            ("pos", (G, cap), torch.int32), ("used", (G, 3), torch.int32)):
        t = o.get(name)
        if t is None:
            o[name] = lead.new_empty(shape, dtype=dt)
        else:
            _step_dense(t, name, dt, shape, dev)
    b = _Batch(F, _row_stride(lead), _row_stride(free), G, n, free.shape[1], block, width, cap)
    st = _step_stream(stream, dev, (ids, tokens, free, *o.values()))
    scratch = _capturing() and _step_scratch(  # noqa: F841 held until the call is enqueued
        b, dev, stream, "nopfs_batch_tables_scratch")
    _check(lib().nopfs_batch_tables(
        ctypes.byref(b), None if ids is None else ids.data_ptr(), tokens.data_ptr(),
        free.data_ptr(), o["start"].data_ptr(), o["table"].data_ptr(), o["slot"].data_ptr(),
        o["row"].data_ptr(), o["pos"].data_ptr(), o["used"].data_ptr(), st), "nopfs_batch_tables")
    return o


def _no_outputs_given(name, *outputs):
    if any(t is not None for t in outputs):
        raise ValueError(f"{name}: given outputs are not part of the graph of an input that "
                         "requires a gradient (detach it, or call under torch.no_grad())")


def _call_in_backward(stream, call):
    """A call that the forward pass made on `stream`, behind what the backward
    pass has on its own stream and before what follows there."""
    if stream is None:
        return call()
    here = torch.cuda.current_stream()
    stream.wait_stream(here)
    out = call()
    here.wait_stream(stream)
    return out


_HALVES = (torch.bfloat16, torch.float16)


def _attention(q, k, v, start, scale, dev):
    _step_tensor(q, "q", _HALVES, 3, dev)
    T, heads, width = q.shape
    same = (q.dtype,)
    kv_heads = _step_tensor(k, "k", same, 3, dev).shape[1]
    _step_shape(k, "k", (T, kv_heads, width))
    _step_shape(_step_tensor(v, "v", same, 3, dev), "v", (T, kv_heads, width))
    if _dense(_step_tensor(start, "start", _I32, 1, dev), "start").shape[0] < 1:
        raise ValueError("start must have an entry before every sample and one behind the last")
    if scale is None:
        scale = width ** -0.5 if width else 0.0
    return T, start.shape[0] - 1, heads, kv_heads, width, _DTYPES[q.dtype], scale


def _strides(*tensors):
    """Token and head strides of each. That of a single token or head says
    nothing: what the array would have when dense."""
    out = []
    for t in tensors:
        T, heads, width = t.shape
        token, head, _ = t.stride()
        out += (token if T > 1 else heads * width, head if heads > 1 else width)
    return out


class _PackedAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, start, scale, stream):
        o, lse = packed_attention(q, k, v, start, scale, stream=stream)
        ctx.save_for_backward(q, k, v, o, lse, start)
        ctx.scale, ctx.stream = scale, stream
        ctx.set_materialize_grads(False)
        return o, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do, dlse):
        if dlse is not None:
            raise RuntimeError("packed_attention: lse has no gradient (detach it)")
        if do is None:
            return (None,) * 6
        q, k, v, o, lse, start = ctx.saved_tensors
        token, head, element = do.stride()
        if element != 1 or token % 8 or head % 8 or min(token, head) < do.shape[2] or do.data_ptr() % 16:
            do = do.clone(memory_format=torch.contiguous_format)
        grads = _call_in_backward(ctx.stream, lambda: packed_attention_grad(
            do, q, k, v, o, lse, start, ctx.scale, stream=ctx.stream))
        return (*grads, None, None, None)


def packed_attention(q, k, v, start, scale=None, o=None, lse=None, stream=None):
    """Causal attention over packed samples (nopfs_packed_attention): q
    [T][heads][width], k and v [T][kv_heads][width], bfloat16 or float16, any
    token and head strides of whole 16 bytes (slices of one projection, say);
    start [n+1] int32, a row of batch_tables' start. Returns o (as q) and lse
    [heads][T] float32. scale: 1/sqrt(width) unless given. Autograd takes o back to
    q, k and v by packed_attention_grad."""
    if (q.requires_grad or k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        _no_outputs_given("packed_attention", o, lse)
        return _PackedAttention.apply(q, k, v, start, scale, stream)
    dev = torch.cuda.current_device()
    a = _attention(q, k, v, start, scale, dev)
    if o is None:
        o = q.new_empty(q.shape)
    else:
        _step_shape(_step_tensor(o, "o", (q.dtype,), 3, dev), "o", q.shape)
    if lse is None:
        lse = q.new_empty((a[2], a[0]), dtype=torch.float32)
    else:
        _step_dense(lse, "lse", torch.float32, (a[2], a[0]), dev)
    a = _Attention(*a, *_strides(q, k, v, o))
    st = _step_stream(stream, dev, (q, k, v, start, o, lse))
    scratch = _capturing() and _step_scratch(  # noqa: F841
        a, dev, stream, "nopfs_packed_attention_scratch", 0)
    _check(lib().nopfs_packed_attention(ctypes.byref(a), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                        start.data_ptr(), o.data_ptr(), lse.data_ptr(), st),
           "nopfs_packed_attention")
    return o, lse


def packed_attention_grad(do, q, k, v, o, lse, start, scale=None, dq=None, dk=None, dv=None,
                          stream=None):
    """Gradient of packed_attention (nopfs_packed_attention_grad) from its
    outputs and the gradient `do` of o. Returns dq, dk, dv (as q, k, v; slices
    of one preallocated array, say), which autograd does not differentiate again."""
    dev = torch.cuda.current_device()
    a = _attention(q, k, v, start, scale, dev)
    same = (q.dtype,)
    for name, t in (("do", do), ("o", o)):
        _step_shape(_step_tensor(t, name, same, 3, dev), name, q.shape)
    _step_dense(lse, "lse", torch.float32, (a[2], a[0]), dev)
    grads = []
    for name, t, like in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        if t is None:
            t = q.new_empty(like.shape)
        else:
            _step_shape(_step_tensor(t, name, same, 3, dev), name, like.shape)
        grads.append(t)
    dq, dk, dv = grads
    a = _Attention(*a, *_strides(q, k, v, o, do, dq, dk, dv))
    st = _step_stream(stream, dev, (do, q, k, v, o, lse, start, dq, dk, dv))
    scratch = _capturing() and _step_scratch(  # noqa: F841
        a, dev, stream, "nopfs_packed_attention_scratch", 1)
    _check(lib().nopfs_packed_attention_grad(
        ctypes.byref(a), do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
        lse.data_ptr(), start.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), st),
        "nopfs_packed_attention_grad")
    return dq, dk, dv


class _TopkDistill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, index, teacher, tau, weight, stream):
        loss, dlogits = topk_distill(logits, index, teacher, tau, weight, stream=stream)
        ctx.save_for_backward(dlogits)
        ctx.mark_non_differentiable(dlogits)
        ctx.set_materialize_grads(False)
        ctx.stream = stream
        return loss, dlogits

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, _):
        if dloss is None:
            return (None,) * 6
        dlogits, = ctx.saved_tensors
        if ctx.stream is not None:
            torch.cuda.current_stream().wait_stream(ctx.stream)
        return ((dlogits * dloss[:, None]).to(dlogits.dtype), None, None, None, None, None)


def topk_distill(logits, index, teacher, tau=1.0, weight=None, grad=True, loss=None, dlogits=None,
                 stream=None):
    """Distillation from a teacher's top logits (nopfs_topk_distill): logits
    [T][V], index [T][K] int32 and teacher [T][K], the teacher's K classes per
    row and their logits; weight [T] float32 scales a row's loss (0: the row is
    masked). Returns loss [T] float32 and, unless grad is False, its gradient
    by the logits (in their type; dlogits may be logits itself). Autograd takes the
    loss back to the logits by that gradient; with grad False the loss is outside
    its graph. Teacher and weight are data and may not require gradients."""
    if teacher.requires_grad or weight is not None and weight.requires_grad:
        if torch.is_grad_enabled():
            raise ValueError("topk_distill has no gradient by teacher and weight (detach them)")
    if grad and logits.requires_grad and torch.is_grad_enabled():
        _no_outputs_given("topk_distill", loss, dlogits)
        return _TopkDistill.apply(logits, index, teacher, tau, weight, stream)
    dev = torch.cuda.current_device()
    T, V = _step_tensor(logits, "logits", _DTYPES, 2, dev).shape
    K = _step_tensor(index, "index", _I32, 2, dev).shape[1]
    _step_shape(index, "index", (T, K))
    _step_shape(_step_tensor(teacher, "teacher", _DTYPES, 2, dev), "teacher", (T, K))
    if weight is not None:
        _step_dense(weight, "weight", torch.float32, (T,), dev)
    if loss is None:
        loss = logits.new_empty(T, dtype=torch.float32)
    else:
        _step_dense(loss, "loss", torch.float32, (T,), dev)
    if not grad:
        dlogits = None
    elif dlogits is None:
        dlogits = logits.new_empty((T, V))
    else:
        _step_shape(_step_tensor(dlogits, "dlogits", (logits.dtype,), 2, dev), "dlogits", (T, V))
    d = _Distill(T, V, _row_stride(logits), 0 if dlogits is None else _row_stride(dlogits),
                 _row_stride(index), _row_stride(teacher), K, _DTYPES[logits.dtype],
                 _DTYPES[teacher.dtype], tau)
    st = _step_stream(stream, dev, (logits, index, teacher, weight, loss, dlogits))
    _check(lib().nopfs_topk_distill(
        ctypes.byref(d), logits.data_ptr(), index.data_ptr(), teacher.data_ptr(),
        None if weight is None else weight.data_ptr(), loss.data_ptr(),
        None if dlogits is None else dlogits.data_ptr(), st), "nopfs_topk_distill")
    return loss, dlogits


# -- measurement aids -----------------------------------------------------------
def profile_enable(on: bool):
    _check(lib().nopfs_profile_enable(1 if on else 0), "nopfs_profile_enable")


def profile_results():
    """{kernel name: (launches, total ms)} for kernels since profile_enable(True)."""
    out = {}
    idx = 0
    while True:
        name = ctypes.c_char_p()
        n = ctypes.c_int64()
        ms = ctypes.c_double()
        rc = lib().nopfs_profile_query(idx, ctypes.byref(name), ctypes.byref(n), ctypes.byref(ms))
        if rc == NOPFS_EINVAL:
            break
        _check(rc, "nopfs_profile_query")
        out[name.value.decode()] = (n.value, ms.value)
        idx += 1
    return out


def scratch_release(stream=None):
    """Frees the scratch block of (current device, stream) after the
    stream's work completes (nopfs_scratch_release)."""
    _check(lib().nopfs_scratch_release(_stream(stream)), "nopfs_scratch_release")


def calibration_copy(src, dst, nbytes: int, stream=None):
    _check(lib().nopfs_calibration_copy(_ptr(src), _ptr(dst), int(nbytes), _stream(stream)),
           "nopfs_calibration_copy")


def debug_set(which: int, value: int):
    _check(lib().nopfs_debug_set(int(which), int(value)), "nopfs_debug_set")
