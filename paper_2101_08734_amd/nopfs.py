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
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

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


_SCRATCH = [("scratch", ctypes.c_void_p), ("scratch_bytes", ctypes.c_int64)]


class _Embed(ctypes.Structure):
    _fields_ = ([(x, ctypes.c_int64) for x in ("T", "V", "n_ids", "weight_stride", "out_stride")]
                + [(x, ctypes.c_int32) for x in ("width", "weight_dtype", "dtype", "id_bytes")]
                + [("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + _SCRATCH)


class _Rotate(ctypes.Structure):
    # a stride[2] of the C struct is a pair of fields here: token, head
    _fields_ = ([("T", ctypes.c_int64)]
                + [(x, ctypes.c_int32) for x in ("heads", "kv_heads", "width", "rotated", "interleaved",
                                                 "dtype", "weight_dtype")]
                + [("eps", ctypes.c_float)]
                + [(f"{x}_{y}", ctypes.c_int64)
                   for x in ("q", "k", "q_out", "k_out", "dq", "dk") for y in ("token", "head")]
                + _SCRATCH)


class _Scan(ctypes.Structure):
    _fields_ = ([("T", ctypes.c_int64)]
                + [(x, ctypes.c_int32) for x in ("n", "channels", "dtype", "reserved")]
                + [(x + "_stride", ctypes.c_int64) for x in ("x", "gate", "h", "dh", "dx", "dgate")]
                + _SCRATCH)


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
            "nopfs_token_embed": [ctypes.POINTER(_Embed)] + [P] * 5,
            "nopfs_token_embed_names": [ctypes.POINTER(_Embed)] + [P] * 6,
            "nopfs_token_embed_grad": [ctypes.POINTER(_Embed)] + [P] * 5,
            "nopfs_token_embed_scratch": [ctypes.POINTER(_Embed), P],
            "nopfs_norm_rotate": [ctypes.POINTER(_Rotate)] + [P] * 9,
            "nopfs_norm_rotate_grad": [ctypes.POINTER(_Rotate)] + [P] * 13,
            "nopfs_norm_rotate_scratch": [ctypes.POINTER(_Rotate), P],
            "nopfs_gated_scan": [ctypes.POINTER(_Scan)] + [P] * 8,
            "nopfs_gated_scan_grad": [ctypes.POINTER(_Scan)] + [P] * 11,
            "nopfs_gated_scan_scratch": [ctypes.POINTER(_Scan), I32, P],
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
            "nopfs_topk_distill", "nopfs_token_embed", "nopfs_token_embed_names", "nopfs_token_embed_grad",
            "nopfs_token_embed_scratch", "nopfs_norm_rotate", "nopfs_norm_rotate_grad",
            "nopfs_norm_rotate_scratch", "nopfs_gated_scan", "nopfs_gated_scan_grad",
            "nopfs_gated_scan_scratch", "nopfs_strerror",
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


def _written(*given):
    """Tells autograd that a call has written these tensors of its caller's: a backward
    pass that has one saved as it was before is then refused instead of wrong."""
    given = [t for t in given if t is not None]
    if given:
        increment_version(given)


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


_I32, _I64, _F64 = (torch.int32,), (torch.int64,), (torch.float64,)


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
    o, given = dict(out) if out else {}, []
    for name, shape, dt in (("start", (G, n + 1), torch.int32), ("table", (G, n, width), torch.int32),
                            ("slot", (G, cap), torch.int64), ("row", (G, cap), torch.int32),
                            ("pos", (G, cap), torch.int32), ("used", (G, 3), torch.int32)):
        t = o.get(name)
        if t is None:
            o[name] = lead.new_empty(shape, dtype=dt)
        else:
            given.append(_step_dense(t, name, dt, shape, dev))
    b = _Batch(F, _row_stride(lead), _row_stride(free), G, n, free.shape[1], block, width, cap)
    st = _step_stream(stream, dev, (ids, tokens, free, *o.values()))
    scratch = _capturing() and _step_scratch(  # noqa: F841 held until the call is enqueued
        b, dev, stream, "nopfs_batch_tables_scratch")
    _check(lib().nopfs_batch_tables(
        ctypes.byref(b), None if ids is None else ids.data_ptr(), tokens.data_ptr(),
        free.data_ptr(), o["start"].data_ptr(), o["table"].data_ptr(), o["slot"].data_ptr(),
        o["row"].data_ptr(), o["pos"].data_ptr(), o["used"].data_ptr(), st), "nopfs_batch_tables")
    _written(*given)
    return o


def _no_outputs_given(name, *outputs):
    if any(t is not None for t in outputs):
        raise ValueError(f"{name}: given outputs are not part of the graph of an input that "
                         "requires a gradient (detach it, or call under torch.no_grad())")


def _no_tangents(name, *inputs):
    """Refuses inputs with forward-mode derivatives, which the kernels would drop."""
    if getattr(forward_ad, "_current_level", 0) < 0:  # none anywhere
        return
    if any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in inputs):
        raise ValueError(f"{name} has no forward-mode derivative (autograd takes its outputs back, "
                         "or call it with the primals)")


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
    _no_tangents("packed_attention", q, k, v)
    if (q.requires_grad or k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        _no_outputs_given("packed_attention", o, lse)
        return _PackedAttention.apply(q, k, v, start, scale, stream)
    dev = torch.cuda.current_device()
    given = (o, lse)
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
    _written(*given)
    return o, lse


def packed_attention_grad(do, q, k, v, o, lse, start, scale=None, dq=None, dk=None, dv=None,
                          stream=None):
    """Gradient of packed_attention (nopfs_packed_attention_grad) from its
    outputs and the gradient `do` of o. Returns dq, dk, dv (as q, k, v; slices
    of one preallocated array, say), which autograd does not differentiate again."""
    _no_tangents("packed_attention_grad", do, q, k, v, o, lse)
    dev = torch.cuda.current_device()
    given = (dq, dk, dv)
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
    _written(*given)
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
    _no_tangents("topk_distill", logits, teacher, weight)
    if teacher.requires_grad or weight is not None and weight.requires_grad:
        if torch.is_grad_enabled():
            raise ValueError("topk_distill has no gradient by teacher and weight (detach them)")
    if grad and logits.requires_grad and torch.is_grad_enabled():
        _no_outputs_given("topk_distill", loss, dlogits)
        return _TopkDistill.apply(logits, index, teacher, tau, weight, stream)
    dev = torch.cuda.current_device()
    given = (loss, dlogits if grad else None)
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
    _written(*given)
    return loss, dlogits


# -- layers of a token model over the packed samples ---------------------------------
_IDS = (torch.int32, torch.int64)


def _row_gradient(d):
    """A gradient as the kernels read it, its rows apart from each other. Autograd
    hands over broadcast and transposed ones too."""
    if d.is_contiguous():
        return d
    return d.clone(memory_format=torch.contiguous_format)


def _tokens(ids, slot, dev):
    """Entries of ids, and the tokens."""
    n_ids = _dense(_step_tensor(ids, "ids", _IDS, 1, dev), "ids").shape[0]
    return n_ids, n_ids if slot is None else _dense(_step_tensor(slot, "slot", _I64, 1, dev), "slot").shape[0]


def _float_types(dtype):
    """The types that a tensor may have where `dtype` was asked for."""
    if dtype is None:
        return _DTYPES
    if dtype not in _DTYPES:
        raise ValueError("dtype must be " + " or ".join(str(d) for d in _DTYPES))
    return (dtype,)


class _TokenEmbed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, ids, scale, slot, dtype, stream):
        # what the tokens name, not ids and slot: the token buffer and its tables go on
        # to the next batch while this one's gradient is to come
        out, names = _token_embed(weight, ids, scale, slot, dtype, None, True, stream)
        ctx.save_for_backward(names)
        ctx.rows, ctx.dtype, ctx.scale, ctx.stream = weight.shape[0], weight.dtype, scale, stream
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        names, = ctx.saved_tensors
        dout = _row_gradient(dout)
        dweight = _call_in_backward(ctx.stream, lambda: token_embed_grad(
            dout, names, ctx.rows, ctx.scale, None, ctx.dtype, stream=ctx.stream))
        return dweight, None, None, None, None, None


def token_embed(weight, ids, scale=1.0, slot=None, dtype=None, out=None, stream=None):
    """The rows of an embedding that the packed tokens name, times `scale`
    (nopfs_token_embed): weight [V][width], ids [T] int32 or int64; with slot [T]
    int64 (a row of batch_tables' slot) ids is a token buffer, and token t is
    ids[slot[t]]. Slots and ids out of range, -1 among them, are padding: rows of
    zeros. Returns [T][width] of `dtype` (weight's unless given). Autograd takes it
    back to weight by token_embed_grad, from what the tokens named in this call: ids
    and slot may change before the backward pass."""
    _no_tangents("token_embed", weight)
    if weight.requires_grad and torch.is_grad_enabled():
        _no_outputs_given("token_embed", out)
        return _TokenEmbed.apply(weight, ids, scale, slot, dtype, stream)
    return _token_embed(weight, ids, scale, slot, dtype, out, False, stream)[0]


def _token_embed(weight, ids, scale, slot, dtype, out, names, stream):
    """The rows, and if asked for what the tokens name, int32 (-1: padding)."""
    dev = torch.cuda.current_device()
    given = (out,)
    V, width = _step_tensor(weight, "weight", _DTYPES, 2, dev).shape
    n_ids, T = _tokens(ids, slot, dev)
    types = _float_types(dtype)
    if out is None:
        out = weight.new_empty((T, width), dtype=dtype)
    else:
        _step_shape(_step_tensor(out, "out", types, 2, dev), "out", (T, width))
    e = _Embed(T, V, n_ids, _row_stride(weight), _row_stride(out), width, _DTYPES[weight.dtype],
               _DTYPES[out.dtype], ids.element_size(), scale)
    names = ids.new_empty(T, dtype=torch.int32) if names else None
    st = _step_stream(stream, dev, (weight, ids, slot, out, names))
    args = (ctypes.byref(e), weight.data_ptr(), ids.data_ptr(), None if slot is None else slot.data_ptr(),
            out.data_ptr())
    if names is None:
        _check(lib().nopfs_token_embed(*args, st), "nopfs_token_embed")
    else:
        _check(lib().nopfs_token_embed_names(*args, names.data_ptr(), st), "nopfs_token_embed_names")
    _written(*given)
    return out, names


def token_embed_grad(dout, ids, rows: int, scale=1.0, slot=None, dtype=None, dweight=None,
                     stream=None):
    """Gradient of token_embed by its weight of `rows` rows (nopfs_token_embed_grad),
    from `dout` [T][width], the gradient of its output. Returns all of it,
    [rows][width] of `dtype` (dout's unless given)."""
    _no_tangents("token_embed_grad", dout)
    dev = torch.cuda.current_device()
    given = (dweight,)
    n_ids, T = _tokens(ids, slot, dev)
    width = _step_tensor(dout, "dout", _DTYPES, 2, dev).shape[1]
    _step_shape(dout, "dout", (T, width))
    rows, types = int(rows), _float_types(dtype)
    if not 0 < rows < 2**31:
        raise ValueError("rows must be positive and below 2^31")
    if dweight is None:
        dweight = dout.new_empty((rows, width), dtype=dtype)
    else:
        _step_shape(_step_tensor(dweight, "dweight", types, 2, dev), "dweight", (rows, width))
    e = _Embed(T, rows, n_ids, _row_stride(dweight), _row_stride(dout), width, _DTYPES[dweight.dtype],
               _DTYPES[dout.dtype], ids.element_size(), scale)
    st = _step_stream(stream, dev, (dout, ids, slot, dweight))
    scratch = _capturing() and _step_scratch(e, dev, stream, "nopfs_token_embed_scratch")  # noqa: F841
    _check(lib().nopfs_token_embed_grad(ctypes.byref(e), dout.data_ptr(), ids.data_ptr(),
                                        None if slot is None else slot.data_ptr(),
                                        dweight.data_ptr(), st), "nopfs_token_embed_grad")
    _written(*given)
    return dweight


def _rotate(q, k, pos, freq, q_weight, k_weight, eps, interleaved, dev):
    """What comes before the strides in the call's description."""
    _step_tensor(q, "q", _DTYPES, 3, dev)
    T, heads, width = q.shape
    kv_heads = _step_tensor(k, "k", (q.dtype,), 3, dev).shape[1]
    _step_shape(k, "k", (T, kv_heads, width))
    _step_dense(pos, "pos", torch.int32, (T,), dev)
    rotated = 0
    if freq is not None:
        rotated = 2 * _dense(_step_tensor(freq, "freq", _F64, 1, dev), "freq").shape[0]
    kind = None
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _step_shape(_step_tensor(w, name, _DTYPES, 1, dev), name, (width,))
            if kind is not None and w.dtype is not kind:
                raise ValueError("q_weight and k_weight must be of one type")
            kind = w.dtype
    return (T, heads, kv_heads, width, rotated, 1 if interleaved else 0, _DTYPES[q.dtype],
            0 if kind is None else _DTYPES[kind], eps)


def _heads_like(t, name, like, dev):
    """An output as the heads of `like`: as given, or a new one."""
    if t is None:
        return like.new_empty(like.shape)
    _step_shape(_step_tensor(t, name, (like.dtype,), 3, dev), name, like.shape)
    return t


def _optional(t):
    return None if t is None else t.data_ptr()


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, pos, freq, q_weight, k_weight, eps, interleaved, stream):
        ctx.save_for_backward(q, k, pos, freq, q_weight, k_weight)
        ctx.eps, ctx.interleaved, ctx.stream = eps, interleaved, stream
        return norm_rotate(q, k, pos, freq, q_weight, k_weight, eps, interleaved, stream=stream)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq_out, dk_out):
        need = ctx.needs_input_grad
        dq_out, dk_out = _row_gradient(dq_out), _row_gradient(dk_out)
        dq, dk, dqw, dkw = _call_in_backward(ctx.stream, lambda: norm_rotate_grad(
            dq_out, dk_out, *ctx.saved_tensors, ctx.eps, ctx.interleaved, weights=need[4] or need[5],
            stream=ctx.stream))
        return dq, dk, None, None, dqw, dkw, None, None, None


def norm_rotate(q, k, pos, freq=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                q_out=None, k_out=None, stream=None):
    """Root-mean-square norms of queries and keys per head and their rotation by
    position (nopfs_norm_rotate): q [T][heads][width], k [T][kv_heads][width], any
    strides (slices of one projection, say); pos [T] int32, a row of batch_tables'
    pos (-1: padding, rows of zeros); freq float64, the angle per position of each
    pair of elements (base ** (-2 i / rotated), say; None: no rotation; fewer than
    width / 2: the elements behind are not rotated). Pairs are (i, i + rotated/2),
    or neighbours if interleaved. q_weight, k_weight [width] of one type, or None.
    Returns q_out, k_out; they may be q and k. Autograd takes them back to q, k and
    the weights by norm_rotate_grad; freq is data."""
    _no_tangents("norm_rotate", q, k, freq, q_weight, k_weight)
    if freq is not None and freq.requires_grad and torch.is_grad_enabled():
        raise ValueError("norm_rotate has no gradient by freq (detach it)")
    if (q.requires_grad or k.requires_grad or q_weight is not None and q_weight.requires_grad
            or k_weight is not None and k_weight.requires_grad) and torch.is_grad_enabled():
        _no_outputs_given("norm_rotate", q_out, k_out)
        return _NormRotate.apply(q, k, pos, freq, q_weight, k_weight, eps, interleaved, stream)
    dev = torch.cuda.current_device()
    given = (q_out, k_out)
    r = _rotate(q, k, pos, freq, q_weight, k_weight, eps, interleaved, dev)
    q_out, k_out = _heads_like(q_out, "q_out", q, dev), _heads_like(k_out, "k_out", k, dev)
    r = _Rotate(*r, *_strides(q, k, q_out, k_out))
    st = _step_stream(stream, dev, (q, k, pos, freq, q_weight, k_weight, q_out, k_out))
    _check(lib().nopfs_norm_rotate(ctypes.byref(r), q.data_ptr(), k.data_ptr(), pos.data_ptr(),
                                   _optional(freq), _optional(q_weight), _optional(k_weight),
                                   q_out.data_ptr(), k_out.data_ptr(), st), "nopfs_norm_rotate")
    _written(*given)
    return q_out, k_out


def norm_rotate_grad(dq_out, dk_out, q, k, pos, freq=None, q_weight=None, k_weight=None, eps=1e-6,
                     interleaved=False, weights=True, dq=None, dk=None, stream=None):
    """Gradient of norm_rotate (nopfs_norm_rotate_grad) from its inputs and the
    gradients of its outputs. Returns dq, dk (given, they may be dq_out and dk_out) and
    the gradients of the weights, None of a weight that is None, or with weights False."""
    _no_tangents("norm_rotate_grad", dq_out, dk_out, q, k, freq, q_weight, k_weight)
    dev = torch.cuda.current_device()
    given = (dq, dk)
    r = _rotate(q, k, pos, freq, q_weight, k_weight, eps, interleaved, dev)
    for name, d, like in (("dq_out", dq_out, q), ("dk_out", dk_out, k)):
        _step_shape(_step_tensor(d, name, (q.dtype,), 3, dev), name, like.shape)
    dq, dk = _heads_like(dq, "dq", q, dev), _heads_like(dk, "dk", k, dev)
    dqw, dkw = (torch.empty_like(w) if weights and w is not None else None for w in (q_weight, k_weight))
    r = _Rotate(*r, *_strides(q, k, dq_out, dk_out, dq, dk))
    st = _step_stream(stream, dev, (dq_out, dk_out, q, k, pos, freq, q_weight, k_weight, dq, dk, dqw, dkw))
    scratch = _capturing() and _step_scratch(r, dev, stream, "nopfs_norm_rotate_scratch")  # noqa: F841
    _check(lib().nopfs_norm_rotate_grad(
        ctypes.byref(r), dq_out.data_ptr(), dk_out.data_ptr(), q.data_ptr(), k.data_ptr(), pos.data_ptr(),
        _optional(freq), _optional(q_weight), _optional(k_weight), dq.data_ptr(), dk.data_ptr(),
        _optional(dqw), _optional(dkw), st), "nopfs_norm_rotate_grad")
    _written(*given)
    return dq, dk, dqw, dkw


SCAN_CHUNK = 16  # NOPFS_SCAN_CHUNK


def _scan(x, gate, start, h0, dev):
    T, channels = _step_tensor(x, "x", _DTYPES, 2, dev).shape
    _step_shape(_step_tensor(gate, "gate", (x.dtype,), 2, dev), "gate", (T, channels))
    n = _dense(_step_tensor(start, "start", _I32, 1, dev), "start").shape[0] - 1
    if n < 0:
        raise ValueError("start must have an entry before every sample and one behind the last")
    if h0 is not None:
        _step_dense(h0, "h0", torch.float32, (n, channels), dev)
    return T, n, channels, -(-T // SCAN_CHUNK)


def _rows_of(t, name, dtype, shape, like, dev):
    """An output's rows: as given, or new ones."""
    if t is None:
        return like.new_empty(shape, dtype=dtype)
    _step_shape(_step_tensor(t, name, (dtype,), 2, dev), name, shape)
    return t


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, start, h0, stream):
        h, last, carry = gated_scan(x, gate, start, h0, stream=stream)
        ctx.save_for_backward(x, gate, start, h0, carry)
        ctx.stream = stream
        ctx.mark_non_differentiable(carry)
        ctx.set_materialize_grads(False)
        return h, last, carry

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dlast, _):
        if dh is None and dlast is None:
            return (None,) * 5
        x, gate, start, h0, carry = ctx.saved_tensors
        dh = torch.zeros_like(x, memory_format=torch.contiguous_format) if dh is None else _row_gradient(dh)
        dlast = None if dlast is None else dlast.contiguous()
        dx, dgate, dh0 = _call_in_backward(ctx.stream, lambda: gated_scan_grad(
            dh, x, gate, start, carry, h0, dlast, stream=ctx.stream))
        return dx, dgate, None, dh0, None


def gated_scan(x, gate, start, h0=None, keep=True, h=None, last=None, stream=None):
    """A gated linear recurrence over packed samples (nopfs_gated_scan), for each
    channel by itself: with a = sigmoid(gate), h_t = a_t h_(t-1) + (1 - a_t) x_t.
    x and gate [T][channels], any row strides (halves of one projection, say);
    start [n+1] int32, a row of batch_tables' start; h0 [n][channels] float32, the
    state before each sample (0 if None). Returns h (as x), last [n][channels]
    float32, the state behind each sample, and carry, which the gradient starts from
    (None if keep is False). Samples of one token with h0 are the step of a
    generation; last may not be h0. Autograd takes h and last back to x, gate and h0
    by gated_scan_grad."""
    _no_tangents("gated_scan", x, gate, h0)
    if (x.requires_grad or gate.requires_grad
            or h0 is not None and h0.requires_grad) and torch.is_grad_enabled():
        _no_outputs_given("gated_scan", h, last)
        h, last, carry = _GatedScan.apply(x, gate, start, h0, stream)
        return h, last, carry if keep else None
    dev = torch.cuda.current_device()
    given = (h, last)
    T, n, channels, chunks = _scan(x, gate, start, h0, dev)
    h = _rows_of(h, "h", x.dtype, (T, channels), x, dev)
    if last is None:
        last = x.new_empty((n, channels), dtype=torch.float32)
    else:
        _step_dense(last, "last", torch.float32, (n, channels), dev)
    carry = x.new_empty((chunks, channels), dtype=torch.float32) if keep else None
    s = _Scan(T, n, channels, _DTYPES[x.dtype], 0, _row_stride(x), _row_stride(gate), _row_stride(h))
    st = _step_stream(stream, dev, (x, gate, start, h0, h, last, carry))
    scratch = _capturing() and _step_scratch(s, dev, stream, "nopfs_gated_scan_scratch", 0)  # noqa: F841
    _check(lib().nopfs_gated_scan(ctypes.byref(s), x.data_ptr(), gate.data_ptr(), start.data_ptr(),
                                  _optional(h0), h.data_ptr(), last.data_ptr(), _optional(carry), st),
           "nopfs_gated_scan")
    _written(*given)
    return h, last, carry


def gated_scan_grad(dh, x, gate, start, carry, h0=None, dlast=None, dx=None, dgate=None, stream=None):
    """Gradient of gated_scan (nopfs_gated_scan_grad) from its inputs, its carry and
    the gradients of h and last (None: 0). Returns dx, dgate (as x) and dh0 (None
    without h0)."""
    _no_tangents("gated_scan_grad", dh, x, gate, carry, h0, dlast)
    dev = torch.cuda.current_device()
    given = (dx, dgate)
    T, n, channels, chunks = _scan(x, gate, start, h0, dev)
    _step_shape(_step_tensor(dh, "dh", (x.dtype,), 2, dev), "dh", (T, channels))
    _step_dense(carry, "carry", torch.float32, (chunks, channels), dev)
    if dlast is not None:
        _step_dense(dlast, "dlast", torch.float32, (n, channels), dev)
    dx = _rows_of(dx, "dx", x.dtype, (T, channels), x, dev)
    dgate = _rows_of(dgate, "dgate", x.dtype, (T, channels), x, dev)
    dh0 = None if h0 is None else torch.empty_like(h0)
    s = _Scan(T, n, channels, _DTYPES[x.dtype], 0, _row_stride(x), _row_stride(gate), 0,
              _row_stride(dh), _row_stride(dx), _row_stride(dgate))
    st = _step_stream(stream, dev, (dh, x, gate, start, carry, h0, dlast, dx, dgate, dh0))
    scratch = _capturing() and _step_scratch(s, dev, stream, "nopfs_gated_scan_scratch", 1)  # noqa: F841
    _check(lib().nopfs_gated_scan_grad(
        ctypes.byref(s), dh.data_ptr(), _optional(dlast), x.data_ptr(), gate.data_ptr(), start.data_ptr(),
        _optional(h0), carry.data_ptr(), dx.data_ptr(), dgate.data_ptr(), _optional(dh0), st),
        "nopfs_gated_scan_grad")
    _written(*given)
    return dx, dgate, dh0


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
