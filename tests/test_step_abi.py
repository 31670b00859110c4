"""What the operators of a training step refuse, on the host (no GPU): every
call below returns an error, or has nothing to do, before anything is enqueued.
Pointers are never dereferenced."""
import ctypes

import pytest

nopfs = pytest.importorskip("paper_2101_08734_amd.nopfs")
torch = pytest.importorskip("torch")

P = ctypes.c_void_p(0x1000)  # 16-byte aligned
ODD = ctypes.c_void_p(0x1008)
EINVAL, ERANGE, ENOMEM = nopfs.NOPFS_EINVAL, nopfs.NOPFS_ERANGE, nopfs.NOPFS_ENOMEM


@pytest.fixture(scope="module")
def L():
    return nopfs.lib()


def _batch(**kw):
    d = dict(F=100, ids_stride=8, free_stride=20, G=2, n=8, blocks=20, block=16, width=4, cap=64)
    d.update(kw)
    return nopfs._Batch(**d)


BATCH_ARGS = ("ids", "tokens", "free", "start", "table", "slot", "row", "pos", "used")


def _tables(L, b, **kw):
    args = [kw.get(x, P) for x in BATCH_ARGS]
    return L.nopfs_batch_tables(None if b is None else ctypes.byref(b), *args, None)


@pytest.mark.parametrize("kw,code", [
    (dict(G=0), EINVAL), (dict(n=0), EINVAL), (dict(block=0), EINVAL), (dict(width=0), EINVAL),
    (dict(blocks=-1), EINVAL), (dict(cap=-1), EINVAL), (dict(F=0), EINVAL),
    (dict(ids_stride=7), EINVAL), (dict(free_stride=19), EINVAL), (dict(cap=2**30 + 1), ERANGE),
    (dict(n=2**30 + 1, ids_stride=2**31), ERANGE),
    (dict(n=2**30, ids_stride=2**30, width=2**20), ERANGE)])
def test_batch_refusals(L, kw, code):
    assert _tables(L, _batch(**kw)) == code
    assert L.nopfs_last_error()


@pytest.mark.parametrize("kw", [dict(G=2**22), dict(G=2**20, cap=2**20)])
def test_batch_launch_limits(L, kw):
    """A launch has fewer than 2^32 threads."""
    assert _tables(L, _batch(**kw)) == ERANGE


def test_batch_null_pointers(L):
    assert _tables(L, None) == EINVAL
    for name in BATCH_ARGS[1:]:
        assert _tables(L, _batch(), **{name: None}) == EINVAL, name


def _attention(**kw):
    d = dict(T=100, n=3, heads=4, kv_heads=2, width=64, dtype=nopfs._DTYPES[torch.bfloat16],
             scale=0.125)
    for x in ("q", "k", "v", "o", "do", "dq", "dk", "dv"):
        d[x + "_token"], d[x + "_head"] = 4 * 64, 64
    d.update(kw)
    return nopfs._Attention(**d)


FORWARD = ("q", "k", "v", "start", "o", "lse")
GRAD = ("do", "q", "k", "v", "o", "lse", "start", "dq", "dk", "dv")


def _forward(L, a, **kw):
    return L.nopfs_packed_attention(None if a is None else ctypes.byref(a),
                                    *[kw.get(x, P) for x in FORWARD], None)


def _grad(L, a, **kw):
    return L.nopfs_packed_attention_grad(None if a is None else ctypes.byref(a),
                                         *[kw.get(x, P) for x in GRAD], None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(n=-1), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=0), EINVAL),
    (dict(heads=5), EINVAL), (dict(width=0), EINVAL), (dict(width=60), EINVAL),
    (dict(width=136, q_head=136), ERANGE), (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL),
    (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(T=2**31), ERANGE), (dict(n=2**30 + 1), ERANGE),
    (dict(n=2**29, heads=64), ERANGE),
    (dict(q_token=260), EINVAL), (dict(k_head=68), EINVAL), (dict(v_token=0), EINVAL),
    (dict(k_head=0), EINVAL), (dict(o_token=-256), EINVAL), (dict(q_token=2**41), ERANGE)])
def test_attention_refusals(L, kw, code):
    assert _forward(L, _attention(**kw)) == code
    assert L.nopfs_last_error()
    assert _grad(L, _attention(**kw)) == code


@pytest.mark.parametrize("name", ["do", "dq", "dk", "dv"])
def test_attention_gradient_strides(L, name):
    assert _grad(L, _attention(**{name + "_token": 63 * 4})) == EINVAL
    assert _grad(L, _attention(**{name + "_head": 8})) == EINVAL


def test_attention_null_and_unaligned(L):
    assert _forward(L, None) == EINVAL and _grad(L, None) == EINVAL
    for name in FORWARD:
        assert _forward(L, _attention(), **{name: None}) == EINVAL, name
    for name in GRAD:
        assert _grad(L, _attention(), **{name: None}) == EINVAL, name
    for name in ("q", "k", "v", "o"):
        assert _forward(L, _attention(), **{name: ODD}) == EINVAL, name
    for name in ("do", "q", "dq", "dk", "dv"):
        assert _grad(L, _attention(), **{name: ODD}) == EINVAL, name
    # no row: nothing is touched
    assert _forward(L, _attention(T=0), **{x: None for x in FORWARD}) == 0
    assert _grad(L, _attention(T=0), **{x: None for x in GRAD}) == 0


def _distill(**kw):
    d = dict(T=10, V=100, logits_stride=100, grad_stride=100, index_stride=5, teacher_stride=5, K=5,
             dtype=0, teacher_dtype=1, tau=1.0)
    d.update(kw)
    return nopfs._Distill(**d)


LOSS = ("logits", "index", "teacher", "weight", "loss", "grad")


def _loss(L, d, **kw):
    return L.nopfs_topk_distill(None if d is None else ctypes.byref(d),
                                *[kw.get(x, P) for x in LOSS], None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(V=0), EINVAL), (dict(K=0), EINVAL), (dict(dtype=3), EINVAL),
    (dict(dtype=-1), EINVAL), (dict(teacher_dtype=3), EINVAL), (dict(tau=0.0), EINVAL),
    (dict(tau=-1.0), EINVAL), (dict(tau=float("nan")), EINVAL), (dict(tau=float("inf")), EINVAL),
    (dict(logits_stride=99), EINVAL), (dict(grad_stride=99), EINVAL), (dict(index_stride=4), EINVAL),
    (dict(teacher_stride=4), EINVAL), (dict(K=1_025, index_stride=1_025, teacher_stride=1_025), ERANGE),
    (dict(T=2**31), ERANGE), (dict(V=2**31, logits_stride=2**31, grad_stride=2**31), ERANGE)])
def test_distill_refusals(L, kw, code):
    assert _loss(L, _distill(**kw)) == code
    assert L.nopfs_last_error()


def test_distill_null_pointers(L):
    assert _loss(L, None) == EINVAL
    for name in ("logits", "index", "teacher", "loss"):
        assert _loss(L, _distill(), **{name: None}) == EINVAL, name
    assert _loss(L, _distill(T=0), **{x: None for x in LOSS}) == 0


def test_no_memory_for_scratch(L):
    for call in (lambda: _tables(L, _batch(n=5_000, ids_stride=5_000)), lambda: _grad(L, _attention())):
        assert L.nopfs_debug_set(3, 1) == 0
        assert call() == ENOMEM
        assert b"scratch" in L.nopfs_last_error()
    assert L.nopfs_debug_set(3, 0) == 0


def test_host_tensors_are_refused():
    """The binding takes device tensors only (without a GPU even the question
    for the current device fails)."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU to ask for")
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    start = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        nopfs.packed_attention(q, q, q, start)
    with pytest.raises(TypeError):
        nopfs.batch_tables(None, start[None], start[None], 4, 4, 4)
    with pytest.raises(TypeError):
        nopfs.topk_distill(q[0], start[None], q[0], 1.0)


@pytest.mark.parametrize("x", [2.0**-61, 2.0**61, 1e-40])
def test_scales_and_temperatures_out_of_range(L, x):
    assert _forward(L, _attention(scale=x)) == ERANGE and _grad(L, _attention(scale=x)) == ERANGE
    assert _loss(L, _distill(tau=x)) == ERANGE


def _size(L, call, *args):
    need = ctypes.c_int64(-1)
    rc = call(*args, ctypes.byref(need))
    return rc, need.value


def test_scratch_sizes(L):
    """On the host, from the description alone; what the refused calls refuse."""
    batch = lambda **kw: _size(L, L.nopfs_batch_tables_scratch, ctypes.byref(_batch(**kw)))  # noqa: E731
    assert batch() == (0, 0)  # one launch makes its sums itself
    rc, need = batch(n=5_000, ids_stride=5_000)
    assert rc == 0 and need >= 2 * 5_001 * 4
    assert batch(n=0) == (EINVAL, 0) and L.nopfs_batch_tables_scratch(ctypes.byref(_batch()), None) == EINVAL

    def attention(gradient, **kw):
        return _size(L, L.nopfs_packed_attention_scratch, ctypes.byref(_attention(**kw)), gradient)

    assert attention(0) == (0, 0)
    rc, need = attention(1)
    assert rc == 0 and need >= 4 * 100 * 4
    one = dict(T=6_000, n=1)  # parts of the keys: 32-bit sums and a row's statistics
    assert attention(0, **one)[1] >= 6_000 * 4 * (64 * 4 + 8) * 2
    assert attention(1, **one)[1] >= 6_000 * 4 * 64 * 4 * 2
    assert attention(0, T=0) == (0, 0) and attention(1, T=0) == (0, 0)
    assert attention(1, width=60) == (EINVAL, 0) and attention(0, T=2**31) == (ERANGE, 0)


def test_scratch_refusals(L):
    """Too little of it, or in the wrong place, before anything is enqueued."""
    one = dict(T=6_000, n=1)
    for call, kw, make, size in (
            (_tables, dict(n=5_000, ids_stride=5_000), _batch,
             lambda d: _size(L, L.nopfs_batch_tables_scratch, ctypes.byref(d))),
            (_forward, one, _attention,
             lambda d: _size(L, L.nopfs_packed_attention_scratch, ctypes.byref(d), 0)),
            (_grad, one, _attention,
             lambda d: _size(L, L.nopfs_packed_attention_scratch, ctypes.byref(d), 1))):
        need = size(make(**kw))[1]
        assert call(L, make(**kw, scratch=0x1010, scratch_bytes=need)) == EINVAL
        assert call(L, make(**kw, scratch=0x1000, scratch_bytes=-1)) == EINVAL
        assert call(L, make(**kw, scratch=0x1000, scratch_bytes=need - 1)) == ENOMEM
        assert b"scratch" in L.nopfs_last_error()
