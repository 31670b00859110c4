"""What the layers of a token model refuse, on the host (no GPU): every call below
returns an error, or has nothing to do, before anything is enqueued. Pointers are
never dereferenced."""
import ctypes

import pytest

nopfs = pytest.importorskip("paper_2101_08734_amd.nopfs")
torch = pytest.importorskip("torch")

P = ctypes.c_void_p(0x1000)
EINVAL, ERANGE, ENOMEM = nopfs.NOPFS_EINVAL, nopfs.NOPFS_ERANGE, nopfs.NOPFS_ENOMEM
BF, FP, F32 = (nopfs._DTYPES[t] for t in (torch.bfloat16, torch.float16, torch.float32))


@pytest.fixture(scope="module")
def L():
    return nopfs.lib()


def _call(fn, desc, names, kw):
    return fn(None if desc is None else ctypes.byref(desc), *[kw.get(x, P) for x in names], None)


def _embed(**kw):
    d = dict(T=100, V=50, n_ids=100, weight_stride=64, out_stride=64, width=64, weight_dtype=F32, dtype=BF,
             id_bytes=4, scale=1.0)
    d.update(kw)
    return nopfs._Embed(**d)


LOOK = ("weight", "ids", "slot", "out")
LOOK_GRAD = ("dout", "ids", "slot", "dweight")


def _look(L, d, **kw):
    return _call(L.nopfs_token_embed, d, LOOK, dict(slot=None, **kw))


def _look_grad(L, d, **kw):
    return _call(L.nopfs_token_embed_grad, d, LOOK_GRAD, dict(slot=None, **kw))


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(V=0), EINVAL), (dict(width=0), EINVAL), (dict(n_ids=-1), EINVAL),
    (dict(n_ids=99), EINVAL), (dict(weight_dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(id_bytes=2), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(weight_stride=63), EINVAL),
    (dict(out_stride=63), EINVAL), (dict(T=2**31, n_ids=2**31), ERANGE), (dict(V=2**31 - 1), ERANGE),
    (dict(out_stride=2**28 + 1), ERANGE), (dict(weight_stride=2**28 + 1), ERANGE)])
def test_embed_refusals(L, kw, code):
    assert _look(L, _embed(**kw)) == code
    assert L.nopfs_last_error()
    assert _look_grad(L, _embed(**kw)) == code


def test_embed_null_pointers(L):
    assert _look(L, None) == EINVAL and _look_grad(L, None) == EINVAL
    for name in ("weight", "ids", "out"):
        assert _look(L, _embed(), **{name: None}) == EINVAL, name
    for name in ("dout", "ids", "dweight"):
        assert _look_grad(L, _embed(), **{name: None}) == EINVAL, name
    assert _look(L, _embed(T=0, n_ids=0), weight=None, ids=None, out=None) == 0


def _rotate(**kw):
    d = dict(T=100, heads=4, kv_heads=2, width=64, rotated=64, interleaved=0, dtype=BF, weight_dtype=F32, eps=1e-6)
    for x, heads in (("q", 4), ("k", 2), ("q_out", 4), ("k_out", 2), ("dq", 4), ("dk", 2)):
        d[x + "_token"], d[x + "_head"] = heads * 64, 64
    d.update(kw)
    return nopfs._Rotate(**d)


TURN = ("q", "k", "pos", "freq", "q_weight", "k_weight", "q_out", "k_out")
TURN_GRAD = ("dq_out", "dk_out", "q", "k", "pos", "freq", "q_weight", "k_weight", "dq", "dk", "dqw", "dkw")


def _turn(L, d, **kw):
    return _call(L.nopfs_norm_rotate, d, TURN, kw)


def _turn_grad(L, d, **kw):
    return _call(L.nopfs_norm_rotate_grad, d, TURN_GRAD, kw)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(heads=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(width=0), EINVAL),
    (dict(width=60, rotated=56), EINVAL), (dict(rotated=72), EINVAL), (dict(rotated=4), EINVAL),
    (dict(rotated=-8), EINVAL), (dict(interleaved=2), EINVAL), (dict(dtype=3), EINVAL), (dict(weight_dtype=-1), EINVAL),
    (dict(eps=0.0), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(eps=float("inf")), EINVAL), (dict(eps=2.0**-61), ERANGE), (dict(eps=2.0**61), ERANGE),
    (dict(width=264, rotated=64, q_head=264, q_token=2_000), ERANGE), (dict(T=2**31), ERANGE),
    (dict(heads=2**16 + 1, q_token=2**24), ERANGE), (dict(q_token=255), EINVAL), (dict(k_head=63), EINVAL),
    (dict(q_out_token=0), EINVAL), (dict(k_out_head=-64), EINVAL), (dict(q_token=2**30 + 1), ERANGE)])
def test_rotate_refusals(L, kw, code):
    assert _turn(L, _rotate(**kw)) == code
    assert L.nopfs_last_error()
    assert _turn_grad(L, _rotate(**kw)) == code


def test_rotate_gradient_strides(L):
    assert _turn_grad(L, _rotate(dq_token=255)) == EINVAL and _turn_grad(L, _rotate(dk_head=8)) == EINVAL


def test_rotate_null_pointers(L):
    assert _turn(L, None) == EINVAL and _turn_grad(L, None) == EINVAL
    for name in set(TURN) - {"q_weight", "k_weight"}:
        assert _turn(L, _rotate(), **{name: None}) == EINVAL, name
    for name in set(TURN_GRAD) - {"q_weight", "k_weight", "dqw", "dkw"}:
        assert _turn_grad(L, _rotate(), **{name: None}) == EINVAL, name
    assert _turn(L, _rotate(T=0), **{x: None for x in TURN}) == 0
    assert _turn_grad(L, _rotate(T=0), **{x: None for x in TURN_GRAD}) == 0


def _scan(**kw):
    d = dict(T=1_000, n=3, channels=64, dtype=BF)
    for x in ("x", "gate", "h", "dh", "dx", "dgate"):
        d[x + "_stride"] = 64
    d.update(kw)
    return nopfs._Scan(**d)


SCAN = ("x", "gate", "start", "h0", "h", "last", "carry")
SCAN_GRAD = ("dh", "dlast", "x", "gate", "start", "h0", "carry", "dx", "dgate", "dh0")
OTHER = ctypes.c_void_p(0x2000)


def _scanned(L, d, **kw):
    return _call(L.nopfs_gated_scan, d, SCAN, dict(dict(last=OTHER), **kw))


def _scan_grad(L, d, **kw):
    return _call(L.nopfs_gated_scan_grad, d, SCAN_GRAD, dict(dict(dh0=OTHER), **kw))


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), EINVAL), (dict(n=-1), EINVAL), (dict(channels=0), EINVAL), (dict(dtype=3), EINVAL),
    (dict(T=2**31), ERANGE), (dict(n=2**30 + 1), ERANGE), (dict(x_stride=63), EINVAL), (dict(gate_stride=0), EINVAL),
    (dict(x_stride=2**30 + 1), ERANGE), (dict(T=2**31 - 1, channels=2**20, x_stride=2**20, gate_stride=2**20,
                                              h_stride=2**20, dh_stride=2**20, dx_stride=2**20,
                                              dgate_stride=2**20), ERANGE)])
def test_scan_refusals(L, kw, code):
    assert _scanned(L, _scan(**kw)) == code
    assert L.nopfs_last_error()
    assert _scan_grad(L, _scan(**kw)) == code


def test_scan_strides_and_null_pointers(L):
    assert _scanned(L, _scan(h_stride=8)) == EINVAL
    for name in ("dh", "dx", "dgate"):
        assert _scan_grad(L, _scan(**{name + "_stride": 63})) == EINVAL
    assert _scanned(L, None) == EINVAL and _scan_grad(L, None) == EINVAL
    for name in ("x", "gate", "start", "h"):
        assert _scanned(L, _scan(), **{name: None}) == EINVAL, name
    for name in ("dh", "x", "gate", "start", "carry", "dx", "dgate"):
        assert _scan_grad(L, _scan(), **{name: None}) == EINVAL, name
    assert _scanned(L, _scan(), last=P) == EINVAL  # h0
    assert _scan_grad(L, _scan(), dh0=P) == EINVAL  # dlast


def _size(call, *args):
    need = ctypes.c_int64(-1)
    rc = call(*args, ctypes.byref(need))
    return rc, need.value


def _sizes(L):
    return ((_look_grad, _embed, lambda d: _size(L.nopfs_token_embed_scratch, ctypes.byref(d))),
            (_turn_grad, _rotate, lambda d: _size(L.nopfs_norm_rotate_scratch, ctypes.byref(d))),
            (_scanned, _scan, lambda d: _size(L.nopfs_gated_scan_scratch, ctypes.byref(d), 0)),
            (_scan_grad, _scan, lambda d: _size(L.nopfs_gated_scan_scratch, ctypes.byref(d), 1)))


def test_scratch_sizes(L):
    """On the host, from the description alone; what the refused calls refuse."""
    for _, make, size in _sizes(L):
        rc, need = size(make())
        assert rc == 0 and 0 < need < 2**24
        assert size(make(T=-1)) == (EINVAL, 0)
        assert size(make(T=2**31, **(dict(n_ids=2**31) if make is _embed else {}))) == (ERANGE, 0)
    assert _size(L.nopfs_gated_scan_scratch, ctypes.byref(_scan(T=16)), 0) == (0, 0)  # one stretch
    assert L.nopfs_token_embed_scratch(ctypes.byref(_embed()), None) == EINVAL


def test_scratch_refusals(L):
    """Too little of it, or in the wrong place, before anything is enqueued."""
    for call, make, size in _sizes(L):
        need = size(make())[1]
        assert call(L, make(scratch=0x1010, scratch_bytes=need)) == EINVAL
        assert call(L, make(scratch=0x1000, scratch_bytes=-1)) == EINVAL
        assert call(L, make(scratch=0x1000, scratch_bytes=need - 1)) == ENOMEM
        assert b"scratch" in L.nopfs_last_error()


def test_no_memory_for_scratch(L):
    for call, make, _ in _sizes(L):
        assert L.nopfs_debug_set(3, 1) == 0
        assert call(L, make()) == ENOMEM
        assert b"scratch" in L.nopfs_last_error()
    assert L.nopfs_debug_set(3, 0) == 0
