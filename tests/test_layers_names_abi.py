"""What nopfs_token_embed_names refuses, on the host (no GPU)."""
import ctypes

import pytest

nopfs = pytest.importorskip("paper_2101_08734_amd.nopfs")
torch = pytest.importorskip("torch")

P = ctypes.c_void_p(0x1000)
F32 = nopfs._DTYPES[torch.float32]


def _call(names=P, e=True, weight=P, ids=P, out=P, **kw):
    d = dict(T=100, V=50, n_ids=100, weight_stride=64, out_stride=64, width=64, weight_dtype=F32, dtype=F32,
             id_bytes=4, scale=1.0)
    d.update(kw)
    e = ctypes.byref(nopfs._Embed(**d)) if e else None
    return nopfs.lib().nopfs_token_embed_names(e, weight, ids, None, out, names, None)


def test_refusals():
    for kw in (dict(names=None), dict(weight=None), dict(ids=None), dict(out=None), dict(e=False), dict(T=-1),
               dict(n_ids=99), dict(width=0), dict(out_stride=63), dict(id_bytes=2), dict(scale=float("inf"))):
        assert _call(**kw) == nopfs.NOPFS_EINVAL, kw
        assert nopfs.lib().nopfs_last_error()
    assert _call(V=2**31 - 1) == nopfs.NOPFS_ERANGE
    assert _call(T=0, n_ids=0, names=None, weight=None, ids=None, out=None) == 0
