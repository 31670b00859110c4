"""Outputs that a caller gives count as written: a backward pass that saved what stood
there is refused, not wrong."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2101_08734_amd import nopfs  # noqa: E402

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _tables(lengths, out=None):
    lengths = torch.tensor([lengths], dtype=torch.int32, device="cuda")
    free = torch.arange(12, dtype=torch.int32, device="cuda")[None]
    return nopfs.batch_tables(None, lengths, free, 16, 4, 100, out=out)


@pytest.mark.parametrize("call", ["rotate", "scan", "attention"])
def test_tables_that_a_backward_pass_needs(call):
    tables = _tables([37, 1, 0, 30])
    start, pos = tables["start"][0], tables["pos"][0]
    q = torch.randn((100, 2, 16), device="cuda").to(BF).requires_grad_()
    if call == "rotate":
        freq = 10.0 ** (-torch.arange(8, dtype=torch.float64, device="cuda"))
        f = lambda: nopfs.norm_rotate(q, q, pos, freq)[0]  # noqa: E731
    elif call == "scan":
        f = lambda: nopfs.gated_scan(q.view(100, 32), q.view(100, 32), start)[0]  # noqa: E731
    else:
        f = lambda: nopfs.packed_attention(q, q, q, start)[0]  # noqa: E731
    out = f()
    out.float().sum().backward()  # before the next tables: as ever
    out = f()
    _tables([30, 2, 5, 9], out=tables)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.float().sum().backward()
    f().float().sum().backward()


def _outputs():
    start = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    ids = torch.arange(6, device="cuda")
    q, a, b = (torch.randn((6, 2, 8), device="cuda").to(BF) for _ in range(3))
    x, y, z = (torch.randn((6, 8), device="cuda") for _ in range(3))
    s = torch.zeros((1, 8), device="cuda")
    carry = nopfs.gated_scan(x, y, start)[2]
    o, lse = nopfs.packed_attention(q, q, q, start)
    index = torch.zeros((6, 1), dtype=torch.int32, device="cuda")
    yield "embed", lambda: nopfs.token_embed(x, ids, out=y), (y,)
    yield "embed_grad", lambda: nopfs.token_embed_grad(x, ids, 6, dweight=y), (y,)
    yield "rotate", lambda: nopfs.norm_rotate(q, a, pos, q_out=q, k_out=a), (q, a)
    yield "rotate_grad", lambda: nopfs.norm_rotate_grad(q, q, q, q, pos, dq=a, dk=b), (a, b)
    yield "scan", lambda: nopfs.gated_scan(x, y, start, h=z, last=s), (z, s)
    yield "scan_grad", lambda: nopfs.gated_scan_grad(x, x, x, start, carry, dx=y, dgate=z), (y, z)
    yield "attention", lambda: nopfs.packed_attention(q, q, q, start, o=a, lse=lse), (a, lse)
    yield "attention_grad", lambda: nopfs.packed_attention_grad(o, q, q, q, o, lse, start, dq=a, dk=b), (a, b)
    yield "distill", lambda: nopfs.topk_distill(x, index, y[:, :1], dlogits=x), (x,)


def test_every_given_output():
    for name, call, given in _outputs():
        before = [t._version for t in given]
        call()
        assert all(t._version > v for t, v in zip(given, before)), name
    t = _tables([3])
    before = {k: v._version for k, v in t.items()}
    _tables([4], out=dict(pos=t["pos"]))
    assert t["pos"]._version > before["pos"] and t["slot"]._version == before["slot"]
    with torch.inference_mode():
        for name, call, given in _outputs():
            call()
