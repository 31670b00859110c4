"""The gradient of token_embed is that of the tokens that the forward call looked up,
whatever becomes of the token buffer and its tables before the backward pass."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import ctypes  # noqa: E402

import layer_ref  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


@pytest.mark.parametrize("T", [1, 5, 700, 5_003, 300_000])
@pytest.mark.parametrize("width,wide,slots", [(1, False, False), (7, True, True), (8, True, False), (250, False, True),
                                              (2_100, True, True)])
def test_names(T, width, wide, slots):
    """Of every token, to the last, and the rows as without them."""
    if T * width > 2**27:
        T = 5_003
    g = torch.Generator().manual_seed(T + width)
    V, n = 90, 777 if slots else T
    ids = torch.randint(-3, V + 3, (n,), generator=g).to(torch.int64 if wide else torch.int32)
    slot = torch.randint(-5, n + 5, (T,), generator=g) if slots else None
    weight = torch.randn((V, width), generator=g).cuda()
    args = (weight, ids.cuda(), 0.5, None if slot is None else slot.cuda())
    held = torch.full((T + 64,), 77, dtype=torch.int32, device="cuda")
    out = torch.full((T, width), 9.0, dtype=BF, device="cuda")
    e = nopfs._Embed(T, V, n, width, width, width, nopfs._DTYPES[F32], nopfs._DTYPES[BF], 8 if wide else 4, 0.5)
    assert nopfs.lib().nopfs_token_embed_names(
        ctypes.byref(e), weight.data_ptr(), args[1].data_ptr(), args[3].data_ptr() if slots else None,
        out.data_ptr(), held.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert held[:T].tolist() == layer_ref.names(ids, slot, V) and bool((held[T:] == 77).all())
    assert torch.equal(out, nopfs.token_embed(*args, dtype=BF))


@pytest.mark.parametrize("seen", [True, False])
@pytest.mark.parametrize("slots", [True, False])
def test_buffer_and_tables_go_on(seen, slots):
    """Written by torch, and by calls that autograd does not see."""
    g = torch.Generator().manual_seed(1)
    w = torch.randn((60, 24), generator=g).cuda()
    ids = torch.randint(-1, 60, (200,), generator=g).cuda()
    slot = torch.randint(-1, 200, (150,), generator=g).cuda() if slots else None
    T = 150 if slots else 200
    d = torch.randn((T, 24), generator=g).to(BF).cuda()
    want = nopfs.token_embed_grad(d, ids, 60, 0.7, slot=slot, dtype=F32)
    w.requires_grad_()
    out = nopfs.token_embed(w, ids, 0.7, slot=slot, dtype=BF)
    for t in (ids, slot):
        if t is not None:
            (t if seen else t.data).fill_(3)
    out.backward(d)
    assert torch.equal(w.grad, want)


def test_tables_of_the_next_batch_in_place():
    """A worker lays out its next batch, and reads it into the buffer, between the two."""
    lengths = torch.tensor([[37, 1, 0, 30]], dtype=torch.int32, device="cuda")
    free = torch.arange(12, dtype=torch.int32, device="cuda")[None]
    tables = nopfs.batch_tables(None, lengths, free, 16, 4, 100)
    buffer = (torch.arange(12 * 16, device="cuda") * 7) % 50
    w = torch.randn((50, 16), device="cuda", requires_grad=True)
    d = torch.randn((100, 16), device="cuda")
    slot = tables["slot"][0]
    want = nopfs.token_embed_grad(d, buffer, 50, slot=slot)
    out = nopfs.token_embed(w, buffer, slot=slot)
    nopfs.batch_tables(None, lengths.flip(1).contiguous(), free.flip(1).contiguous(), 16, 4, 100, out=tables)
    buffer[:64] = 0
    out.backward(d)
    assert torch.equal(w.grad, want)
