"""The operators of a training step under autograd: outputs are in the graph of
inputs that require gradients, with the gradients of the calls that make them,
and what cannot be differentiated is refused."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _qkv(dtype=BF):
    g = torch.Generator().manual_seed(1)
    x = torch.randn((150, 8, 64), generator=g).to(dtype).cuda()
    start = torch.tensor([0, 70, 71, 140], dtype=torch.int32, device="cuda")
    return x, start


def _heads(x):
    return x[:, :4], x[:, 4:6], x[:, 6:]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("scale", [None, 0.3])
def test_attention(dtype, scale):
    x, start = _qkv(dtype)
    want_o, want_lse = nopfs.packed_attention(*_heads(x), start, scale)
    w = torch.randn_like(want_o)
    want = nopfs.packed_attention_grad(w, *_heads(x), want_o, want_lse, start, scale)
    x.requires_grad_()
    o, lse = nopfs.packed_attention(*_heads(x), start, scale)
    assert torch.equal(o, want_o) and torch.equal(lse, want_lse)
    (o * w).sum().backward()
    for a, b in zip(_heads(x.grad), want):
        assert torch.equal(a, b)
    # a gradient that is broadcast, one that is transposed, one of odd strides
    for do in (torch.ones((), dtype=dtype, device="cuda").expand(o.shape),
               torch.randn((4, 150, 64), device="cuda").to(dtype).transpose(0, 1),
               torch.randn((150, 4, 67), device="cuda").to(dtype)[:, :, 1:65],
               torch.randn((150, 4, 128), device="cuda").to(dtype)[:, :, ::2]):
        x.grad = None
        o, _ = nopfs.packed_attention(*_heads(x), start, scale)
        o.backward(do)
        want = nopfs.packed_attention_grad(do.contiguous(), *_heads(x), want_o, want_lse, start, scale)
        for a, b in zip(_heads(x.grad), want):
            assert torch.equal(a, b)


def test_attention_of_one_input():
    """Only k requires a gradient."""
    x, start = _qkv()
    q, k, v = (t.contiguous() for t in _heads(x))
    o, lse = nopfs.packed_attention(q, k, v, start)
    want = nopfs.packed_attention_grad(torch.ones_like(o), q, k, v, o, lse, start)[1]
    k.requires_grad_()
    nopfs.packed_attention(q, k, v, start)[0].sum().backward()
    assert torch.equal(k.grad, want) and q.grad is None


def test_on_another_stream():
    x, start = _qkv()
    o, lse = nopfs.packed_attention(*_heads(x), start)
    want = nopfs.packed_attention_grad(torch.ones_like(o), *_heads(x), o, lse, start)
    x.requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, _ = nopfs.packed_attention(*_heads(x), start, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    o.sum().backward()
    for a, b in zip(_heads(x.grad), want):
        assert torch.equal(a, b)


def test_what_attention_refuses():
    x, start = _qkv()
    x.requires_grad_()
    o, lse = nopfs.packed_attention(*_heads(x), start)
    with pytest.raises(RuntimeError, match="lse"):
        (o.sum() + lse[:, :140].sum()).backward()
    with pytest.raises(ValueError, match="given outputs"):
        nopfs.packed_attention(*_heads(x), start, o=torch.empty_like(o))
    x.grad = None
    grad, = torch.autograd.grad(nopfs.packed_attention(*_heads(x), start)[0].float().square().sum(), x,
                                create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
    with torch.no_grad():
        o, lse = nopfs.packed_attention(*_heads(x), start, o=torch.empty_like(o))
    assert not o.requires_grad and not lse.requires_grad


def _logits(dtype):
    g = torch.Generator().manual_seed(2)
    s = torch.randn((30, 700), generator=g).to(dtype).cuda()
    index = torch.stack([torch.randperm(700, generator=g)[:9] for _ in range(30)]).int().cuda()
    return s, index, torch.randn((30, 9), generator=g).half().cuda(), torch.rand(30, generator=g).cuda()


@pytest.mark.parametrize("dtype", [BF, FP, F32])
def test_distill(dtype):
    s, index, y, w = _logits(dtype)
    want_loss, want = nopfs.topk_distill(s, index, y, 2.0, weight=w)
    s.requires_grad_()
    loss, ds = nopfs.topk_distill(s, index, y, 2.0, weight=w)
    assert torch.equal(loss, want_loss) and torch.equal(ds, want) and not ds.requires_grad
    loss.sum().backward()
    assert torch.equal(s.grad, want)
    s.grad = None
    each = torch.rand(30, device="cuda")
    (nopfs.topk_distill(s, index, y, 2.0, weight=w)[0] * each).sum().backward()
    assert torch.equal(s.grad, (want.float() * each[:, None]).to(dtype))


def test_what_distill_refuses():
    s, index, y, w = _logits(F32)
    s.requires_grad_()
    with pytest.raises(ValueError, match="teacher and weight"):
        nopfs.topk_distill(s, index, y, weight=w.clone().requires_grad_())
    with pytest.raises(ValueError, match="given outputs"):
        nopfs.topk_distill(s, index, y, dlogits=torch.empty_like(s))
    loss, none = nopfs.topk_distill(s, index, y, grad=False)
    assert none is None and not loss.requires_grad
    with torch.no_grad():
        loss, ds = nopfs.topk_distill(s, index, y, dlogits=torch.empty_like(s))
    assert not loss.requires_grad
