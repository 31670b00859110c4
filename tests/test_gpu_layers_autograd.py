"""The layers of a token model under autograd: outputs are in the graph of inputs
that require gradients, with the gradients of the calls that make them, on any
stream, and what cannot be differentiated is refused."""
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


def _broken(shape, dtype):
    """Gradients as autograd may hand them over: broadcast, transposed, of odd strides."""
    yield torch.ones((), dtype=dtype, device="cuda").expand(shape)
    back = torch.randn(tuple(reversed(shape)), device="cuda").to(dtype)
    yield back.permute(*reversed(range(len(shape))))
    yield torch.randn((*shape[:-1], 2 * shape[-1]), device="cuda").to(dtype)[..., ::2]
    yield torch.randn((*shape[:-1], shape[-1] + 3), device="cuda").to(dtype)[..., 1:-2]


@pytest.mark.parametrize("slots", [False, True])
def test_embed(slots):
    w = torch.randn((60, 24), device="cuda")
    ids = torch.randint(-1, 60, (200,), device="cuda")
    slot = torch.randint(-1, 200, (150,), device="cuda") if slots else None
    out = nopfs.token_embed(w, ids, 0.7, slot=slot, dtype=BF)
    w.requires_grad_()
    for d in _broken(tuple(out.shape), BF):
        w.grad = None
        got = nopfs.token_embed(w, ids, 0.7, slot=slot, dtype=BF)
        assert torch.equal(got, out)
        got.backward(d)
        assert torch.equal(w.grad, nopfs.token_embed_grad(d.contiguous(), ids, 60, 0.7, slot=slot, dtype=F32))
    with pytest.raises(ValueError, match="given outputs"):
        nopfs.token_embed(w, ids, out=torch.empty((200, 24), device="cuda"))
    with torch.no_grad():
        assert not nopfs.token_embed(w, ids).requires_grad


def _qk(dtype=BF):
    x = torch.randn((70, 6, 32), device="cuda").to(dtype)
    pos = torch.arange(70, device="cuda", dtype=torch.int32) - 1
    freq = 100.0 ** (-torch.arange(0, 32, 2, dtype=torch.float64, device="cuda") / 32)
    return x, pos, freq, torch.rand(32, device="cuda") + 0.5, torch.rand(32, device="cuda") + 0.5


def test_rotate():
    x, pos, freq, qw, kw = _qk()
    outs = nopfs.norm_rotate(x[:, :4], x[:, 4:], pos, freq, qw, kw, interleaved=True)
    for t in (x, qw, kw):
        t.requires_grad_()
    for dq, dk in zip(_broken((70, 4, 32), BF), _broken((70, 2, 32), BF)):
        x.grad = qw.grad = kw.grad = None
        got = nopfs.norm_rotate(x[:, :4], x[:, 4:], pos, freq, qw, kw, interleaved=True)
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
        torch.autograd.backward(got, (dq, dk))
        with torch.no_grad():
            want = nopfs.norm_rotate_grad(dq.contiguous(), dk.contiguous(), x[:, :4], x[:, 4:], pos, freq, qw, kw,
                                          interleaved=True)
        assert torch.equal(x.grad, torch.cat(want[:2], 1))
        assert torch.equal(qw.grad, want[2]) and torch.equal(kw.grad, want[3])
    with pytest.raises(ValueError, match="given outputs"):
        nopfs.norm_rotate(x[:, :4], x[:, 4:], pos, freq, q_out=torch.empty_like(outs[0]))
    with pytest.raises(ValueError, match="gradient by freq"):
        nopfs.norm_rotate(x[:, :4], x[:, 4:], pos, freq.clone().requires_grad_())


def test_rotate_of_one_output_or_input():
    x, pos, freq, qw, kw = _qk(F32)
    k = x[:, 4:].clone().requires_grad_()
    q_out, k_out = nopfs.norm_rotate(x[:, :4], k, pos, freq, qw, kw)
    k_out.sum().backward()
    want = nopfs.norm_rotate_grad(torch.zeros_like(q_out), torch.ones_like(k_out), x[:, :4], k.detach(), pos, freq,
                                  qw, kw)
    assert torch.equal(k.grad, want[1])
    qw.requires_grad_()
    nopfs.norm_rotate(x[:, :4], x[:, 4:], pos, freq, qw, None)[0].sum().backward()
    assert qw.grad is not None and kw.grad is None


def _scan_inputs(dtype=BF, state=True):
    both = torch.randn((90, 2 * 20), device="cuda").to(dtype)
    start = torch.tensor([0, 30, 30, 85], dtype=torch.int32, device="cuda")
    return both, start, torch.randn((3, 20), device="cuda") if state else None


@pytest.mark.parametrize("state", [False, True])
def test_scan(state):
    both, start, h0 = _scan_inputs(state=state)
    h, last, carry = nopfs.gated_scan(both[:, :20], both[:, 20:], start, h0)
    both.requires_grad_()
    if state:
        h0.requires_grad_()
    for dh in _broken((90, 20), BF):
        both.grad = None
        a, b, c = nopfs.gated_scan(both[:, :20], both[:, 20:], start, h0)
        assert torch.equal(a, h) and torch.equal(b, last) and not c.requires_grad
        dlast = torch.randn((20, 3), device="cuda").T
        if state:
            h0.grad = None
        torch.autograd.backward((a, b), (dh, dlast))
        with torch.no_grad():
            want = nopfs.gated_scan_grad(dh.contiguous(), both[:, :20], both[:, 20:], start, carry, h0,
                                         dlast.contiguous())
        assert torch.equal(both.grad, torch.cat(want[:2], 1))
        if state:
            assert torch.equal(h0.grad, want[2])
    # of one output alone
    both.grad = None
    nopfs.gated_scan(both[:, :20], both[:, 20:], start, h0)[1].sum().backward()
    with torch.no_grad():
        want = nopfs.gated_scan_grad(torch.zeros_like(h), both[:, :20], both[:, 20:], start, carry, h0,
                                     torch.ones_like(last))
    assert torch.equal(both.grad, torch.cat(want[:2], 1))
    with pytest.raises(ValueError, match="given outputs"):
        nopfs.gated_scan(both[:, :20], both[:, 20:], start, h=torch.empty_like(h))


def test_gradients_of_gradients_are_refused():
    both, start, _ = _scan_inputs(F32)
    both.requires_grad_()
    h = nopfs.gated_scan(both[:, :20], both[:, 20:], start)[0]
    grad, = torch.autograd.grad(h.square().sum(), both, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()


def test_on_another_stream():
    x, pos, freq, qw, kw = _qk()
    both, start, h0 = _scan_inputs()
    w, ids = torch.randn((60, 24), device="cuda"), torch.randint(0, 60, (200,), device="cuda")
    leaves = [w, x, qw, kw, both, h0]
    for t in leaves:
        t.requires_grad_()

    def run(stream):
        for t in leaves:
            t.grad = None
        out = nopfs.token_embed(w, ids, stream=stream)
        q, k = nopfs.norm_rotate(x[:, :4], x[:, 4:], pos, freq, qw, kw, stream=stream)
        h, last, _ = nopfs.gated_scan(both[:, :20], both[:, 20:], start, h0, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        total = out.sum() + q.float().square().sum() + k.float().sum() + h.float().square().sum() + last.sum()
        total.backward()
        return [t.grad for t in leaves]

    want = run(None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for a, b in zip(run(s), want):
        assert torch.equal(a, b)
