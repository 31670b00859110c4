"""gated_scan(keep=False) returns no carry, in autograd's graph or not."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2101_08734_amd import nopfs  # noqa: E402


@pytest.mark.parametrize("state", [False, True])
def test_keep(state):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x, gate, dh = (torch.randn((200, 12), device="cuda") for _ in range(3))
    start = torch.tensor([0, 150, 190], dtype=torch.int32, device="cuda")
    h0 = torch.randn((2, 12), device="cuda") if state else None
    h, last, carry = nopfs.gated_scan(x, gate, start, h0)
    want = nopfs.gated_scan_grad(dh, x, gate, start, carry, h0)
    x.requires_grad_()
    for keep in (False, True):
        a, b, c = nopfs.gated_scan(x, gate, start, h0, keep=keep)
        assert torch.equal(a, h) and torch.equal(b, last)
        assert torch.equal(c, carry) and not c.requires_grad if keep else c is None
        grad, = torch.autograd.grad(a, x, dh)
        assert torch.equal(grad, want[0])
