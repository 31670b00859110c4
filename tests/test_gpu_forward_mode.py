"""Forward-mode derivatives of device tensors are refused; without any the calls run."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from torch.autograd import forward_ad  # noqa: E402

from paper_2101_08734_amd import nopfs  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def test_dual_tensors():
    w, ids = torch.randn((9, 16), device="cuda"), torch.arange(9, device="cuda")
    start = torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    q = torch.randn((9, 2, 8), device="cuda")
    calls = (lambda x: nopfs.token_embed(x, ids), lambda x: nopfs.gated_scan(x, w, start)[0],
             lambda x: nopfs.gated_scan(w, x, start)[0],
             lambda x: nopfs.norm_rotate(x.view(9, 2, 8), q, ids.int())[0])
    for f in calls:
        want = f(w)
        with forward_ad.dual_level():
            with pytest.raises(ValueError, match="forward-mode"):
                f(forward_ad.make_dual(w, w))
            assert torch.equal(f(w), want)
        with pytest.raises(ValueError, match="forward-mode"):
            torch.func.jvp(f, (w,), (w,))
        assert torch.equal(f(w), want)
