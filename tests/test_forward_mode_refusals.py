"""Forward-mode derivatives are refused by every call of a training step that would
drop them, before anything else is looked at (no GPU)."""
import pytest

nopfs = pytest.importorskip("paper_2101_08734_amd.nopfs")
torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

X = torch.zeros((4, 2, 8))  # tokens by heads
R, V = torch.zeros((4, 8)), torch.zeros(8)
I, S = torch.zeros(4, dtype=torch.int32), torch.tensor([0, 4], dtype=torch.int32)

CALLS = {
    "token_embed": (nopfs.token_embed, [R, I], [0]),
    "token_embed_grad": (nopfs.token_embed_grad, [R, I, 4], [0]),
    "norm_rotate": (nopfs.norm_rotate, [X, X, I, V[:4].double(), V, V], [0, 1, 3, 4, 5]),
    "norm_rotate_grad": (nopfs.norm_rotate_grad, [X, X, X, X, I, V[:4].double(), V, V], [0, 1, 2, 3, 5, 6, 7]),
    "gated_scan": (nopfs.gated_scan, [R, R, S, R[:1]], [0, 1, 3]),
    "gated_scan_grad": (nopfs.gated_scan_grad, [R, R, R, S, R[:1], R[:1], R[:1]], [0, 1, 2, 4, 5, 6]),
    "packed_attention": (nopfs.packed_attention, [X, X, X, S], [0, 1, 2]),
    "packed_attention_grad": (nopfs.packed_attention_grad, [X, X, X, X, X, V, S], [0, 1, 2, 3, 4, 5]),
    "topk_distill": (nopfs.topk_distill, [R, R.int(), R, 1.0, V[:4]], [0, 2, 4]),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("requires_grad", [False, True])
def test_tangents(name, requires_grad):
    call, args, duals = CALLS[name]
    for i in duals:
        with forward_ad.dual_level():
            given = list(args)
            given[i] = forward_ad.make_dual(given[i].clone().requires_grad_(requires_grad), torch.ones_like(given[i]))
            with pytest.raises(ValueError, match="forward-mode"):
                call(*given)
            given[i] = forward_ad.unpack_dual(given[i]).primal.detach()
            with pytest.raises((TypeError, RuntimeError)):  # the next thing that is wrong: no GPU, or not there
                call(*given)


@pytest.mark.parametrize("name", ["token_embed", "norm_rotate", "gated_scan"])
def test_jvp(name):
    call, args, _ = CALLS[name]
    with pytest.raises(ValueError, match="forward-mode"):
        torch.func.jvp(lambda x: call(x, *args[1:]), (args[0],), (args[0],))
