"""nopfs_norm_rotate's angles to more than 32 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from layer_ref import E, close  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

F32, F64 = torch.float32, torch.float64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


@pytest.mark.parametrize("T", [40, 1_500])
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_close_to_a_quarter_turn(T, interleaved):
    """Angles of odd quarter turns and up to 10^-3 more: the cosine is small and as good
    as the angle. Of x = (1, 0) in each pair, out = (y cos, y sin), y off by er =
    (W / 2 + 8) E; the cosine by 4 E of itself in 32 bits, E by the correction, which is
    2^-26 turns at most and known to E, the angle's reduction in 64 bits by 2^-52 of all
    its turns, twice; products and sum 3 E, the result's rounding E. An angle rounded to
    32 bits alone would be off by up to 2^-26 turns, 9.4e-8 of y. Likewise backwards, of
    a gradient (1, 0), whose dx goes through the same angles: with g = (cos, -sin), z =
    (y, 0), dx_b = r g_b and dx_a = r (g_a - z_a mean g z)."""
    W, R = 16, 16
    i, odd = torch.arange(R // 2, dtype=F64), 2 * torch.arange(T) + 1
    freq = math.pi / 2 + 1e-4 * (i + 1) / (R * T)
    a, b = (2 * i.long(), 2 * i.long() + 1) if interleaved else (i.long(), i.long() + R // 2)
    x = torch.zeros((T, 1, W))
    x[:, :, a] = 1.0
    pos = odd.int().cuda()
    X = x.cuda()
    eps = 2.0**-20
    out = nopfs.norm_rotate(X, X, pos, freq.cuda(), eps=eps, interleaved=interleaved)
    angle = odd.to(F64)[:, None, None] * freq
    far = 2 * 2.0**-52 * angle / (2 * math.pi) * 2 * math.pi
    r = (0.5 + eps) ** -0.5
    er = (W / 2 + 8) * E
    cos, sin = angle.cos(), angle.sin()
    assert float(cos.abs().max()) < 1e-3
    bound = lambda v: (er + 9 * E) * v.abs() * r + r * (far + 2 * math.pi * 2.0**-26 * 2 * E)  # noqa: E731
    for t in out:
        close("cos", t[:, :, a], r * cos, bound(cos))
        close("sin", t[:, :, b], r * sin, bound(sin))
    dx = nopfs.norm_rotate_grad(X, X, X, X, pos, freq.cuda(), eps=eps, interleaved=interleaved)[:2]
    dot = (cos * r).sum(2, keepdim=True) / W
    for t in dx:
        close("dx b", t[:, :, b], -r * sin, bound(sin))
        close("dx a", t[:, :, a], r * (cos - r * dot),
              bound(cos) + r * ((2 * er + 10 * E + W * E) * r * (cos.abs() * r).sum(2, keepdim=True) / W
                                + r * r * (far.amax() + 2 * math.pi * 2.0**-26 * 2 * E)))


def test_sums_of_the_weights_gradients():
    """65,536 tokens of 64 heads whose terms are z = 1 times a gradient of 1 in the first
    tokens' first heads and of E in all others, which a sum of 1 does not see one by one. A
    lane adds up 16 heads of a token, 16 tokens, 4 lanes of a wave, 4 waves, 16 parts, and
    10 more: 70 E of the terms' sum, 4 E for z and the products. One chain of a lane's 256
    terms would lose 255 E."""
    T, H, W = 65_536, 64, 64
    x = torch.ones((T, H, W), dtype=torch.bfloat16, device="cuda")
    d = torch.full_like(x, E)
    d[:4_096, :4] = 1.0
    w = torch.ones(W, device="cuda")
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    dqw, dkw = nopfs.norm_rotate_grad(d, d, x, x, pos, None, w, w, eps=2.0**-60)[2:]
    want = torch.full((W,), 4_096 * 4 + (T * H - 4_096 * 4) * E, dtype=F64)
    for got in (dqw, dkw):
        close("dw", got, want, 1.01 * 75 * E * want)


@pytest.mark.parametrize("T", [4_095, 4_096 * 64, 4_096 * 64 + 1, 4_096 * 65, 600_001])
def test_sums_over_many_tokens(T):
    """Every token is in the sums once, in runs of any length: whole numbers, exactly."""
    x = torch.ones((T, 1, 8), dtype=torch.bfloat16, device="cuda")
    d = (torch.arange(T, device="cuda") % 7 - 3).bfloat16()[:, None, None].expand(T, 1, 8).contiguous()
    w = torch.ones(8, device="cuda")
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    pos[5::11] = -1
    dqw, dkw = nopfs.norm_rotate_grad(d, d, x, x, pos, None, w, w, eps=2.0**-60)[2:]
    want = d[pos >= 0].double().sum((0, 1))
    assert torch.equal(dqw.double(), want) and torch.equal(dkw.double(), want)
