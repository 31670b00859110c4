"""The gradient of nopfs_packed_attention where a few keys have most of a row's
weight: there dP - delta is small on them, and delta = do.o from the rounded o
would be off by more than that."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _ratio(lengths, heads, width, dtype, spread, seed):
    """Square sums over all rows of what dq and dk are off by, over what they
    may be. dS and the outputs are rounded to the inputs' type, of unit u (half the
    spacing over the least value that has it): each rounding is off by u / sqrt(3)
    of its value at most in the mean square, all of them independent. Products in
    32 bits leave dP off by 2^-23 sum |do||v|. delta is off by the roundings of o
    and of P in it, in the mean square sqrt(sum do^2 o^2 + sum P^2 dP^2) u / sqrt(3),
    which may reach dq with the keys that have less than a 16th of the row."""
    g = torch.Generator().manual_seed(seed)
    T = sum(lengths)
    q, k, v, do = (torch.randn((T, heads, width), generator=g) for _ in range(4))
    q, k = q * spread**0.5, k * spread**0.5
    q, k, v, do = (x.to(dtype).cuda() for x in (q, k, v, do))
    start = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    o, lse = nopfs.packed_attention(q, k, v, start)
    dq, dk, _ = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
    u, scale = (2.0**-8 if dtype == BF else 2.0**-11), width**-0.5
    off, allowed = [0.0, 0.0], [0.0, 0.0]
    a = 0
    for L in lengths:
        b = a + L
        for h0 in range(0, heads, 16):
            hs = slice(h0, min(heads, h0 + 16))
            qi, ki, vi, di = (x[a:b, hs].double().transpose(0, 1).contiguous() for x in (q, k, v, do))
            seen = torch.ones(L, L, dtype=torch.bool, device="cuda").tril()
            s = torch.where(seen, qi @ ki.transpose(1, 2).contiguous() * scale, -math.inf)
            p, dp = torch.softmax(s, 2), di @ vi.transpose(1, 2).contiguous()
            ds = p * (dp - (p * dp).sum(2, keepdim=True))
            noise = ds**2 * u**2 / 3 + (p * (di.abs() @ vi.abs().transpose(1, 2).contiguous()) * 2.0**-23)**2
            wq, wk = ds @ ki * scale, ds.transpose(1, 2).contiguous() @ qi * scale
            eps = ((di**2 * (p @ vi)**2).sum(2) + (p**2 * dp**2).sum(2)) * u**2 / 3
            light = torch.where(p < 1 / 16, p, 0.0) @ ki
            off[0] += float(((dq[a:b, hs].double().transpose(0, 1) - wq)**2).sum())
            off[1] += float(((dk[a:b, hs].double().transpose(0, 1) - wk)**2).sum())
            allowed[0] += float((noise @ ki**2).sum() * scale**2 + (wq**2).sum() * u**2 / 3)
            allowed[0] += float((eps * (light**2).sum(2)).sum() * scale**2)
            allowed[1] += float((noise.transpose(1, 2).contiguous() @ qi**2).sum() * scale**2
                                + (wk**2).sum() * u**2 / 3)
        a = b
    return [x / y for x, y in zip(off, allowed)]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("spread", [1.0, 4.0, 9.0, 16.0])
@pytest.mark.parametrize("lengths,heads,width", [
    ([700, 1, 130, 33], 2, 64), ([1_024], 1, 128), ([640, 64], 3, 80), ([900], 2, 32),
    ([300, 70, 2], 200, 64), ([200, 129], 260, 128), ([3_300, 500], 1, 64), ([3_300], 1, 128),
    ([5_000], 3, 96)])
def test_sharp_rows(lengths, heads, width, spread, dtype):
    dq, dk = _ratio(lengths, heads, width, dtype, spread, int(spread) + width)
    assert dq <= 1.0 and dk <= 1.0, (dq, dk)
