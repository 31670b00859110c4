"""The gradient of nopfs_packed_attention in fp16 over the magnitudes of do that
its type has: dS may pass 65504 or fall among the subnormals where dq and dk do
neither."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2101_08734_amd import nopfs  # noqa: E402

FP = torch.float16
U = 2.0**-11


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _ratios(lengths, heads, kv_heads, width, do, seed, spread=1.0, scale=None):
    """For dq, dk and dv the mean over rows of a row's square error over what it
    may be off by in the mean square: dS, P and the outputs are each rounded by
    U / sqrt(3) of their value at most (outputs below 2^-14 by 2^-25 / sqrt(3)),
    independently; delta and products as in the bfloat16 test of sharp rows. A
    value beyond 65504 has to be infinite, and no other."""
    g = torch.Generator().manual_seed(seed)
    T = sum(lengths)
    q = (torch.randn((T, heads, width), generator=g) * spread).to(FP).cuda()
    k, v = ((torch.randn((T, kv_heads, width), generator=g) * spread).to(FP).cuda() for _ in range(2))
    d = (torch.randn((T, heads, width), generator=g) * do(T, heads, g)).clamp(-65504, 65504).to(FP).cuda()
    start = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    scale = width**-0.5 if scale is None else scale
    o, lse = nopfs.packed_attention(q, k, v, start, scale=scale)
    got = nopfs.packed_attention_grad(d, q, k, v, o, lse, start, scale=scale)
    group = heads // kv_heads
    want = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in got]
    may = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in got]
    a = 0
    for L in lengths:
        b = a + L
        for h in range(heads):
            qi, ki, vi, di = (x.double() for x in (q[a:b, h], k[a:b, h // group], v[a:b, h // group], d[a:b, h]))
            seen = torch.ones(L, L, dtype=torch.bool, device="cuda").tril()
            p = torch.softmax(torch.where(seen, qi @ ki.T.contiguous() * scale, -math.inf), 1)
            dp = di @ vi.T.contiguous()
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            noise = ds**2 * U**2 / 3 + (p * (di.abs() @ vi.abs().T.contiguous()) * 2.0**-23)**2
            eps = ((di**2 * (p @ vi)**2).sum(1) + (p**2 * dp**2).sum(1)) * U**2 / 3
            light = torch.where(p < 1 / 8, p, 0.0) @ ki
            want[0][a:b, h] = ds @ ki * scale
            may[0][a:b, h] = (noise @ ki**2 + eps[:, None] * light**2) * scale**2
            want[1][a:b, h // group] += ds.T.contiguous() @ qi * scale
            may[1][a:b, h // group] += noise.T.contiguous() @ qi**2 * scale**2
            want[2][a:b, h // group] += p.T.contiguous() @ di
            may[2][a:b, h // group] += (p**2).T.contiguous() @ di**2 * U**2 / 3
        a = b
    out = []
    for x, w, m in zip(got, want, may):
        x = x.double()
        m = m + torch.clamp(w.abs() * U, min=2.0**-25)**2 / 3
        big = w.abs() > 65504 * (1 + 2.0**-10)
        edge = (w.abs() > 65504 * (1 - 2.0**-8)) & ~big
        assert bool(torch.isinf(x[big]).all())
        assert bool(torch.isfinite(x[~big & ~edge]).all()), int((~torch.isfinite(x[~big & ~edge])).sum())
        ok = ~big & ~edge
        off = torch.where(ok, (x - w)**2, 0.0).nan_to_num(0.0, 0.0, 0.0).sum(2)
        out.append(float((off / torch.where(ok, m, 0.0).sum(2).clamp(min=1e-300)).mean()))
    return out


def _check(*args, **kw):
    r = _ratios(*args, **kw)
    assert max(r) <= 1.0, r


SHAPES = [([256], 2, 2, 64), ([700, 64, 33, 1, 0, 100], 3, 1, 80), ([1_500], 2, 1, 128), ([90, 200], 260, 260, 64),
          ([64, 200], 260, 130, 128), ([3_300, 100], 1, 1, 64), ([3_300], 2, 1, 128)]


@pytest.mark.parametrize("lengths,heads,kv_heads,width", SHAPES)
@pytest.mark.parametrize("size", [1e-6, 1e-4, 1e-2, 1.0, 1e3, 1.5e4])
def test_sizes_of_do(size, lengths, heads, kv_heads, width):
    _check(lengths, heads, kv_heads, width, lambda *_: size, width)


@pytest.mark.parametrize("lengths,heads,kv_heads,width", SHAPES)
def test_rows_and_heads_of_different_sizes(lengths, heads, kv_heads, width):
    """do of a row and head between 1e-4 and 1e3."""
    _check(lengths, heads, kv_heads, width,
           lambda T, H, g: 10.0**(torch.rand((T, H, 1), generator=g) * 7 - 4), width)


@pytest.mark.parametrize("grow", [False, True])
def test_do_along_a_sample(grow):
    """From 1e-5 to 1e4 along the rows, and back: the running scales move."""
    def do(T, H, g):
        x = 10.0**torch.linspace(-5, 4, T)[:, None, None]
        return x if grow else x.flip(0)
    for shape in SHAPES:
        _check(*shape, do, 5)


@pytest.mark.parametrize("T", [8_192, 20_000])
@pytest.mark.parametrize("size", [1e-3, 10.0])
def test_long_samples(T, size):
    _check([T], 1, 1, 64, lambda *_: size, 6)


def test_large_sums_of_small_outputs():
    """dS beyond 65504 where the scale brings dq and dk back."""
    _check([256], 2, 2, 64, lambda *_: 1.6e4, 7, spread=2.0, scale=2.0**-7)
    _check([40] * 6, 2, 2, 128, lambda *_: 1.6e4, 8, spread=4.0, scale=2.0**-9)


def test_a_row_of_infinities_and_not_a_number():
    """They reach the rows that depend on them and the neighbours that the header
    names, and take no scale from the others."""
    lengths = [200, 300]
    g = torch.Generator().manual_seed(9)
    q, k, v, do = (torch.randn((500, 2, 64), generator=g).to(FP).cuda() for _ in range(4))
    do *= 1e-3
    start = torch.tensor([0, 200, 500], dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, start)
    clean = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
    for bad in (math.inf, math.nan):
        d = do.clone()
        d[300, 0, 3] = bad  # row 100 of the second sample: keys 200..300 of head 0, 31 more at most
        dq, dk, dv = nopfs.packed_attention_grad(d, q, k, v, o, lse, start)
        assert torch.equal(dq[:300], clean[0][:300]) and torch.equal(dq[301:], clean[0][301:])
        assert torch.equal(dq[:, 1], clean[0][:, 1])
        for x, c in ((dk, clean[1]), (dv, clean[2])):
            assert torch.equal(x[:200], c[:200]) and torch.equal(x[:, 1], c[:, 1])
            far = x[352:, 0].double() - c[352:, 0].double()
            assert float(far.abs().max()) <= 2.0**-10 * float(c[352:, 0].double().abs().max())
