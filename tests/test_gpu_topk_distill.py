"""nopfs_topk_distill against 64 bits within step_ref's bounds: every type of
logits and teacher, odd widths and strides (rows that are not aligned), rows
masked by weight or by their entries, classes named twice, infinities, in-place
gradients, and the gradient against differences."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import step_ref  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
NAMES = {BF: "bf16", FP: "fp16", F32: "fp32"}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _inputs(T, V, K, dtype, teacher, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    s = (torch.randn((T, V), generator=g) * spread).to(dtype)
    index = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).to(torch.int32)
    y = (torch.randn((T, K), generator=g) * 2 + 3).to(teacher)
    w = torch.rand(T, generator=g) + 0.1
    return s.cuda(), index.cuda(), y.cuda(), w.cuda()


def _close(name, got, val, err):
    got = got.detach().cpu().double()
    inf = torch.isinf(val)
    assert torch.equal(got[inf], val[inf]), name
    diff = (got - val)[~inf].abs()
    bad = ~(diff <= err[~inf])
    assert not bad.any(), (name, float(diff[bad].max()), int(bad.sum()))


def _run_and_check(s, index, y, tau=1.0, w=None):
    ref = step_ref.distill(s, index, y, tau, w)
    loss, ds = nopfs.topk_distill(s, index, y, tau, weight=w)
    _close("loss", loss, ref[0], ref[2])
    _close("gradient", ds, ref[1], ref[3])
    alone, none = nopfs.topk_distill(s, index, y, tau, weight=w, grad=False)
    assert none is None and torch.equal(alone, loss)
    return loss, ds


@pytest.mark.parametrize("dtype", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 255, 1_000, 2_047, 4_097, 21_841, 50_021, 131_072,
                               150_001])
def test_widths(dtype, V):
    K = min(V, 37)
    s, index, y, w = _inputs(5 if V < 30_000 else 3, V, K, dtype, FP, V)
    _run_and_check(s, index, y, 1.0, w)


@pytest.mark.parametrize("teacher", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("tau", [0.25, 1.0, 4.0])
def test_teachers_and_temperatures(teacher, tau):
    s, index, y, w = _inputs(9, 777, 33, BF, teacher, 3)
    _run_and_check(s, index, y, tau, w)
    _run_and_check(s, index, y, tau)


@pytest.mark.parametrize("K", [1, 63, 64, 65, 300, 1_024])
def test_entries(K):
    s, index, y, w = _inputs(4, 3_001, K, BF, FP, K)
    _run_and_check(s, index, y, 2.0, w)


@pytest.mark.parametrize("T", [1, 2, 255, 4_099])
def test_rows(T):
    s, index, y, w = _inputs(T, 50, 5, F32, F32, T)
    _run_and_check(s, index, y, 1.5, w)


@pytest.mark.parametrize("dtype", [BF, F32], ids=NAMES.get)
@pytest.mark.parametrize("stride,shift", [(1_000, 0), (1_003, 1), (1_024, 3), (1_016, 8)])
def test_strided_rows(dtype, stride, shift):
    """Rows of a wider array from any element on, gradients into another of
    another alignment; what lies between the rows stays."""
    s0, index, y, w = _inputs(7, 990, 20, dtype, FP, stride)
    wide = torch.full((7, stride), math.nan, dtype=dtype, device="cuda").view(-1)
    s = torch.as_strided(wide, (7, 990), (stride, 1), shift)
    s.copy_(s0)
    want = _run_and_check(s0, index, y, 1.0, w)
    got = _run_and_check(s, index, y, 1.0, w)
    flat = torch.full((7 * 1_001 + 5,), 9.0, dtype=dtype, device="cuda")
    ds = torch.as_strided(flat, (7, 990), (1_001, 1), 5)
    got2 = nopfs.topk_distill(s, index, y, 1.0, weight=w, dlogits=ds)
    for a in (got, got2):
        assert torch.allclose(a[0], want[0], rtol=1e-5, atol=0)
    _close("gradient", ds, *step_ref.distill(s0, index, y, 1.0, w)[1::2])
    outside = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(outside, (7, 990), (1_001, 1), 5).fill_(False)
    assert bool((flat[outside] == 9.0).all())
    teacher = torch.full((7, 31), -5.0, dtype=FP, device="cuda")
    teacher[:, 3:23] = y
    names = torch.full((7, 25), 4, dtype=torch.int32, device="cuda")
    names[:, 5:] = index
    again = nopfs.topk_distill(s, names[:, 5:], teacher[:, 3:23], 1.0, weight=w)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("V", [990, 40_000, 200_003])
@pytest.mark.parametrize("dtype", [FP, F32], ids=NAMES.get)
def test_in_place(V, dtype):
    s, index, y, w = _inputs(6, V, 9, dtype, FP, V)
    w[2] = 0.0
    loss, ds = nopfs.topk_distill(s, index, y, 2.0, weight=w)
    loss2, same = nopfs.topk_distill(s, index, y, 2.0, weight=w, dlogits=s)
    assert same is s and torch.equal(loss, loss2) and torch.equal(ds, s)


def test_masked_rows_and_entries():
    s, index, y, w = _inputs(8, 300, 6, BF, F32, 1)
    w[0] = 0.0
    s[0] = math.nan        # masked by its weight: not read
    index[1] = -1
    s[1] = math.inf        # masked by its entries
    y[2] = -math.inf
    index[3, 2:] = 300     # entries beyond the classes
    y[4, :3] = -math.inf   # entries of no mass
    index[4, :3] = index[4, 3]
    index[5, 1] = -2**31
    y[6] = torch.finfo(F32).min
    loss, ds = _run_and_check(s, index, y, 1.0, w)
    assert not loss[:3].any() and not ds[:3].any()
    assert bool((loss[3:] > 0).all())


def test_classes_named_twice():
    s, index, y, w = _inputs(5, 64, 40, F32, F32, 2)
    index[:, 1::2] = index[:, ::2]
    index[4] = 7
    _run_and_check(s, index, y, 1.0, w)


def test_infinite_and_lowest_logits():
    s, index, y, w = _inputs(6, 5_000, 8, BF, F32, 4)
    s[0, ::2] = -math.inf              # classes that a mask took out
    s[0, index[0].long()] = 1.0
    s[1, :] = torch.finfo(BF).min
    s[1, index[1].long()] = 0.0
    s[2, :] = -math.inf
    s[2, 4_999] = 2.0
    index[2, :] = 4_999
    s[3, :4_000] = -math.inf           # a long stretch of them
    s[3, index[3].long()] = 0.5
    s[4, :] = 3.0e38                   # the largest, all equal
    s[5, int(index[5, 0])] = -math.inf  # the teacher wants what the student cannot give
    loss, ds = nopfs.topk_distill(s, index, y, 1.0, weight=w)
    ref = step_ref.distill(s[:5], index[:5], y[:5], 1.0, w[:5])
    _close("loss", loss[:5], ref[0], ref[2])
    _close("gradient", ds[:5], ref[1], ref[3])
    assert float(loss[5]) == math.inf and bool(torch.isfinite(ds[5]).all())


def test_not_a_number_is_not_hidden():
    s, index, y, w = _inputs(3, 500, 4, F32, F32, 5)
    s[0, 17] = math.nan
    y[1, 2] = math.nan
    loss, ds = nopfs.topk_distill(s, index, y, 1.0, weight=w)
    assert math.isnan(loss[0]) and math.isnan(loss[1]) and bool(torch.isfinite(loss[2]))
    assert bool(torch.isnan(ds[0]).all()) and bool(torch.isnan(ds[1, index[1].long()]).all())


def test_gradient_against_differences():
    """Logits in 32 bits, step 2^-5: a central difference is off by h^2 / 6
    times a third derivative (at most w / tau^2 per class and entry pair here)
    and by the loss's own 2^-20 over h."""
    T, V, K = 3, 20, 4
    s, index, y, w = _inputs(T, V, K, F32, F32, 6, 1.0)
    h, tau = 2.0**-5, 1.5
    _, ds = nopfs.topk_distill(s, index, y, tau, weight=w)
    for v in range(V):
        up, down = s.clone(), s.clone()
        up[:, v] += h
        down[:, v] -= h
        step = up[:, v].double() - down[:, v].double()
        f1 = nopfs.topk_distill(up, index, y, tau, weight=w, grad=False)[0].double()
        f0 = nopfs.topk_distill(down, index, y, tau, weight=w, grad=False)[0].double()
        diff = (f1 - f0) / step
        assert float((diff - ds[:, v].double()).abs().max()) <= h * h / tau + 2.0**-17 / h


def test_more_rows_than_one_launch_dimension_holds():
    """2^26 workgroups of 64 threads are 2^32 threads."""
    T = 2**26 + 5
    s, index, y, w = _inputs(64, 8, 1, BF, BF, 7)

    def rows(x):
        return x[:61].repeat(T // 61 + 1, *[1] * (x.dim() - 1))[:T]

    loss, ds = nopfs.topk_distill(rows(s), rows(index), rows(y), 1.0, weight=rows(w))
    one, grad = nopfs.topk_distill(s[:61], index[:61], y[:61], 1.0, weight=w[:61])
    assert torch.equal(loss, rows(one)) and torch.equal(ds, rows(grad))


def test_offsets_past_32_bits():
    """Rows so far apart that byte offsets pass 2^32."""
    T, V, stride = 36, 700, 2**26 + 8
    s, index, y, w = _inputs(T, V, 9, BF, FP, 8)
    one, grad = nopfs.topk_distill(s, index, y, 1.0, weight=w)
    far = torch.empty((T - 1) * stride + V, dtype=BF, device="cuda").as_strided((T, V), (stride, 1))
    far.copy_(s)
    loss, ds = nopfs.topk_distill(far, index, y, 1.0, weight=w, dlogits=far)
    assert torch.equal(loss, one) and torch.equal(ds, grad)
