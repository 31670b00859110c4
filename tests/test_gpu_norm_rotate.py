"""nopfs_norm_rotate and its gradient against 64 bits within layer_ref's bounds: the
types, widths, kinds of pairs and parts rotated, far positions, padding, strides of
any alignment, in place, values whose squares overflow, and differences."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import layer_ref  # noqa: E402
from layer_ref import close  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
NAMES = {BF: "bf16", FP: "fp16", F32: "fp32"}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _freq(R):
    return 10_000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / max(R, 1)) if R else None


def _inputs(T, H, Hk, W, dt=BF, wd=F32, R=None, seed=0, far=0, weights=True, padding=True):
    g = torch.Generator().manual_seed(seed)
    x = (1.5 * torch.randn((T, H + Hk, W), generator=g)).to(dt).cuda()
    pos = torch.randint(0, far + 300, (T,), generator=g).int()
    if padding and T > 4:
        pos[[1, T - 1]] = -1
    w = [(1 + 0.2 * torch.randn(W, generator=g)).to(wd).cuda() if weights else None for _ in range(2)]
    d = torch.randn((T, H + Hk, W), generator=g).to(dt).cuda()
    return x[:, :H], x[:, H:], pos.cuda(), _freq(W if R is None else R), *w, d[:, :H], d[:, H:]


def _check(q, k, pos, freq, qw, kw, dq, dk, eps=1e-6, interleaved=False):
    args, how = (q, k, pos, freq, qw, kw), dict(eps=eps, interleaved=interleaved)
    outs = nopfs.norm_rotate(*args, **how)
    grads = nopfs.norm_rotate_grad(dq, dk, *args, **how)
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    for i, (x, w, d) in enumerate(((q, qw, dq), (k, kw, dk))):
        val, err = layer_ref.rotate(x, pos, freq, w, eps32, interleaved, d)
        close(f"out {i}", outs[i], val["out"], err["out"])
        close(f"dx {i}", grads[i], val["dx"], err["dx"])
        if w is None:
            assert grads[2 + i] is None
        else:
            assert grads[2 + i].dtype is w.dtype
            close(f"dw {i}", grads[2 + i], val["dw"], err["dw"])
    again = nopfs.norm_rotate_grad(dq, dk, *args, **how)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(grads, again))
    return outs, grads


@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("wd", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("interleaved", [False, True])
def test_types(dt, wd, interleaved):
    _check(*_inputs(37, 4, 2, 64, dt, wd), interleaved=interleaved)


@pytest.mark.parametrize("W", [8, 16, 24, 32, 40, 64, 80, 96, 112, 128, 136, 200, 256])
@pytest.mark.parametrize("part", [0, 1, 2, 3])
def test_widths(W, part):
    R = [0, 8, W // 16 * 8, W][part]
    _check(*_inputs(21, 3, 1, W, BF, F32, R=R, seed=W), interleaved=part == 1)
    _check(*_inputs(9, 2, 5, W, F32, F32, R=R, seed=W + 1), interleaved=W % 16 == 0)


@pytest.mark.parametrize("T", [0, 1, 2, 3, 4, 5, 1_023, 1_024, 1_025, 1_030, 4_097])
def test_tokens(T):
    _check(*_inputs(T, 2, 1, 16, seed=T, wd=BF))


@pytest.mark.parametrize("H,Hk", [(1, 1), (7, 1), (16, 4), (32, 8), (5, 33), (40, 40)])
def test_heads(H, Hk):
    _check(*_inputs(6, H, Hk, 128, seed=H))
    _check(*_inputs(6, H, Hk, 32, FP, FP, seed=H))


@pytest.mark.parametrize("far", [100_000, 2**24, 2**31 - 400])
def test_far_positions(far):
    _check(*_inputs(40, 2, 1, 64, F32, F32, far=far))


def test_without_weights():
    a = _inputs(50, 4, 2, 64, weights=False)
    _check(*a)
    one = list(a)
    one[4] = torch.rand(64, device="cuda").to(BF)
    _check(*one)
    assert nopfs.norm_rotate_grad(*one[6:], *one[:6], weights=False)[2] is None


@pytest.mark.parametrize("T", [40, 1_500])
def test_padding_alone(T):
    q, k, pos, freq, qw, kw, dq, dk = _inputs(T, 2, 2, 32)
    pos.fill_(-1)
    for x in (q, k, dq, dk):
        x.fill_(math.nan)
    outs = nopfs.norm_rotate(q, k, pos, freq, qw, kw)
    grads = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw)
    assert all(bool((x == 0).all()) for x in (*outs, *grads))


def test_nan_stays_in_its_head():
    q, k, pos, freq, qw, kw, dq, dk = _inputs(30, 4, 4, 32, padding=False)
    want = nopfs.norm_rotate(q, k, pos, freq, qw, kw)
    want_g = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw)
    q[5, 2, 7] = math.nan
    k[6, 3] = math.inf
    outs = nopfs.norm_rotate(q, k, pos, freq, qw, kw)
    grads = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw)
    for a, b, (t, h) in ((outs[0], want[0], (5, 2)), (outs[1], want[1], (6, 3)),
                         (grads[0], want_g[0], (5, 2)), (grads[1], want_g[1], (6, 3))):
        same = torch.ones(a.shape[:2], dtype=torch.bool)
        same[t, h] = False
        assert torch.equal(a[same], b[same]) and bool(torch.isnan(a[t, h]).any())
    # 1 / sqrt(inf) is 0: without a rotation the finite elements of such a head are 0
    for dt in (BF, FP, F32):
        x = torch.ones((1, 1, 32), dtype=dt, device="cuda")
        x[0, 0, 3] = -math.inf
        y = nopfs.norm_rotate(x, x, pos[:1])[0][0, 0]
        assert bool(torch.isnan(y[3])) and int((y == 0).sum()) == 31


@pytest.mark.parametrize("dt,big", [(BF, 1e30), (F32, 1e30), (F32, 2e19), (BF, 3e38), (F32, 3e38)])
def test_squares_that_overflow(dt, big):
    """The norm does not see how large x is; dx is as small as x is large."""
    a = list(_inputs(20, 2, 1, 64, dt, F32))
    for i in (0, 1):
        a[i] = (a[i].float() / a[i].abs().max().float() * big).to(dt)
    _check(*a)


@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("eps", [2.0**-60, 1e-6, 1.0, 2.0**60])
def test_eps_and_zero_heads(dt, eps):
    a = _inputs(20, 2, 1, 64, dt, F32)
    a[0][3] = 0.0
    a[0][4] *= 1e-3
    if eps < 1e-6 and dt is FP:
        a[6][3] = 0.0  # r = 2^30: out of fp16's range
    if eps < 1e-6:
        a[6][3] *= 2.0**-20
    _check(*a, eps=eps)


@pytest.mark.parametrize("dt", [BF, F32], ids=NAMES.get)
@pytest.mark.parametrize("shift,token,head", [(0, 200, 40), (1, 203, 41), (3, 640, 128), (0, 40, 40 * 33)])
def test_strides(dt, shift, token, head):
    """Heads of wider arrays from any element on, head-major among them; what lies
    between them stays."""
    T, H, W = 33, 4, 40
    q0, k0, pos, freq, qw, kw, dq0, dk0 = _inputs(T, H, H, W, dt, F32)
    outs, grads = _check(q0, k0, pos, freq, qw, kw, dq0, dk0)

    def strided(like, fill):
        flat = torch.full((T * token + H * head + 8,), fill, dtype=dt, device="cuda")
        view = torch.as_strided(flat, (T, H, W), (token, head, 1), shift)
        if like is not None:
            view.copy_(like)
        return flat, view

    q, k, dq, dk = (strided(x, math.nan)[1] for x in (q0, k0, dq0, dk0))
    (fq, oq), (fk, ok) = strided(None, 5.0), strided(None, 6.0)
    nopfs.norm_rotate(q, k, pos, freq, qw, kw, q_out=oq, k_out=ok)
    assert torch.equal(oq, outs[0]) and torch.equal(ok, outs[1])
    (gq, wq), (gk, wk) = strided(None, 5.0), strided(None, 6.0)
    got = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw, dq=wq, dk=wk)
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    held = torch.ones_like(fq, dtype=torch.bool)
    torch.as_strided(held, (T, H, W), (token, head, 1), shift).fill_(False)
    for flat, fill in ((fq, 5.0), (fk, 6.0), (gq, 5.0), (gk, 6.0)):
        assert bool((flat[held] == fill).all())


@pytest.mark.parametrize("T", [50, 2_000])
def test_in_place(T):
    q, k, pos, freq, qw, kw, dq, dk = _inputs(T, 4, 2, 64)
    outs = nopfs.norm_rotate(q, k, pos, freq, qw, kw)
    grads = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw)
    a, b = dq.clone(), dk.clone()
    got = nopfs.norm_rotate_grad(a, b, q, k, pos, freq, qw, kw, dq=a, dk=b)
    assert got[0] is a and all(torch.equal(x, y) for x, y in zip(got, grads))
    nopfs.norm_rotate(q, k, pos, freq, qw, kw, q_out=q, k_out=k)
    assert torch.equal(q, outs[0]) and torch.equal(k, outs[1])


def test_scores_go_by_distance():
    """Rotated by positions that all lie 1,000 further on, products of queries and
    keys are the same: 4 u of |q||k| for their roundings, and the angles'."""
    q, k, pos, freq, qw, kw, *_ = _inputs(30, 2, 2, 64, F32, F32, padding=False)
    a, b = nopfs.norm_rotate(q, k, pos, freq, qw, kw)
    c, d = nopfs.norm_rotate(q, k, pos + 1_000, freq, qw, kw)
    s, t = (torch.einsum("thw,uhw->htu", x.double().cpu(), y.double().cpu()) for x, y in ((a, b), (c, d)))
    size = torch.einsum("thw,uhw->htu", a.abs().double().cpu(), b.abs().double().cpu())
    assert bool(((s - t).abs() <= 4 * (6 + 2 * math.pi + 40) * 2.0**-24 * 2 * size).all())


def test_gradient_against_differences():
    q, k, pos, freq, qw, kw, dq, dk = _inputs(9, 2, 1, 24, F32, F32, R=16)
    grads = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw)
    g = torch.Generator().manual_seed(5)
    args = [q, k, qw, kw]
    moves = [torch.randn(x.shape, generator=g).cuda() for x in args]

    def f(step):
        a, b, c, d = (x + step * m for x, m in zip(args, moves))
        o, p = nopfs.norm_rotate(a, b, pos, freq, c, d)
        return float((o.double() * dq.double()).sum() + (p.double() * dk.double()).sum())

    step = 2.0**-7
    diff = (8 * (f(step) - f(-step)) - (f(2 * step) - f(-2 * step))) / (12 * step)
    want = sum(float((a.double() * m.double()).sum()) for a, m in zip(grads, moves))
    # values are off by about 30 E of theirs, 18 of them over 12 steps; the formula's own
    # error is of the order of step^4 times the sum
    size = sum(float((x.abs() * 3).sum()) for x in (dq, dk))
    assert abs(diff - want) <= size * (2 * 30 * 2.0**-24 / step + 30 * step**4)


def test_refusals():
    q, k, pos, freq, qw, kw, dq, dk = _inputs(6, 2, 1, 16)
    for bad in (lambda: nopfs.norm_rotate(q, k.half(), pos, freq), lambda: nopfs.norm_rotate(q, k[:5], pos, freq),
                lambda: nopfs.norm_rotate(q, k, pos.long(), freq), lambda: nopfs.norm_rotate(q, k, pos[:5], freq),
                lambda: nopfs.norm_rotate(q, k, pos, freq.float()),
                lambda: nopfs.norm_rotate(q, k, pos, freq, qw, kw.half()),
                lambda: nopfs.norm_rotate(q, k, pos, freq, qw[:8], kw),
                lambda: nopfs.norm_rotate(q, k, pos, freq, q_out=q[:, :1]),
                lambda: nopfs.norm_rotate_grad(dq[:, :1], dk, q, k, pos, freq)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        nopfs.norm_rotate(q.cpu(), k, pos, freq)
    for bad in (lambda: nopfs.norm_rotate(q, k, pos, _freq(24)), lambda: nopfs.norm_rotate(q, k, pos, _freq(12)),
                lambda: nopfs.norm_rotate(q, k, pos, freq, eps=0.0),
                lambda: nopfs.norm_rotate(q[..., :12], k[..., :12], pos),
                lambda: nopfs.norm_rotate(q[:, :1].expand(6, 2, 16), k, pos, freq)):
        with pytest.raises(nopfs.NopfsError):
            bad()


def test_far_offsets():
    """Tokens whose elements pass 2^31 and their bytes 2^32."""
    T, stride = 40_000, 2**17
    q0, k0, pos, freq, qw, kw, dq0, dk0 = _inputs(T, 2, 2, 16)
    wide = torch.empty(T * stride, dtype=BF, device="cuda")
    views = [torch.as_strided(wide, (T, 2, 16), (stride, 16, 1), 32 * i) for i in range(8)]
    for view, x in zip(views, (q0, k0, dq0, dk0)):
        view.copy_(x)
    q, k, dq, dk, *outs = views
    want = nopfs.norm_rotate(q0, k0, pos, freq, qw, kw)
    nopfs.norm_rotate(q, k, pos, freq, qw, kw, q_out=outs[0], k_out=outs[1])
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    want = nopfs.norm_rotate_grad(dq0, dk0, q0, k0, pos, freq, qw, kw)
    got = nopfs.norm_rotate_grad(dq, dk, q, k, pos, freq, qw, kw, dq=outs[2], dk=outs[3])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_more_workgroups_than_one_launch_dimension_holds():
    T = 4 * 2**20 + 77  # four tokens a workgroup
    x = torch.randn((T, 2, 8), device="cuda").to(BF)
    pos = (torch.arange(T, device="cuda") % 1_000 - 1).int()
    q, k = nopfs.norm_rotate(x[:, :1], x[:, 1:], pos, _freq(8))
    half = T // 2 // 4 * 4
    for a, b in ((0, half), (half, T)):
        want = nopfs.norm_rotate(x[a:b, :1], x[a:b, 1:], pos[a:b], _freq(8))
        assert torch.equal(q[a:b], want[0]) and torch.equal(k[a:b], want[1])
