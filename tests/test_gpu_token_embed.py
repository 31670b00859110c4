"""nopfs_token_embed and its gradient against 64 bits within layer_ref's bounds: the
types, widths and strides of any alignment, ids and slots out of range, one token
and many, one name for all of them, and the gradient against differences."""
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


def _ids(T, V, seed, skew=True, dtype=torch.int32):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(T, generator=g, dtype=torch.float64)
    ids = ((V + 1.0) ** u - 1 if skew else u * V).long().clamp(0, V - 1)
    return ids.to(dtype).cuda()


def _check(T, V, D, wd=BF, dt=BF, scale=1.5, seed=0, skew=True, ids=None, slot=None, idt=torch.int32):
    g = torch.Generator().manual_seed(seed + 1)
    w = torch.randn((V, D), generator=g).to(wd).cuda()
    if ids is None:
        ids = _ids(T, V, seed, skew, idt)
    rows = len(ids) if slot is None else len(slot)
    d = torch.randn((rows, D), generator=g).to(dt).cuda()
    out = nopfs.token_embed(w, ids, scale, slot=slot, dtype=dt)
    assert out.dtype is dt
    close("out", out, *layer_ref.embed(w, ids, slot, scale, dt))
    dw = nopfs.token_embed_grad(d, ids, V, scale, slot=slot, dtype=wd)
    assert dw.dtype is wd
    close("dweight", dw, *layer_ref.embed_grad(d, ids, slot, V, scale, wd))
    assert torch.equal(dw, nopfs.token_embed_grad(d, ids, V, scale, slot=slot, dtype=wd))
    return w, ids, d, out, dw


@pytest.mark.parametrize("wd", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
def test_types(wd, dt):
    _check(777, 300, 72, wd, dt)


@pytest.mark.parametrize("D", [1, 2, 7, 8, 9, 63, 64, 250, 513, 1_024, 2_047, 2_056, 5_001])
def test_widths(D):
    _check(301, 97, D, F32, BF, seed=D)
    _check(64, 33, D, BF, BF, seed=D)


@pytest.mark.parametrize("T", [0, 1, 2, 31, 32, 33, 63, 64, 65, 1_023, 1_024, 1_025, 4_096, 4_097, 9_001])
def test_tokens(T):
    _check(T, 1_000, 24, seed=T)
    _check(T, 3, 16, F32, F32, seed=T)


@pytest.mark.parametrize("V", [1, 2, 255, 256, 1_023, 1_024, 1_025, 32_768, 70_001, 1_048_577])
def test_rows(V):
    _check(2_500, V, 8, seed=V, skew=V % 2 == 0)


@pytest.mark.parametrize("T,V,D", [(5_000, 1, 40), (20_000, 2, 64), (6_000, 50_000, 24), (3_000, 7, 2_048)])
def test_one_name_for_all(T, V, D):
    """Runs that go over many workgroups."""
    ids = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    _check(T, V, D, F32, BF, ids=ids)
    ids[: T // 3] = 0
    ids[T // 2] = -1
    _check(T, V, D, BF, FP, ids=ids)


def test_large_batch():
    _check(140_003, 60_000, 4, F32, BF, skew=True)


@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_padding(idt):
    ids = _ids(500, 90, 3, dtype=idt)
    big = 2**31 - 1 if idt is torch.int32 else 2**40
    for i, x in ((0, -1), (7, 90), (8, big), (9, -big), (499, -1)):
        ids[i] = x
    _, _, d, out, dw = _check(500, 90, 40, ids=ids)
    assert bool((out[[0, 7, 8, 9, 499]] == 0).all())
    d[[0, 7, 8, 9, 499]] = math.nan  # is not read
    assert torch.equal(nopfs.token_embed_grad(d, ids, 90, 1.5), dw)
    none = torch.full((33,), -1, dtype=idt, device="cuda")
    _check(33, 90, 40, ids=none)


@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_slots(idt):
    ids = _ids(640, 90, 4, dtype=idt)
    g = torch.Generator().manual_seed(5)
    slot = torch.randint(0, 640, (1_500,), generator=g)
    for i, x in ((0, -1), (3, 640), (4, 2**40), (5, -(2**40)), (1_499, -1)):
        slot[i] = x
    ids[int(slot[10])] = -7
    _check(0, 90, 56, ids=ids, slot=slot.cuda())
    _check(0, 90, 56, ids=ids, slot=slot[:0].cuda())
    empty = ids[:0]
    out = nopfs.token_embed(torch.ones((4, 8), device="cuda"), empty, slot=slot.cuda())
    assert bool((out == 0).all())


@pytest.mark.parametrize("ws,shift,os", [(40, 0, 40), (43, 1, 41), (64, 3, 56)])
@pytest.mark.parametrize("dt", [BF, F32], ids=NAMES.get)
def test_strides(ws, shift, os, dt):
    """Rows of wider arrays from any element on; what lies between them stays."""
    V, D, T = 50, 40, 130
    w0, ids, d0, out0, dw0 = _check(T, V, D, dt, dt)
    wide = torch.full((V * ws + 8,), math.nan, dtype=dt, device="cuda")
    w = torch.as_strided(wide, (V, D), (ws, 1), shift)
    w.copy_(w0)
    flat = torch.full((T * os + 8,), 9.0, dtype=dt, device="cuda")
    out = torch.as_strided(flat, (T, D), (os, 1), shift)
    assert nopfs.token_embed(w, ids, 1.5, out=out) is out and torch.equal(out, out0)
    held = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(held, (T, D), (os, 1), shift).fill_(False)
    assert bool((flat[held] == 9.0).all())
    d = torch.as_strided(flat, (T, D), (os, 1), shift)
    d.copy_(d0)
    wide.fill_(7.0)
    assert torch.equal(nopfs.token_embed_grad(d, ids, V, 1.5, dweight=w), dw0)
    held = torch.ones_like(wide, dtype=torch.bool)
    torch.as_strided(held, (V, D), (ws, 1), shift).fill_(False)
    assert bool((wide[held] == 7.0).all())


def test_infinities_stay_in_their_rows():
    w = torch.randn((9, 16), device="cuda")
    w[3] = math.inf
    w[4] = math.nan
    ids = torch.tensor([0, 3, 4, 8, 3], dtype=torch.int32, device="cuda")
    out = nopfs.token_embed(w, ids, 2.0)
    assert bool(torch.isinf(out[[1, 4]]).all()) and bool(torch.isnan(out[2]).all())
    assert torch.equal(out[[0, 3]], 2.0 * w[[0, 8]])
    dw = nopfs.token_embed_grad(out, ids, 9)
    assert bool(torch.isinf(dw[3]).all()) and bool(torch.isnan(dw[4]).all())
    assert bool(torch.isfinite(dw[[0, 1, 2, 5, 6, 7, 8]]).all())


def test_far_rows():
    """Rows whose elements pass 2^31 and their bytes 2^32."""
    V, D = 600_000, 4_096
    w = torch.empty((V, D), dtype=BF, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 1, 524_288, 524_287, -1], dtype=torch.int64, device="cuda")
    w[ids[:5]] = torch.arange(5, device="cuda")[:, None].to(BF) + 1
    out = nopfs.token_embed(w, ids, 0.5, dtype=F32)
    assert torch.equal(out[:5], 0.5 * w[ids[:5]].float()) and bool((out[5] == 0).all())
    d = torch.arange(6 * D, device="cuda").view(6, D).remainder(113).to(BF)
    nopfs.token_embed_grad(d, ids, V, 2.0, dweight=w)
    want = torch.zeros((3, D), device="cuda")
    for row, t in enumerate((1, 4, 3)):
        want[row] = 2.0 * d[t].float()
    assert torch.equal(w[[0, 524_287, 524_288]].float(), want.to(BF).float())
    assert torch.equal(w[V - 1], (2.0 * (d[0].float() + d[2].float())).to(BF))
    assert int(torch.count_nonzero(w.view(-1, 1_000, D).abs().amax((1, 2)))) == 3


def test_gradient_against_differences():
    """The sum of out * d is linear in weight: its difference over any step is the
    gradient times that step."""
    g = torch.Generator().manual_seed(11)
    w = torch.randn((40, 24), generator=g).cuda()
    ids = _ids(200, 40, 12)
    d = torch.randn((200, 24), generator=g).cuda()
    move = torch.randn((40, 24), generator=g).cuda()
    dw = nopfs.token_embed_grad(d, ids, 40, 1.25)
    f = lambda x: (nopfs.token_embed(x, ids, 1.25).double() * d.double()).sum()  # noqa: E731
    diff = float(f(w + move) - f(w - move)) / 2
    want = float((dw.double() * move.double()).sum())
    # 2 E of each product of the sums' roundings, and (200 + 1) E of the gradient's
    bound = 2.0**-24 * float((3 * (w.abs() + move.abs())[ids.long()] * 1.25 * d.abs()).sum()
                             + 201 * 1.25 * (move.abs()[ids.long()] * d.abs()).sum())
    assert abs(diff - want) <= bound


def test_refusals():
    w, ids = torch.zeros((4, 8), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (lambda: nopfs.token_embed(w.double(), ids), lambda: nopfs.token_embed(w, ids.short()),
                lambda: nopfs.token_embed(w, ids, dtype=torch.int32), lambda: nopfs.token_embed(w, ids[None]),
                lambda: nopfs.token_embed(w, ids, slot=ids),
                lambda: nopfs.token_embed(w, ids, out=torch.zeros((2, 8), device="cuda")),
                lambda: nopfs.token_embed(w, ids, dtype=BF, out=torch.zeros((3, 8), device="cuda")),
                lambda: nopfs.token_embed(w, torch.zeros(6, dtype=torch.int32, device="cuda")[::2]),
                lambda: nopfs.token_embed_grad(w, ids, 4), lambda: nopfs.token_embed_grad(w[:3], ids, 0),
                lambda: nopfs.token_embed_grad(w[:3], ids, 4, dweight=w[:3])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        nopfs.token_embed(w, ids.cpu())
    for scale in (math.inf, math.nan):
        with pytest.raises(nopfs.NopfsError):
            nopfs.token_embed(w, ids, scale)


@pytest.mark.parametrize("T", [6_143, 6_144, 6_145])
@pytest.mark.parametrize("V", [200, 70_000, 262_144, 262_145])
def test_both_sides_of_the_small_sort(T, V):
    _check(T, V, 5, F32, F32, seed=T + V)


@pytest.mark.parametrize("V", [300, 40_000])
def test_tokens_of_a_name_in_order(V):
    """Sums are made in the order of the batch: of terms that differ by 2^30, the small
    ones count only behind the large one's opposite."""
    for T in (30, 5_000, 20_000):
        ids = torch.full((T,), V // 2, dtype=torch.int32, device="cuda")
        d = torch.zeros((T, 8), device="cuda")
        d[0], d[1], d[2], d[3] = 2.0**30, 1.0, -(2.0**30), 1.0
        dw = nopfs.token_embed_grad(d, ids, V)
        assert bool((dw[V // 2] == 1.0).all())


@pytest.mark.parametrize("T,V", [(0, 300_000), (3, 2_000_003), (7_000, 1_500_001), (130_000, 900_001)])
def test_many_more_rows_than_tokens(T, V):
    ids = _ids(T, V, 7, skew=False)
    d = torch.randn((T, 8), device="cuda")
    dw = torch.full((V, 8), math.nan, device="cuda")
    nopfs.token_embed_grad(d, ids, V, 1.0, dweight=dw)
    want = torch.zeros((V, 8), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), d.double())
    mag = torch.zeros((V, 8), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), d.double().abs())
    # at most 9 tokens a row here: 8 additions in 32 bits
    assert int(torch.bincount(ids, minlength=1).max()) <= 9
    assert bool(((dw.double() - want).abs() <= 9 * 2.0**-24 * mag).all())


def test_more_workgroups_than_one_launch_dimension_holds():
    """A row of more than 2,048 elements is a workgroup's: 2^20 of them and a few."""
    T, V, D = 2**20 + 37, 5, 2_056
    w = torch.randn((V, D), device="cuda").to(BF)
    ids = (torch.arange(T, device="cuda") % (V + 1) - 1).int()  # -1: padding
    out = nopfs.token_embed(w, ids)
    rows = torch.cat([torch.zeros((1, D), dtype=BF, device="cuda"), w])
    for a in range(0, T, 2**18):
        part = ids[a:a + 2**18].long() + 1
        assert torch.equal(out[a:a + 2**18], rows[part])
