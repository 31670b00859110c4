"""nopfs_packed_attention and its gradient against 64 bits, within the bounds
that step_ref derives: sample lengths around the tiles' edges, of zero and one,
rows of no sample, head groups, widths that are no power of two, both types,
strided inputs and outputs, infinities and NaN where nothing may look, large
scores, and the gradient against differences of the forward pass."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import step_ref  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _starts(lengths):
    out = [0]
    for x in lengths:
        out.append(out[-1] + x)
    return out


def _inputs(lengths, tail, heads, kv_heads, width, dtype, seed, spread=1.0):
    """q, k, v as slices of one projection, and the gradient of o."""
    g = torch.Generator().manual_seed(seed)
    T = sum(lengths) + tail
    x = (torch.randn((T, heads + 2 * kv_heads, width), generator=g) * spread).to(dtype).cuda()
    do = torch.randn((T, heads, width), generator=g).to(dtype).cuda()
    return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], do


def _close(name, got, val, err):
    """Not-a-number fails, and -inf (rows of no sample) has to be equal."""
    got = got.detach().cpu().double()
    inf = torch.isinf(val)
    assert torch.equal(got[inf], val[inf]), name
    diff = (got - val)[~inf].abs()
    bad = ~(diff <= err[~inf])
    assert not bad.any(), (name, float(diff[bad].max()), int(bad.sum()), tuple(got.shape))


def _run_and_check(q, k, v, do, start, scale=None):
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, st, scale=scale)
    dq, dk, dv = nopfs.packed_attention_grad(do, q, k, v, o, lse, st, scale=scale)
    sc = q.shape[2] ** -0.5 if scale is None else scale
    val, err = step_ref.attention(q, k, v, start, sc, do)
    for name, t in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        _close(name, t, val[name], err[name])
    return o, lse, dq, dk, dv


EDGES = [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 257]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("width", [64, 128])
def test_lengths_around_the_tiles(dtype, width):
    lengths = EDGES + [0, 1, 0, 0, 300]
    q, k, v, do = _inputs(lengths, 0, 2, 1, width, dtype, width)
    _run_and_check(q, k, v, do, _starts(lengths))


@pytest.mark.parametrize("length", EDGES + [640, 1_111])
def test_one_sample(length):
    q, k, v, do = _inputs([length], 0, 2, 2, 64, BF, length)
    _run_and_check(q, k, v, do, [0, length])


@pytest.mark.parametrize("lengths", [[640], [1_111], [2_050, 33], [1_025, 0]])
@pytest.mark.parametrize("width", [32, 80, 128])
def test_few_long_samples(lengths, width):
    """Few workgroups: all four waves share 32 queries."""
    q, k, v, do = _inputs(lengths, 2, 2, 1, width, FP, sum(lengths))
    _run_and_check(q, k, v, do, _starts(lengths))


@pytest.mark.parametrize("lengths,tail,heads,kv_heads,width,dtype", [
    ([3_200], 0, 1, 1, 32, BF),
    ([3_137, 1], 70, 2, 1, 64, FP),
    ([1, 4_700, 0, 5], 3, 3, 1, 80, BF),
    ([2_600, 2_222], 0, 6, 2, 128, FP),
    ([5_000], 33, 6, 6, 64, BF),
    ([4_900, 63, 0, 1, 1_500, 128, 65, 2, 900, 300, 31, 1_800], 110, 2, 2, 128, BF),
])
def test_parts_of_the_keys(lengths, tail, heads, kv_heads, width, dtype):
    """Few, long samples: several workgroups share a query tile's keys, and
    tiles of few keys leave some of them without any."""
    q, k, v, do = _inputs(lengths, tail, heads, kv_heads, width, dtype, sum(lengths))
    start = _starts(lengths)
    o, lse, dq, dk, dv = _run_and_check(q, k, v, do, start)
    again = torch.tensor(start, dtype=torch.int32, device="cuda")
    o2, lse2 = nopfs.packed_attention(q, k, v, again)
    for a, b in zip((o, lse, dq, dk, dv), (o2, lse2, *nopfs.packed_attention_grad(do, q, k, v, o2, lse2, again))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (6, 2), (8, 1), (5, 5), (16, 4)])
def test_head_groups(heads, kv_heads):
    lengths = [70, 1, 200]
    q, k, v, do = _inputs(lengths, 3, heads, kv_heads, 32, BF, heads)
    _run_and_check(q, k, v, do, _starts(lengths))


@pytest.mark.parametrize("width", [8, 16, 24, 40, 48, 72, 80, 96, 104, 112, 120])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_widths(width, dtype):
    lengths = [150, 37]
    q, k, v, do = _inputs(lengths, 0, 2, 1, width, dtype, width)
    _run_and_check(q, k, v, do, _starts(lengths))


@pytest.mark.parametrize("n", [1, 63, 64, 65, 200, 5_000])
def test_many_short_samples(n):
    g = torch.Generator().manual_seed(n)
    lengths = torch.randint(0, 4, (n,), generator=g).tolist()
    q, k, v, do = _inputs(lengths, 5, 1, 1, 16, BF, n)
    _run_and_check(q, k, v, do, _starts(lengths))


@pytest.mark.parametrize("n", [2**20 + 70, 2**23 + 9])
def test_more_workgroups_than_one_launch_dimension_holds(n):
    """Samples of no token, and a few of some: two heads make 2^24 workgroups of
    256 threads."""
    at = {5: 40, 2**20 - 3: 1, 2**20 + 60: 130, n - 1: 33}
    lengths = torch.zeros(n, dtype=torch.int64)
    for i, x in at.items():
        lengths[i] = x
    start = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).to(torch.int32).cuda()
    q, k, v, do = _inputs(list(at.values()), 3, 2, 1, 64, BF, 13)
    o, lse = nopfs.packed_attention(q, k, v, start)
    grads = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
    val, err = step_ref.attention(q, k, v, _starts(list(at.values())), 64**-0.5, do)
    for name, t in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        _close(name, t, val[name], err[name])


@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("kv_heads", [200, 520])
def test_many_heads(width, kv_heads):
    """Enough workgroups for one split: 128 columns each."""
    lengths = [3, 129, 0, 100]
    q, k, v, do = _inputs(lengths, 7, 520, 520, width, BF, 11)
    if kv_heads < 520:
        q, do, k, v = q[:, :400], do[:, :400], k[:, :200], v[:, :200]
    _run_and_check(q, k, v, do, _starts(lengths))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (18, 6)])
@pytest.mark.parametrize("width", [64, 128])
def test_order_by_cost(heads, kv_heads, width):
    """Enough rows and samples for the tiles to be ordered."""
    lengths = [700, 1, 0, 64, 1_500, 130, 128, 900, 0, 33, 620, 200]
    q, k, v, do = _inputs(lengths, 90, heads, kv_heads, width, BF, 12)
    _run_and_check(q, k, v, do, _starts(lengths))


def test_no_sample_and_no_row():
    q, k, v, do = _inputs([], 150, 2, 1, 64, BF, 1)
    for start in ([0], [0, 0, 0]):
        o, lse, dq, dk, dv = _run_and_check(q, k, v, do, start)
        assert not o.any() and not dq.any() and not dk.any() and not dv.any()
        assert bool((lse == -math.inf).all())
    e = q[:0]
    o, lse = nopfs.packed_attention(e, k[:0], v[:0], torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert o.shape == (0, 2, 64) and lse.shape == (2, 0)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_rows_of_no_sample_hold_anything(bad):
    lengths, tail = [100, 29], 300
    q, k, v, do = _inputs(lengths, tail, 4, 2, 64, BF, 3)
    clean = _run_and_check(q, k, v, do, _starts(lengths))
    for t in (q, k, v, do):
        t[sum(lengths):] = bad
    for a, b in zip(clean, _run_and_check(q, k, v, do, _starts(lengths))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_another_sample_holds_anything(bad):
    lengths = [70, 45, 130]
    start = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")
    q, k, v, do = _inputs(lengths, 0, 2, 1, 128, BF, 4)

    def results():
        o, lse = nopfs.packed_attention(q, k, v, start)
        return (o, lse.t(), *nopfs.packed_attention_grad(do, q, k, v, o, lse, start))

    clean = results()
    for t in (q, k, v, do):
        t[70:115] = bad
    for a, b in zip(clean, results()):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[115:], b[115:])


@pytest.mark.parametrize("spread", [0.0, 1e-3, 8.0])
def test_flat_and_steep_rows(spread):
    lengths = [333]
    q, k, v, do = _inputs(lengths, 0, 2, 2, 64, BF, 5, spread)
    _run_and_check(q, k, v, do, _starts(lengths))
    _run_and_check(q, k, v, do, _starts(lengths), scale=0.37)


@pytest.mark.parametrize("scale", [2.0**-60, 2.0**-30, 3.0])
def test_small_and_large_scales(scale):
    q, k, v, do = _inputs([200, 1, 70], 0, 2, 1, 64, BF, 14)
    _run_and_check(q, k, v, do, [0, 200, 201, 271], scale=scale)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("lengths,heads", [([2] * 40 + [1, 0] + [3] * 20, 3), ([2, 3, 2, 4], 300)])
@pytest.mark.parametrize("width", [32, 80, 128])
def test_short_samples_do_not_feel_the_rounding_of_o(lengths, heads, width, dtype):
    """dS and dq are rounded to the inputs' type, of unit u (half the spacing over
    the least value that has it): each rounding is off by u / sqrt(3) of its value
    at most in the mean square, all of them independent. delta from the rounded o
    would add to all dS of a row together, where dP - delta is small."""
    q, k, v, do = _inputs(lengths, 0, heads, heads, width, dtype, 17)
    start = _starts(lengths)
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, st)
    dq = nopfs.packed_attention_grad(do, q, k, v, o, lse, st)[0]
    u, scale = (2.0**-8 if dtype == BF else 2.0**-11), width**-0.5
    off = allowed = 0.0
    for a, b in zip(start, start[1:]):
        if a == b:
            continue
        qi, ki, vi, di = (x[a:b].double().transpose(0, 1).contiguous() for x in (q, k, v, do))
        seen = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").tril()
        s = torch.where(seen, qi @ ki.transpose(1, 2).contiguous() * scale, -math.inf)
        p, dp = torch.softmax(s, 2), di @ vi.transpose(1, 2).contiguous()
        ds = p * (dp - (p * dp).sum(2, keepdim=True))
        want = ds @ ki * scale
        off += float(((dq[a:b].double().transpose(0, 1) - want) ** 2).sum())
        allowed += float((ds**2 @ ki**2).sum() * scale**2 + (want**2).sum()) * u**2 / 3
    assert off <= allowed


def test_scores_that_grow_along_the_keys():
    """The running maximum moves in every tile."""
    T = 700
    q = torch.ones((T, 1, 64), dtype=BF, device="cuda")
    k = (torch.arange(T, device="cuda")[:, None, None] / 8.0).expand(T, 1, 64).to(BF).contiguous()
    _, _, v, do = _inputs([T], 0, 1, 1, 64, BF, 6)
    v = v.contiguous()
    for kk in (k, k.flip(0).contiguous()):
        _run_and_check(q, kk, v, do, [0, T])


def test_outputs_into_slices_and_layouts():
    lengths = [90, 140]
    start = _starts(lengths)
    q, k, v, do = _inputs(lengths, 6, 4, 2, 64, BF, 7)
    want = _run_and_check(q, k, v, do, start)
    T = q.shape[0]
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    # heads first in memory, one array of gradients, an output wider than its head
    qh, kh, vh, dh = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v, do))
    wide = torch.full((T, 4, 72), 5.0, dtype=BF, device="cuda")
    o, lse = nopfs.packed_attention(qh, kh, vh, st, o=wide[:, :, :64])
    grads = torch.full((T, 8, 64), 5.0, dtype=BF, device="cuda")
    nopfs.packed_attention_grad(dh, qh, kh, vh, o, lse, st, dq=grads[:, :4], dk=grads[:, 4:6],
                                dv=grads[:, 6:])
    for a, b in zip(want, (o, lse, grads[:, :4], grads[:, 4:6], grads[:, 6:])):
        assert torch.equal(a, b)
    assert bool((wide[:, :, 64:] == 5.0).all())


@pytest.mark.parametrize("token,head", [(2**23, 72), (72, 2**31 + 8)])
def test_offsets_past_32_bits(token, head):
    """Rows or heads so far apart that byte offsets pass 2^32."""
    lengths = [250, 7, 40]
    q, k, v, do = _inputs(lengths, 5, 2, 1, 64, BF, 15)
    start = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, start)
    grads = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
    T = q.shape[0]

    def far(x):
        size = (T - 1) * token + (x.shape[1] - 1) * head + 64
        y = torch.empty(size, dtype=BF, device="cuda").as_strided(x.shape, (token, head, 1))
        return y.copy_(x)

    fq, fk, fv, fdo, fo = far(q), far(k), far(v), far(do), far(torch.zeros_like(o))
    out, stat = nopfs.packed_attention(fq, fk, fv, start, o=fo)
    assert torch.equal(out, o) and torch.equal(stat, lse)
    far_grads = [far(torch.zeros_like(g)) for g in grads]
    nopfs.packed_attention_grad(fdo, fq, fk, fv, fo, stat, start,
                                **dict(zip(("dq", "dk", "dv"), far_grads)))
    for a, b in zip(far_grads, grads):
        assert torch.equal(a, b)


def test_same_bits_again_and_on_another_stream():
    lengths = [500, 3, 260]
    q, k, v, do = _inputs(lengths, 9, 6, 2, 128, FP, 8)
    start = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")

    def results(stream=None):
        o, lse = nopfs.packed_attention(q, k, v, start, stream=stream)
        return (o, lse, *nopfs.packed_attention_grad(do, q, k, v, o, lse, start, stream=stream))

    want = results()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for got in (results(), results(s)):
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


def test_in_a_graph():
    lengths = [200, 77]
    q, k, v, do = _inputs(lengths, 0, 2, 1, 64, BF, 9)
    start = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, start)
    grads = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
    s = torch.cuda.Stream()
    nopfs.packed_attention_grad(do, q, k, v, o, lse, start, stream=s)  # its scratch
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go, gl = nopfs.packed_attention(q, k, v, start, stream=s)
        gg = nopfs.packed_attention_grad(do, q, k, v, go, gl, start, stream=s)
    for i in range(3):
        for t in (go, gl, *gg):
            t.fill_(3.0)
        q.mul_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        o, lse = nopfs.packed_attention(q, k, v, start)
        grads = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
        torch.cuda.synchronize()
        for a, b in zip((o, lse, *grads), (go, gl, *gg)):
            assert torch.equal(a, b), i


def test_parts_in_a_graph():
    """Parts of the keys and of the queries: partial sums in the stream's scratch."""
    lengths = [3_300, 900]
    q, k, v, do = _inputs(lengths, 20, 2, 1, 64, BF, 16)
    start = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, lse = nopfs.packed_attention(q, k, v, start, stream=s)  # the stream's scratch
    nopfs.packed_attention_grad(do, q, k, v, o, lse, start, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go, gl = nopfs.packed_attention(q, k, v, start, stream=s)
        gg = nopfs.packed_attention_grad(do, q, k, v, go, gl, start, stream=s)
    for i in range(3):
        for t in (go, gl, *gg):
            t.fill_(3.0)
        q.mul_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        o, lse = nopfs.packed_attention(q, k, v, start)
        grads = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
        torch.cuda.synchronize()
        for a, b in zip((o, lse, *grads), (go, gl, *gg)):
            assert torch.equal(a, b), i


def test_gradient_against_differences():
    """f(x) = sum o * do with do held; o rounded to 11 bits limits a difference
    of step h = 1/4 to about 2^-11 sum |o do| / h plus the third-order term, so
    the mean of many directions is compared: directional derivative along a
    random sign vector."""
    lengths = [60, 75]
    q, k, v, do = (t.contiguous() for t in _inputs(lengths, 0, 2, 1, 64, FP, 10, 0.5))
    start = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, start)
    grads = nopfs.packed_attention_grad(do, q, k, v, o, lse, start)
    for i, x in enumerate((q, k, v)):
        g = torch.Generator().manual_seed(i)
        side = (torch.randint(0, 2, x.shape, generator=g) * 2 - 1).to(FP).cuda()
        h = 2.0**-6
        f = []
        for sign in (1, -1):
            args = [q, k, v]
            args[i] = x + sign * h * side
            step = (args[i].double() - x.double())  # as rounded
            ob = nopfs.packed_attention(*args, start)[0]
            f.append(((ob.double() * do.double()).sum(), step))
        moved = f[0][1] - f[1][1]
        want = (grads[i].double() * moved).sum()
        noise = 2 * 2.0**-11 * float((o.double() * do.double()).norm())  # independent roundings
        scale = float((grads[i].double().abs() * moved.abs()).sum())
        assert abs(float(f[0][0] - f[1][0] - want)) <= 6 * noise + 2e-3 * scale
