"""nopfs_gated_scan and its gradient with gates at the ends of their type: a sample's
states forgotten (a = 0) or kept (a = 1) by a gate of the lowest or highest value or an
infinity, by samples one by one and by chunks, against 64 bits within layer_ref's bounds."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import layer_ref  # noqa: E402
from layer_ref import close  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
NAMES = {BF: "bf16", FP: "fp16", F32: "fp32"}
LENGTHS = {"single": [1] * 40, "pairs": [2] * 100 + [0, 1], "samples": [300, 0, 1, 17, 256],
           "one": [2_500]}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _inputs(lengths, C, dt, seed=0):
    g = torch.Generator().manual_seed(seed)
    T, n = sum(lengths), len(lengths)
    x = torch.randn((T, C), generator=g).to(dt)
    gate = (2.5 + 1.5 * torch.randn((T, C), generator=g)).to(dt)
    dh = torch.randn((T, C), generator=g).to(dt)
    h0, dlast = torch.randn((n, C), generator=g), torch.randn((n, C), generator=g)
    start = torch.tensor([0] + list(lengths)).cumsum(0).int()
    return x, gate, start, h0, dh, dlast, g


def _run(x, gate, start, h0, dh, dlast):
    x, gate, start, h0, dh, dlast = (t.cuda() for t in (x, gate, start, h0, dh, dlast))
    h, last, carry = nopfs.gated_scan(x, gate, start, h0)
    dx, dgate, dh0 = nopfs.gated_scan_grad(dh, x, gate, start, carry, h0, dlast)
    return dict(h=h, last=last, dx=dx, dgate=dgate, dh0=dh0)


def _ends(dt):
    top = torch.finfo(dt).max
    return [top, -top, math.inf, -math.inf, 0.75 * top, -0.75 * top, 0.7 * top, -0.7 * top]


@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("lengths", LENGTHS)
def test_some_gates(dt, lengths):
    """A tenth of the gates at the ends. In 64 bits those of 10^4 are the same: 0 and 1."""
    x, gate, start, h0, dh, dlast, g = _inputs(LENGTHS[lengths], 70, dt)
    ends = torch.tensor(_ends(dt), dtype=dt)
    there = torch.rand(gate.shape, generator=g) < 0.1
    gate[there] = ends[torch.randint(0, len(ends), (int(there.sum()),), generator=g)]
    got = _run(x, gate, start, h0, dh, dlast)
    val, err = layer_ref.scan(x, gate.float().clamp(-1e4, 1e4), start.tolist(), h0, dh, dlast)
    for name, t in got.items():
        close(name, t, val[name], err[name])


@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("end", range(8))
def test_every_gate(dt, lengths, end):
    """a = 0: h is x, whose gradient is dh and, at a sample's end, dlast. a = 1: h is h0,
    whose gradient is the sum of all. Nothing is rounded but h, dx and that sum."""
    x, gate, start, h0, dh, dlast, _ = _inputs(LENGTHS[lengths], 33, dt)
    gate.fill_(_ends(dt)[end])
    got = {name: t.cpu() for name, t in _run(x, gate, start, h0, dh, dlast).items()}
    assert not bool(got["dgate"].any())
    for s, (a, b) in enumerate(zip(start[:-1].tolist(), start[1:].tolist())):
        if a == b:
            assert torch.equal(got["last"][s], h0[s]) and torch.equal(got["dh0"][s], dlast[s])
        elif end % 2:
            assert torch.equal(got["h"][a:b], x[a:b]) and torch.equal(got["last"][s], x[b - 1].float())
            assert torch.equal(got["dx"][a:b - 1], dh[a:b - 1])
            assert torch.equal(got["dx"][b - 1], (dh[b - 1].float() + dlast[s]).to(dt))
            assert not bool(got["dh0"][s].any())
        else:
            assert torch.equal(got["h"][a:b], h0[s].to(dt).expand(b - a, -1))
            assert torch.equal(got["last"][s], h0[s])
            assert not bool(got["dx"][a:b].any())
            want = dh[a:b].double().sum(0) + dlast[s].double()
            size = dh[a:b].double().abs().sum(0) + dlast[s].double().abs()
            # b - a additions in 32 bits and a few of maps, each off by half a step of at most `size`
            assert bool(((got["dh0"][s].double() - want).abs() <= 1.01 * (b - a + 24) * 2.0**-24 * size).all())


@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("lengths", ["pairs", "samples"])
def test_nan_gates_stay(dt, lengths):
    """A gate that is NaN makes its channel NaN from there to the sample's end."""
    x, gate, start, h0, dh, dlast, _ = _inputs(LENGTHS[lengths], 20, dt)
    want = _run(x, gate, start, h0, dh, dlast)
    a, b = int(start[0]), int(start[1])
    t = (a + b) // 2
    gate[t, 7] = math.nan
    got = _run(x, gate, start, h0, dh, dlast)
    assert bool(torch.isnan(got["h"][t:b, 7]).all()) and bool(torch.isnan(got["last"][0, 7]))
    assert bool(torch.isnan(got["dx"][a:t + 1, 7]).all()) and bool(torch.isnan(got["dh0"][0, 7]))
    others = torch.ones(len(x), 20, dtype=torch.bool)
    others[a:b, 7] = False
    for name in ("h", "dx", "dgate"):
        assert torch.equal(got[name][others], want[name][others])


@pytest.mark.parametrize("dt", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("n", [300, 1_100])
def test_shares_to_32_bits(dt, n):
    """The smaller of a and 1 - a, of gates of any type: 6 E of it (the exponential 3,
    the sum, the reciprocal and the product 1 each), E for the product with the state or
    the input; 0 below 2^-126. `last` of single tokens, by themselves and by chunks."""
    g = torch.Generator().manual_seed(n)
    gate = (172 * torch.rand((n, 40), generator=g) - 86).to(dt)
    forgets = gate < 0
    y = torch.randn((n, 40), generator=g).to(dt)
    x, h0 = torch.where(forgets, 0, y), torch.where(forgets, y, 0).float()
    start = torch.arange(n + 1, dtype=torch.int32)
    last = nopfs.gated_scan(*(t.cuda() for t in (x, gate, start, h0)))[1]
    val = torch.sigmoid(-gate.double().abs()) * y.double()
    close("last", last, val, 8 * 2.0**-24 * val.abs() + 2.0**-126 * y.double().abs() + 2.0**-149)
