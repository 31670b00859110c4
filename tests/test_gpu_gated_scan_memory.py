"""nopfs_gated_scan and its gradient where gates keep a state over thousands of tokens,
against 64 bits. A state that is multiplied by a rounded 1 - k at every token is off by up
to 2^-25 / k; the bounds here are far below that.

With E = 2^-24, k the smaller share (here 1 - a, at most 2^-8), M_t the magnitudes
M_t = a M_(t-1) + k |x_t|, X the largest |x|:
  - k is off by 8 E of it, which moves the state by 8 E k |x - h| a token;
  - in a wave's 16 tokens, the part B of the state that they bring is at most 16 k X; a
    step rounds the difference (E k (X + B)) and the sum (E B): 8.5 k X E a token; the
    parts of a chunk's 8 waves, added up, round twice per wave: 2 * 4.5 k X E a token, and
    as much for the part K M that they take away: in all 8 + 2 * 20, below 50 k (X + M) E;
  - a chunk of 128 tokens adds its part to the state: E M a chunk, E M / 128 a token, and
    E (128 k (X + M)) a chunk, within the 50 above.
All of this decays with a from token to token. Within its own chunk a token's state has
been rounded at most 8 times by the waves before and 16 by steps, and a chunk may be
begun: 26 E M that do not add up.
Backwards, R_t = a (dh_t + R_(t+1)) of magnitude N, D the largest |dh|: a step rounds the
sum, the small share and the large one, of parts of at most 16 D in a wave (3 * 8.5 D E a
token) and 128 D in a chunk (2 * 4.5 D E a token), in all below 50 (D + k N) E with what K
and k bring; a chunk E N. Within the chunk 3 * 16 + 8 + 2 roundings of N."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from layer_ref import TINY, UNIT, E, close  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
F64 = torch.float64
NAMES = {BF: "bf16", FP: "fp16", F32: "fp32"}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _reference(x, gate, h0, dh, dlast):
    dt = x.dtype
    x, gate, h0, dh, dlast = (t.to(F64) for t in (x, gate, h0, dh, dlast))
    T, C = x.shape
    a, k = torch.sigmoid(gate), torch.sigmoid(-gate)
    assert bool((k <= 2.0**-8).all())
    u, tiny = UNIT[dt], TINY[dt]
    X, D = x.abs().amax(0), dh.abs().amax(0)
    val, err = {}, {}
    h, e, M = h0.clone(), torch.zeros(C, dtype=F64), h0.abs()
    before, ebefore = torch.empty((T, C), dtype=F64), torch.empty((T, C), dtype=F64)
    hs, es = torch.empty((T, C), dtype=F64), torch.empty((T, C), dtype=F64)
    for t in range(T):
        before[t], ebefore[t] = h, e + 26 * E * M
        e = a[t] * e + 50 * E * k[t] * (X + M) + E / 128 * M
        h = a[t] * h + k[t] * x[t]
        M = a[t] * M + k[t] * x[t].abs()
        hs[t], es[t] = h, e + 26 * E * M
    val["h"], err["h"] = hs, es + u * hs.abs() + tiny
    val["last"], err["last"] = h[None], es[-1:]
    R, e, N = dlast.clone(), torch.zeros(C, dtype=F64), dlast.abs()
    Gs, eG, NG = (torch.empty((T, C), dtype=F64) for _ in range(3))
    for t in range(T - 1, -1, -1):
        Gs[t], NG[t] = dh[t] + R, dh[t].abs() + N
        eG[t] = e + 58 * E * NG[t]
        e = a[t] * e + 50 * E * (D + k[t] * N) + E / 128 * N
        R, N = a[t] * Gs[t], a[t] * NG[t]
    val["dh0"], err["dh0"] = R[None], (e + 58 * E * N)[None]
    val["dx"] = k * Gs
    err["dx"] = k * (eG + 9 * E * NG) + u * val["dx"].abs() + tiny
    diff = (before - x).abs()
    val["dgate"] = a * k * (before - x) * Gs
    err["dgate"] = (a * k * (diff * (eG + 18 * E * NG) + (ebefore + E * diff) * NG)
                    + u * val["dgate"].abs() + tiny)
    return val, err


@pytest.mark.parametrize("dt", [F32, FP, BF], ids=NAMES.get)
@pytest.mark.parametrize("kind", ["equal", "decay", "noise"])
def test_states_over_many_tokens(dt, kind):
    """Gates of 5.6 to 12.5, each channel's own at every token: memories of hundreds to
    hundreds of thousands of tokens, over 20,021."""
    T, C = 20_021, 36
    g = torch.Generator().manual_seed(3)
    gate = torch.linspace(5.6, 12.5, C).expand(T, C).to(dt)
    x = (1 + torch.randn((T, C), generator=g)) if kind == "noise" else torch.full((T, C), float(kind == "equal"))
    h0 = torch.zeros((1, C)) if kind == "equal" else 1.37 + torch.rand((1, C), generator=g)
    dh = torch.zeros((T, C)) if kind == "decay" else 0.5 + torch.randn((T, C), generator=g)
    dlast = 3 * torch.randn((1, C), generator=g)
    x, gate, dh = x.to(dt), gate.contiguous(), dh.to(dt)
    start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    X, Gt, H0, Dh, Dl = (t.cuda() for t in (x, gate, h0, dh, dlast))
    h, last, carry = nopfs.gated_scan(X, Gt, start, H0)
    dx, dgate, dh0 = nopfs.gated_scan_grad(Dh, X, Gt, start, carry, H0, Dl)
    val, err = _reference(x, gate, h0[0], dh, dlast[0])
    # far below what products of rounded 1 - k may lose in states of this length
    k = torch.sigmoid(-gate[0].to(F64))
    lost = torch.clamp(1 / k, max=T) * 2.0**-25 * (val["last"][0].abs() + 0.1)
    if kind != "noise":
        assert bool((err["last"][0] < lost)[k < 2.0**-12].all())
    for name, t in dict(h=h, last=last, dx=dx, dgate=dgate, dh0=dh0).items():
        close(name, t, val[name], err[name])
