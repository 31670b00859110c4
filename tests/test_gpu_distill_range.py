"""nopfs_topk_distill over the range of temperatures and logits that it takes,
against 64 bits within step_ref's bounds: where max / tau is so large that its
rounding is no small number any more."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import step_ref  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402
from test_gpu_topk_distill import BF, F32, FP, NAMES, _close, _inputs, _run_and_check  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


@pytest.mark.parametrize("dtype", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("V", [300, 5_000, 40_000, 150_001])
@pytest.mark.parametrize("log_tau", [-60, -45, -30, -20, -10, 10])
def test_temperatures(dtype, V, log_tau):
    s, index, y, w = _inputs(4, V, 30, dtype, FP, V + log_tau, 2.5)
    _run_and_check(s, index, y, 2.0**log_tau, w)


@pytest.mark.parametrize("size", [1e5, 1e7, 1e10, 1e20, 1e35])
@pytest.mark.parametrize("V", [300, 40_000, 280_001])
def test_large_logits(size, V):
    s, index, y, w = _inputs(4, V, 30, F32, F32, V, 1.0)
    s[0] *= size
    s[1] = -s[1].abs() * size - size
    s[2] = size + s[2]          # large, and all but equal
    s[3, ::3] = -size           # a mask's value, large against the rest
    _run_and_check(s, index, y, 1.0, w)


@pytest.mark.parametrize("dtype", [BF, FP, F32], ids=NAMES.get)
@pytest.mark.parametrize("tau", [0.75, 1.0, 2.0, 3.0])
@pytest.mark.parametrize("V", [300, 40_000])
def test_rows_of_the_lowest_value(dtype, tau, V):
    """All classes masked by the type's lowest value: the softmax is flat."""
    s, index, y, w = _inputs(3, V, 30, dtype, F32, V)
    s[0] = torch.finfo(dtype).min
    s[1] = torch.finfo(dtype).max
    s[2, 1:] = torch.finfo(dtype).min
    loss, ds = nopfs.topk_distill(s, index, y, tau, weight=w)
    ref = step_ref.distill(s, index, y, tau, w)
    _close("loss", loss, ref[0].float().double(), ref[2])  # w tau 3.4e38 may be beyond 32 bits: inf
    _close("gradient", ds, ref[1], ref[3])


def test_the_loss_keeps_small_temperatures():
    """tau^2 alone leaves the normal range where the loss does not."""
    s, index, y, w = _inputs(3, 500, 9, F32, F32, 11)
    w *= 2.0**-20
    loss, _ = nopfs.topk_distill(s, index, y, 2.0**-60, weight=w)
    ref = step_ref.distill(s, index, y, 2.0**-60, w)
    _close("loss", loss, ref[0], ref[2])
    assert bool((loss > 0).all()) and math.isfinite(float(loss.sum()))
