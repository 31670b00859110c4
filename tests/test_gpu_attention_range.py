"""nopfs_packed_attention over the range of scales and scores that it takes.

Small whole numbers as q and k make every product and sum exact in 32 bits and
different scores at least 1 apart: at a scale of 2^7 or more the softmax is 1 / c
on the c largest scores of a row, so o is a 32-bit mean of rows of v, rounded
once, and lse = scale max + log c. The exponentials of the largest scores, 1, may
all carry one factor within 2^-15 of 1, which their rounding to 16 bits takes away
and their sum keeps: o is off by 2^-14 more."""
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


def _whole(T, heads, width, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randint(-4, 5, (T, heads, width), generator=g).to(dtype).cuda() for _ in range(2))
    v = torch.randn((T, heads, width), generator=g).to(dtype).cuda()
    return q, k, v


def _check(q, k, v, start, scale, first=0):
    """Rows from `first` on of every sample."""
    st = torch.tensor(start, dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, st, scale=scale)
    u = 2.0**-8 if q.dtype == BF else 2.0**-11
    for a, b in zip(start, start[1:]):
        for h in range(q.shape[1] if b > a else 0):
            s = q[a:b, h].double() @ k[a:b, h].double().T
            s = torch.where(torch.ones_like(s, dtype=torch.bool).tril(), s, -math.inf)
            top = s.amax(1, keepdim=True)
            p = (s == top).double()
            count = p.sum(1, keepdim=True)
            want = (p / count) @ v[a:b, h].double()
            rows = slice(a + first, b)
            off = (o[rows, h].double() - want[first:]).abs()
            assert bool((off <= (u + 2.0**-14) * want[first:].abs() + 2.0**-20).all()), float(off.max())
            z = (scale * top + count.log()).squeeze(1)[first:]
            off = (lse[h, rows].double() - z).abs()
            assert bool((off <= 2.0**-22 * (z.abs() + 1)).all()), float(off.max())


SCALES = [2.0**7, 2.0**20, 2.0**27, 2.0**30, 2.0**45, 2.0**60]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("width", [64, 80, 128])
@pytest.mark.parametrize("scale", SCALES, ids=lambda x: f"2^{int(math.log2(x))}")
def test_scales(scale, width, dtype):
    lengths = [1, 333, 0, 70, 200]
    start = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    _check(*_whole(start[-1], 2, width, dtype, width), start, scale)
    _check(*_whole(700, 1, width, dtype, width), [0, 700], scale)  # four waves share 32 queries


@pytest.mark.parametrize("scale", SCALES[2::2])
@pytest.mark.parametrize("T,heads,width", [(3_300, 1, 64), (3_300, 1, 128), (150, 520, 64), (150, 520, 128)])
def test_scales_of_parts_and_of_many_heads(scale, T, heads, width):
    _check(*_whole(T, heads, width, BF, T), [0, T], scale)


@pytest.mark.parametrize("T,heads,width", [(400, 2, 64), (400, 2, 128), (3_300, 1, 64), (300, 520, 128)])
def test_scores_of_minus_infinity(T, heads, width):
    """A tile of keys whose scores are all -inf: they have no weight, whatever
    comes behind them (rows that see no other key have no value)."""
    q, k, v = _whole(T, heads, width, BF, 3)
    q[:, :, 5] = 1.0
    k[:170, :, 5] = -math.inf
    _check(q, k, v, [0, T], 128.0, first=170)


def test_large_scores_at_an_ordinary_scale():
    q, k, v = _whole(333, 2, 64, BF, 4)
    for size in (2.0**20, 2.0**40):
        _check(q * size, k * size, v, [0, 333], 1.0)


def test_the_gradients_largest_scale():
    """Beyond 2^10 lse in 32 bits says too little of the softmax."""
    q, k, v = _whole(50, 2, 64, BF, 5)
    st = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    o, lse = nopfs.packed_attention(q, k, v, st, scale=2.0**11)
    with pytest.raises(nopfs.NopfsError):
        nopfs.packed_attention_grad(v, q, k, v, o, lse, st, scale=2.0**11)
