"""The order in which nopfs_token_embed_grad adds, bit by bit: a name's tokens in the
order of the batch within a piece of the sorted tokens; the parts of a name of several
pieces every so manieth by a group of lanes, then the groups' sums in order."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2101_08734_amd import nopfs  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _log2_ceil(n):
    return max(0, int(n - 1).bit_length())


def _sums(dout, ids, V):
    """float32 sums in that order."""
    T, width = dout.shape
    lanes = min(8, _log2_ceil(-(-width // 8)))
    per = 32
    while per > 8 and (-(-T // per) << lanes) < 2**17:
        per //= 2
    while -(-T // per) > 8192:
        per *= 2
    keys = np.where((ids >= 0) & (ids < V), ids, V)
    order = np.argsort(keys, kind="stable")
    parts = {}
    for i, t in enumerate(order):
        v = keys[t]
        if v == V:
            break
        rows = parts.setdefault(v, {})
        rows[i // per] = rows[i // per] + dout[t] if i // per in rows else dout[t].copy()
    groups = 256 >> min(6, _log2_ceil(-(-width // 4)))
    out = np.zeros((V, width), dtype=np.float32)
    for v, rows in parts.items():
        rows = [rows[p] for p in sorted(rows)]
        if len(rows) > 1:
            sums = []
            for g in range(groups):
                s = np.zeros(width, dtype=np.float32)
                for r in rows[g::groups]:
                    s = s + r
                sums.append(s)
            rows = sums
        s = rows[0]
        for r in rows[1:]:
            s = s + r
        out[v] = s
    return out, max(len(r) for r in parts.values())


@pytest.mark.parametrize("T,V,kind", [(5_003, 900, "few"), (6_144, 70, "few"), (6_145, 900, "few"),
                                      (30_011, 40_000, "few"), (30_011, 3_000, "many"), (9_001, 5, "even")])
@pytest.mark.parametrize("width", [3, 40, 300])
def test_every_bit(T, V, kind, width):
    """Rows of sizes from 2^-12 to 2^12, so that every other order gives other sums: by
    one workgroup's sort and by passes over tiles, of one digit and of two, names of one
    piece and of hundreds that begin and end anywhere in tiles, waves and pieces."""
    rng = np.random.default_rng(T + V + width)
    ids = rng.integers(-2, V, T)
    if kind == "few":  # a third of the tokens of two names
        ids[rng.random(T) < 0.2] = 3
        ids[rng.random(T) < 0.15] = V - 1
    elif kind == "even":
        ids = np.arange(T) % (V + 1) - 1
    dout = (rng.standard_normal((T, width)) * np.exp2(rng.integers(-12, 13, (T, 1)))).astype(np.float32)
    want, parts = _sums(dout, ids, V)
    assert parts > (1 if kind == "many" else 30)
    got = nopfs.token_embed_grad(torch.from_numpy(dout).cuda(), torch.from_numpy(ids).cuda(), V)
    assert np.array_equal(got.cpu().numpy(), want)
    assert not np.array_equal(want, _sums(dout[::-1], ids[::-1], V)[0])  # the order shows
