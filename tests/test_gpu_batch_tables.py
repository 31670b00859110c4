"""nopfs_batch_tables against the definition, read by read and token by token:
every output equal, over lengths of zero and one, reads that end inside a
block, cuts by tokens, by blocks and by the table's width, padding ids, strided
reads and lists, block ids whose slots pass 32 bits, and streams."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import step_ref  # noqa: E402
from paper_2101_08734_amd import nopfs  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    nopfs.lib()
    yield


def _inputs(G, n, F, blocks, longest, zeros, pads, seed, high=0):
    rng = np.random.default_rng(seed)
    tokens = rng.integers(1, longest + 1, F).astype(np.int32)
    tokens[rng.random(F) < zeros] = 0
    ids = rng.integers(0, F, (G, 2 * n + 1)).astype(np.int32)
    ids[rng.random(ids.shape) < pads] = -1
    free = np.stack([rng.permutation(2 * blocks + 1) for _ in range(G)]).astype(np.int32) + high
    return ids, tokens, free


def _check(ids, tokens, free, block, width, cap, got):
    want = step_ref.tables(ids, tokens, free, block, width, cap)
    for name, w in want.items():
        g = got[name].cpu().numpy()
        assert g.dtype == w.dtype and np.array_equal(g, w), name


CASES = [  # G, n, F, blocks, block, width, cap, longest, zeros, pads
    (1, 1, 1, 1, 1, 1, 1, 1, 0, 0),
    (1, 1, 5, 4, 16, 4, 64, 64, 0, 0),
    (1, 32, 1000, 256, 64, 32, 12_288, 2_048, 0, 0),
    (3, 20, 500, 110, 48, 40, 5_001, 1_900, 0.1, 0.2),    # cut by tokens or by blocks
    (2, 65, 300, 5_000, 17, 9, 20_000, 170, 0.3, 0),      # cut by the width
    (5, 257, 99, 700, 32, 4, 16_385, 100, 0.5, 0.5),
    (2, 1_030, 700, 2_100, 16, 3, 33_000, 40, 0.2, 0.1),  # many reads
    (7, 300, 50, 300, 1, 3, 1_000, 3, 0.3, 0),            # blocks of one token
    (1, 40, 60, 0, 8, 2, 100, 12, 0.5, 0),                # no free block
    (2, 9, 60, 30, 8, 2, 0, 12, 0.9, 0),                  # no room for a token
    (1, 3, 60, 9, 4_096, 5, 9_001, 9_000, 0, 0),          # blocks larger than a read
    (1_030, 2, 60, 9, 8, 5, 33, 30, 0.1, 0),
    (2, 5_000, 2_000, 30_000, 8, 5, 70_001, 30, 0.1, 0.02),
    (1, 20_000, 500, 9_000, 8, 2, 30_000, 12, 0.8, 0),   # thousands of reads in a tile
    (3, 200, 900, 9_000, 16, 40, 120_000, 600, 0.1, 0),   # few reads, many tokens
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_against_the_definition(case):
    G, n, F, blocks, block, width, cap, longest, zeros, pads = case
    ids, tokens, free = _inputs(G, n, F, blocks, longest, zeros, pads, n + G)
    view = torch.from_numpy(ids).cuda()[:, n // 2:n // 2 + n]
    lists = torch.from_numpy(free).cuda()[:, :blocks]
    got = nopfs.batch_tables(view, torch.from_numpy(tokens).cuda(), lists, block, width, cap)
    _check(ids[:, n // 2:n // 2 + n], tokens, free[:, :blocks], block, width, cap, got)
    # the lengths themselves, into used memory
    there = (ids >= 0) & (ids < F)
    lens = np.where(there, tokens[np.where(there, ids, 0)], -3).astype(np.int32)
    for t in got.values():
        t.fill_(77)
    view = torch.from_numpy(lens).cuda()[:, n // 2:n // 2 + n]
    again = nopfs.batch_tables(None, view, lists, block, width, cap, out=got)
    assert all(again[k] is got[k] for k in got)
    _check(None, lens[:, n // 2:n // 2 + n], free[:, :blocks], block, width, cap, got)


@pytest.mark.parametrize("at", [0, 1, 63, 64, 255, 256, 999])
@pytest.mark.parametrize("what", ["tokens", "blocks", "width"])
def test_first_read_that_does_not_fit(at, what):
    """Everything fits but read `at`; the reads behind it are left out too."""
    n, block = 1_000, 4
    tokens = np.full((1, n), 5, np.int32)
    width, cap, blocks = 3, 5 * n, 2 * n
    if what == "width":
        tokens[0, at] = 13
    elif what == "tokens":
        cap = 5 * (at + 1) - 1
    else:
        blocks = 2 * at + 1
    free = np.arange(blocks, dtype=np.int32)[None]
    got = nopfs.batch_tables(None, torch.from_numpy(tokens).cuda(), torch.from_numpy(free).cuda(),
                             block, width, cap)
    _check(None, tokens, free, block, width, cap, got)
    assert got["used"][0].tolist() == [at, 5 * at, 2 * at]


def test_slots_beyond_32_bits_and_lengths_of_int32():
    rng = np.random.default_rng(5)
    free = np.sort(rng.integers(2**31 - 10_000, 2**31 - 1, (1, 50))).astype(np.int32)
    tokens = np.array([[700, 300, 2**31 - 1, 5]], np.int32)
    got = nopfs.batch_tables(None, torch.from_numpy(tokens).cuda(), torch.from_numpy(free).cuda(),
                             100, 8, 4_000)
    _check(None, tokens, free, 100, 8, 4_000, got)
    assert int(got["slot"].max()) > 2**36


def test_reads_of_a_plan_on_another_stream():
    job = nopfs.Job(5_000, 3, 6, 8, 0, 9)
    R = nopfs.access_streams(job)
    tokens = (torch.arange(5_000, device="cuda", dtype=torch.int32) * 37) % 90
    free = torch.arange(600, device="cuda", dtype=torch.int32).repeat(6, 1).contiguous()
    f0 = R.shape[1] - 40  # ends in the padding of the shorter rows
    want = nopfs.batch_tables(R[:, f0:], tokens, free, 16, 6, 3_000)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = nopfs.batch_tables(R[:, f0:], tokens, free, 16, 6, 3_000, stream=s)
    s.synchronize()
    for k in want:
        assert torch.equal(want[k], got[k]), k
    _check(R[:, f0:].cpu().numpy(), tokens.cpu().numpy(), free.cpu().numpy(), 16, 6, 3_000, got)
