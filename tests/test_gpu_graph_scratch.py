"""Scratch under graph capture (include/nopfs.h, conventions): a captured call
allocates nothing, and a block that it used outlives larger calls on its stream."""
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


class Replay:
    """A clairvoyant buffer's replay of a job, with its outputs preallocated."""

    def __init__(self, *shape):
        self.job = nopfs.Job(*shape)
        self.R = nopfs.access_streams(self.job)
        self.next = nopfs.reuse_next(self.job, self.R)
        self.sizes = torch.randint(1, 1_000, (self.job.F,), device="cuda", dtype=torch.int64)
        self.d0 = int(self.sizes.sum()) // 8
        self.hit = torch.empty(self.R.shape, dtype=torch.int8, device="cuda")
        self.hits = torch.empty((self.job.N, 2), dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()

    def call(self, stream=None):
        nopfs.buffer_sim(self.job, self.R, self.next, self.sizes, self.d0, self.hit, self.hits, stream=stream)

    def result(self):
        torch.cuda.synchronize()
        return self.hit.clone(), self.hits.clone()


def _capture(replay, stream):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        graph.capture_begin(capture_error_mode="relaxed")
        try:
            replay.call(stream)
        finally:
            graph.capture_end()
    return graph


def test_a_captured_block_outlives_larger_calls():
    small, large = Replay(20_000, 4, 8, 2, 1, 5), Replay(300_000, 6, 16, 8, 0, 6)
    small.call()
    want = small.result()
    s = torch.cuda.Stream()
    small.call(s)  # the stream's block
    s.synchronize()
    graph = _capture(small, s)
    for _ in range(3):
        large.call(s)  # the first outgrows the block
        s.synchronize()
        # what a freed block would be handed out as, overwritten
        filler = [torch.full((1 << 22,), 77, dtype=torch.int32, device="cuda") for _ in range(8)]
        small.hit.fill_(7)
        small.hits.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        for a, b in zip(want, small.result()):
            assert torch.equal(a, b)
        assert all(bool((x == 77).all()) for x in filler)
        del filler
        torch.cuda.empty_cache()
    del graph
    nopfs.scratch_release(stream=s)


def test_a_capture_allocates_nothing():
    """Without room in the stream's block the call is refused, and the capture goes on."""
    r = Replay(20_000, 4, 8, 2, 1, 5)
    r.call()
    want = r.result()
    s, mark = torch.cuda.Stream(), torch.zeros(64, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin(capture_error_mode="relaxed")
        with pytest.raises(nopfs.NopfsError) as e:
            r.call(s)
        mark.add_(1.0)
        graph.capture_end()
    assert e.value.code == nopfs.NOPFS_ENOMEM and "captured" in str(e.value)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert bool((mark == i + 1.0).all())
    r.call(s)  # eagerly it allocates as ever
    for a, b in zip(want, r.result()):
        assert torch.equal(a, b)
    nopfs.scratch_release(stream=s)
