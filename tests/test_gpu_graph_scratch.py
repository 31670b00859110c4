"""Scratch under graph capture (include/nopfs.h, conventions): a captured call
allocates nothing, and a block that it used outlives larger calls on its stream."""
import gc

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


@pytest.fixture(autouse=True)
def _no_graph_left():
    """A graph that the collector finds, and destroys, during another's capture
    ends the process (torch's destructor may not call the device then)."""
    gc.collect()
    yield
    gc.collect()


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
        code = what = None
        try:  # (an ExceptionInfo would hold the frame and the graph in a cycle)
            r.call(s)
        except nopfs.NopfsError as e:
            code, what = e.code, str(e)
        mark.add_(1.0)
        graph.capture_end()
    assert code == nopfs.NOPFS_ENOMEM and "captured" in what
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert bool((mark == i + 1.0).all())
    r.call(s)  # eagerly it allocates as ever
    for a, b in zip(want, r.result()):
        assert torch.equal(a, b)
    nopfs.scratch_release(stream=s)


# -- the operators of a training step ------------------------------------------------
def _attention_inputs(lengths, heads, kv_heads, width, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(lengths)
    x = torch.randn((T, heads + 2 * kv_heads, width), generator=g, device="cuda").bfloat16()
    do = torch.randn((T, heads, width), generator=g, device="cuda").bfloat16()
    start = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    return (x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]), do, start


def _step(qkv, do, start, stream=None):
    o, lse = nopfs.packed_attention(*qkv, start, stream=stream)
    return (o, lse, *nopfs.packed_attention_grad(do, *qkv, o, lse, start, stream=stream))


SHAPES = {"plain": ([200, 77], 2, 1, 64), "parts": ([3_300, 900], 2, 1, 64),
          "ordered": ([700, 1, 1_500, 64, 900, 33, 1_620], 2, 2, 128)}


@pytest.mark.parametrize("shape", SHAPES)
def test_attention_captured_without_a_call_before(shape):
    """Captured on a stream without a block, replayed between larger eager calls
    on that stream: the graph's scratch is its own."""
    qkv, do, start = _attention_inputs(*SHAPES[shape], 1)
    big = _attention_inputs([6_000, 900], 4, 2, 128, 2)
    want_big = _step(*big)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = _step(qkv, do, start, stream=s)
    for i in range(3):
        for t in got:
            t.fill_(3.0)
        qkv[0].mul_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(_step(qkv, do, start), got):
            assert torch.equal(a, b), i
        for a, b in zip(want_big, _step(*big, stream=s)):
            s.synchronize()
            assert torch.equal(a, b), i
    del graph
    nopfs.scratch_release(stream=s)


def test_two_graphs_of_one_stream_at_once():
    """Captured on one stream, replayed on two beside eager calls on the first."""
    s, others = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    cases = [_attention_inputs([3_300, 900], 2, 1, 64, seed) for seed in (3, 4)]
    eager = _attention_inputs([2_900, 1_300], 2, 1, 64, 5)
    wants = [_step(*c) for c in cases]
    want = _step(*eager)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(_step(*c, stream=s))
        graphs.append(graph)
    for _ in range(5):
        for out in outs:
            for t in out:
                t.fill_(3.0)
        torch.cuda.synchronize()
        for graph, other in zip(graphs, others):
            with torch.cuda.stream(other):
                graph.replay()
        got = _step(*eager, stream=s)
        torch.cuda.synchronize()
        for a, b in zip(sum(wants, ()) + want, sum(outs, ()) + got):
            assert torch.equal(a, b)
    del graphs
    nopfs.scratch_release(stream=s)


def test_tables_captured_without_a_call_before():
    g = torch.Generator(device="cuda").manual_seed(6)
    lengths = torch.randint(0, 90, (4, 3_000), generator=g, device="cuda", dtype=torch.int32)
    free = torch.arange(40_000, device="cuda", dtype=torch.int32).view(4, 10_000)
    args = (None, lengths, free, 16, 6, 120_000)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = nopfs.batch_tables(*args, stream=s)
    for i in range(3):
        for t in got.values():
            t.fill_(3)
        lengths.copy_(lengths.roll(1, 1))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = nopfs.batch_tables(*args)
        for name in want:
            assert torch.equal(want[name], got[name]), (i, name)
    del graph
    nopfs.scratch_release(stream=s)


def test_a_captured_call_without_its_callers_scratch():
    """Refused by the library, the capture goes on; calls that need none are captured."""
    qkv, do, start = _attention_inputs([200, 77], 2, 1, 64, 7)
    o, lse, *grads = _step(qkv, do, start)
    s, mark = torch.cuda.Stream(), torch.zeros(64, device="cuda")
    torch.cuda.synchronize()
    a = nopfs._Attention(277, 2, 2, 1, 64, 0, 0.125, *nopfs._strides(*qkv, o, do, *grads))
    arrays = [t.data_ptr() for t in (do, *qkv, o, lse, start, *grads)]
    again, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin(capture_error_mode="relaxed")
        rc = nopfs.lib().nopfs_packed_attention_grad(a, *arrays, s.cuda_stream)
        detail = nopfs.lib().nopfs_last_error()
        nopfs.packed_attention(*qkv, start, o=again, lse=lse2)
        mark.add_(1.0)
        graph.capture_end()
    assert rc == nopfs.NOPFS_EINVAL and b"captured" in detail
    graph.replay()
    torch.cuda.synchronize()
    assert bool((mark == 1.0).all()) and torch.equal(again, o) and torch.equal(lse2, lse)
