"""Attention over a paged cache from graphs and many streams: calls and replays whose work may overlap
have partial results and arrival counters of their own."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


class Job:
    """A sequence that is split over many CTAs, by the kernel for few rows or for chunks."""

    def __init__(self, sp, seed, n=1, L=30000, heads=4, D=128, page=64):
        g = torch.Generator().manual_seed(seed)
        pages = -(-L // page)
        pools = (torch.randn(pages, 1, page, D, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        self.cache = sp.KVCache(*pools)
        self.batch = sp.PagedBatch(ints([0, n]), ints([L]), torch.randperm(pages, generator=g).to(torch.int32).view(1, -1).cuda(), n)
        self.q = torch.randn(n, heads, D, generator=g).to(torch.bfloat16).cuda()
        self.y = torch.empty_like(self.q)
        self.sp = sp

    def __call__(self, ctx, y=None):
        self.sp.sparoa_paged_attention(ctx, self.q, self.y if y is None else y, self.cache, self.batch)

    def expect(self, ctx):
        """What the call gives alone (results do not depend on timing)."""
        self.want = torch.empty_like(self.y)
        self(ctx, self.want)
        torch.cuda.synchronize()
        return self

    def check(self):
        assert torch.equal(self.y, self.want)
        self.y.fill_(float("nan"))


@pytest.mark.parametrize("n", [(1, 1), (40, 40), (1, 40)])
def test_graphs_of_one_capture_stream(sp, n):
    """Two graphs recorded on the capture stream that all graphs share by default, replayed on two streams."""
    ctx = sp.Context(0)
    jobs = [Job(sp, i, n[i]).expect(ctx) for i in range(2)]
    graphs = []
    for j in jobs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            j(ctx)
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        torch.cuda.synchronize()
        for _ in range(10):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for j in jobs:
            j.check()
    ctx.sync()
    ctx.close()


@pytest.mark.parametrize("n", [1, 40])
def test_graph_beside_calls_on_its_capture_stream(sp, n):
    ctx = sp.Context(0)
    a, b = Job(sp, 3, n).expect(ctx), Job(sp, 4, n).expect(ctx)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a(ctx)
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(t):
            graph.replay()
        with torch.cuda.stream(s):
            b(ctx)
    torch.cuda.synchronize()
    a.check()
    b.check()
    ctx.sync()
    ctx.close()


@pytest.mark.parametrize("n", [1, 40])
def test_streams_of_one_capture(sp, n):
    """Branches of a graph may run at once."""
    ctx = sp.Context(0)
    a, b = Job(sp, 5, n).expect(ctx), Job(sp, 6, n).expect(ctx)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        a(ctx)
        with torch.cuda.stream(side):
            b(ctx)
            b(ctx)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        a.check()
        b.check()
    ctx.sync()
    ctx.close()


def test_both_kernels_in_one_capture(sp):
    """The second call of a capture may want more room than the first has."""
    ctx = sp.Context(0)
    jobs = [Job(sp, 7, 1).expect(ctx), Job(sp, 8, 40).expect(ctx), Job(sp, 9, 1).expect(ctx)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for j in jobs:
            j(ctx)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for j in jobs:
            j.check()
    ctx.sync()
    ctx.close()


def test_more_streams_than_scratch(sp):
    """Streams take turns in the context's scratch; a graph's stays its own."""
    ctx = sp.Context(0)
    kept = Job(sp, 10, 2, 5000).expect(ctx)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        kept(ctx)
    jobs = [Job(sp, 20 + i, 1 + 20 * (i % 2), 5000).expect(ctx) for i in range(20)]
    streams = [torch.cuda.Stream() for _ in jobs]
    assert len({st.cuda_stream for st in streams}) == 20
    torch.cuda.synchronize()
    for _ in range(3):
        for j, st in zip(jobs, streams):
            with torch.cuda.stream(st):
                j(ctx)
            graph.replay()
        torch.cuda.synchronize()
        for j in jobs:
            j.check()
        kept.check()
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=streams[3]):
        jobs[3](ctx)  # (a capture on any of them, too)
    ctx.sync()
    ctx.close()


def test_scratch_of_graphs_that_are_gone(sp):
    """What a destroyed graph leaves is used by the next one."""
    ctx = sp.Context(0)
    job = Job(sp, 11, 40).expect(ctx)
    free = []
    for _ in range(40):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            job(ctx)
        graph.replay()
        torch.cuda.synchronize()
        job.check()
        del graph
        time.sleep(0.02)  # (the driver says so from a thread of its own)
        free.append(torch.cuda.mem_get_info()[0])
    assert free[0] - free[-1] < 10 * (40 << 20), [f >> 20 for f in free]
    ctx.close()


def test_context_before_its_graphs(sp):
    """A graph that outlives its context can be destroyed (though not replayed)."""
    ctx = sp.Context(0)
    job = Job(sp, 12).expect(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        job(ctx)
    ctx.sync()
    ctx.close()
    del graph
    time.sleep(0.02)
    torch.cuda.synchronize()
