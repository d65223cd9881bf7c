"""Trees of drafted tokens checked on the GPU: everything is whole numbers or copies, so results are equal."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2511_19457_gb300 import sparoa
    return sparoa


@pytest.fixture(scope="module")
def ctx(sp):
    c = sp.Context(0)
    yield c
    c.sync()
    c.close()


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


class Case:
    """Sequences of new[i] tokens, len[i] cached, in a shuffled cache; trees, tokens and choices at random,
    with few different tokens so that paths are long and siblings alike."""

    def __init__(self, new, length, page=16, kv_heads=2, hd=64, layers=2, vocab=3, seed=0, lead=0):
        rng = random.Random(seed)
        self.new, self.len, self.page = new, length, page
        need = [-(-max(L, 1) // page) for L in length]
        self.pages = sum(need) + 2
        order = list(range(self.pages))
        rng.shuffle(order)
        width = max(need) + 1
        self.table, at = [], 0
        for k in need:
            self.table.append(order[at:at + k] + [-1] * (width - k))
            at += k
        self.start = [lead]
        for n in new:
            self.start.append(self.start[-1] + n)
        self.T = self.start[-1] + 3
        self.tokens = [rng.randrange(vocab) for _ in range(self.T)]
        self.best = [rng.randrange(-1 if vocab > 5 else 0, vocab) for _ in range(self.T)]
        self.parents, self.tree = [], [rng.getrandbits(64) for _ in range(self.T)]
        for b, n in enumerate(new):
            p = [-1] + [rng.randint(-1 if rng.random() < 0.05 else max(0, i - 4), i - 1) for i in range(1, n)]
            bits = []
            for i, up in enumerate(p):
                bits.append((bits[up] if up >= 0 else 0) | 1 << i)
                # bits at and above the token's own mean nothing
                self.tree[self.start[b] + i] = (bits[i] & ((1 << i) - 1)) | rng.getrandbits(64) >> i << i
            self.parents.append(p)
        g = torch.Generator().manual_seed(seed)
        shape = (layers, self.pages, kv_heads, page, hd)
        self.k = (torch.randn(shape, generator=g)).to(torch.bfloat16)
        self.v = (torch.randn(shape, generator=g)).to(torch.bfloat16)

    def want(self):
        path, count, following, length = [-7] * self.T, [], [], []
        k, v = self.k.clone(), self.v.clone()
        for b, (n, L) in enumerate(zip(self.new, self.len)):
            q0, way = self.start[b], []
            at = 0 if n else None
            while at is not None:
                way.append(at)
                here = self.best[q0 + at]
                to = [i for i in range(n) if self.parents[b][i] == at and self.tokens[q0 + i] == here >= 0]
                at = to[0] if to else None
            for i in range(n):
                path[q0 + i] = way[i] if i < len(way) else -1
            count.append(len(way))
            following.append(self.best[q0 + way[-1]] if way else -1)
            length.append(max(0, L - n + len(way)))
            for to, of in enumerate(way):
                src, dst = L - n + of, L - n + to
                if dst < 0 or src == dst:
                    continue
                p0, p1 = self.table[b][src // self.page], self.table[b][dst // self.page]
                for new, old in ((k, self.k), (v, self.v)):
                    new[:, p1, :, dst % self.page] = old[:, p0, :, src % self.page]
        return path, count, following, length, k, v

    def run(self, sp, ctx):
        i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        B = len(self.new)
        k, v = self.k.cuda(), self.v.cuda()
        caches = [sp.KVCache(a, c) for a, c in zip(k, v)]
        batch = sp.PagedBatch(i(self.start), i(self.len), i(self.table), max_q=max(max(self.new), 1))
        path, count, following, length = i([-7] * self.T), i([0] * B), i([0] * B), i([0] * B)
        tree = torch.tensor([_signed(t) for t in self.tree], device="cuda")
        sp.sparoa_tree_accept(ctx, i(self.tokens), i(self.best), tree, caches, batch, path, count, following, length)
        return path.tolist(), count.tolist(), following.tolist(), length.tolist(), k.cpu(), v.cpu()


def _same(got, want):
    for name, a, b in zip(("path", "count", "following", "length"), got, want):
        assert a == b, name
    for name, a, b in zip("kv", got[4:], want[4:]):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("page,kv_heads,hd,layers", [(16, 1, 64, 1), (32, 3, 128, 2), (64, 8, 128, 5), (128, 12, 64, 1)])
def test_paths(sp, ctx, seed, page, kv_heads, hd, layers):
    rng = random.Random(seed)
    new = [rng.choice([1, 2, 3, 8, 31, 32, 33, 63, 64]) for _ in range(7)]
    c = Case(new, [n + rng.randrange(0, 90) for n in new], page, kv_heads, hd, layers, vocab=rng.choice([1, 2, 3, 6]), seed=seed, lead=2)
    _same(c.run(sp, ctx), c.want())


@pytest.mark.parametrize("layers", [8, 9, 32, 33, 128])
def test_many_layers(sp, ctx, layers):
    c = Case([5, 17, 1], [20, 30, 1], 16, 2, 64, layers, vocab=2, seed=layers)
    _same(c.run(sp, ctx), c.want())


def test_one_path_of_all(sp, ctx):
    """64 tokens that all follow one another (nothing moves), and a path that skips every other token."""
    c = Case([64, 64], [64, 100], vocab=1)
    c.parents[0] = list(range(-1, 63))
    c.parents[1] = [-1, 0] + list(range(0, 62))
    for b in range(2):
        bits = []
        for i, up in enumerate(c.parents[b]):
            bits.append((bits[up] if up >= 0 else 0) | 1 << i)
            c.tree[c.start[b] + i] = bits[-1]
    c.tokens = [i & 1 for i in range(c.T)]
    c.best = [1 - (i & 1) if i < 64 else 0 for i in range(c.T)]
    want = c.want()
    assert want[1] == [64, 32]
    _same(c.run(sp, ctx), want)


def test_fewer_cached_than_new_and_empty(sp, ctx):
    """New tokens before their sequence's first position were not cached; sequences without new tokens."""
    c = Case([9, 0, 5, 0, 20], [4, 30, 5, 0, 7], vocab=1, seed=3)
    want = c.want()
    assert want[1][1] == 0 and want[2][1] == -1 and want[3][1] == 30
    _same(c.run(sp, ctx), want)


def test_choices_below_zero_end_a_path(sp, ctx):
    c = Case([6], [20], vocab=1)
    c.tokens = [-1] * c.T
    c.best = [-1] * c.T
    got = c.run(sp, ctx)
    assert got[1] == [1] and got[2] == [-1] and got[0][:6] == [0] + [-1] * 5


def test_many_sequences(sp, ctx):
    new = [1 + b % 9 for b in range(300)]
    c = Case(new, [n + b % 40 for b, n in enumerate(new)], layers=1, kv_heads=1, vocab=2, seed=11)
    _same(c.run(sp, ctx), c.want())


def test_bad_lists_leave_the_sequence(sp):
    """Trees of more than 64 tokens, rows and lengths out of bounds, pages that are none: reported, the other
    sequences are as ever, the bad one's cache stays (its bad page's token, where it is a page).  Pages are
    read where a token moves: the third sequence's stay where they are with seed 5, and move with seed 7."""
    ctx = sp.Context(0)
    for spoil, seed in (("wide", 5), ("rows", 5), ("length", 5), ("page", 5), ("page", 7)):
        c = Case([6, 6, 6], [30, 30, 30], vocab=1, seed=seed)
        good = c.want()
        if spoil == "wide":
            c = Case([6, 70, 6], [30, 80, 30], vocab=1, seed=5)
            c.parents[1] = None
            c.new[1] = 0
            good = c.want()
            c.new[1] = 6
        if spoil == "rows":
            c.start[3] = c.T + 1
        if spoil == "length":
            c.len[2] = 1000
        if spoil == "page":
            c.table[2] = [c.pages] * len(c.table[2])
        got = c.run(sp, ctx)
        moved = good[0][c.start[2]:c.start[2] + good[1][2]] != list(range(good[1][2]))
        if spoil == "page" and not moved:
            ctx.sync()
        else:
            with pytest.raises(sp.SparoaError) as e:
                ctx.sync()
            assert e.value.status == sp.ERR_INVALID_ARG
        b = 1 if spoil == "wide" else 2
        for s in range(3):
            if s != b:
                assert got[1][s] == good[1][s] and got[2][s] == good[2][s] and got[3][s] == good[3][s]
                for page in c.table[s]:
                    if page >= 0:
                        assert torch.equal(got[4][:, page], good[4][:, page]) and torch.equal(got[5][:, page], good[5][:, page])
        if spoil != "page":
            assert got[1][b] == 0 and got[3][b] == c.len[b]
        else:
            assert got[1][b] == good[1][b]
    ctx.sync()
    ctx.close()


def test_graph(sp, ctx):
    """A captured call follows the lists: another tree on the same places."""
    c, d = (Case([12, 5], [40, 33], vocab=2, seed=s) for s in (1, 2))
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    t64 = lambda v: torch.tensor([_signed(t) for t in v], device="cuda")
    k, v = c.k.cuda(), c.v.cuda()
    caches = [sp.KVCache(a, b) for a, b in zip(k, v)]
    start, lens, table = i(c.start), i(c.len), i(c.table)
    batch = sp.PagedBatch(start, lens, table, max_q=12)
    tokens, best, tree = i(c.tokens), i(c.best), t64(c.tree)
    path, count, following, length = i([-7] * c.T), i([0, 0]), i([0, 0]), i([0, 0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sp.sparoa_tree_accept(ctx, tokens, best, tree, caches, batch, path, count, following, length)
    for case in (d, c):
        for to, of in ((start, i(case.start)), (lens, i(case.len)), (table, i(case.table)), (tokens, i(case.tokens)), (best, i(case.best)),
                       (tree, t64(case.tree)), (k, case.k), (v, case.v)):
            to.copy_(of)
        graph.replay()
        torch.cuda.synchronize()
        _same((path.tolist(), count.tolist(), following.tolist(), length.tolist(), k.cpu(), v.cpu()), case.want())


def test_refusals(sp, ctx):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    batch = sp.PagedBatch(i(3), i(2), i(2, 4), max_q=4)
    cache = sp.KVCache.empty(4, 2, 16, 64)
    other = sp.KVCache.empty(5, 2, 16, 64)
    t = torch.zeros(8, dtype=torch.int64, device="cuda")

    def call(tokens=i(8), best=i(8), tree=t, caches=(cache,), batch=batch, path=i(8), count=i(2), following=i(2), length=i(2)):
        sp.sparoa_tree_accept(ctx, tokens, best, tree, caches, batch, path, count, following, length)

    bad = [{"tree": t.int()}, {"tree": t[:7]}, {"best": i(7)}, {"tokens": t}, {"count": i(3)}, {"length": batch.kv_len}, {"caches": ()},
           {"caches": (cache, other)}, {"caches": (cache,) * 129}, {"batch": sp.PagedBatch(i(3), i(2), i(2, 4), max_q=65)}, {"path": i(16)[::2]}, {"caches": (cache, cache)}, {"caches": (sp.KVCache(cache.k, cache.k),)},
           {"caches": (cache, sp.KVCache(other.k[:4], cache.v))}]
    same = i(8)
    bad += [{"tokens": same, "path": same}, {"best": same, "path": same}]
    for kw in bad:
        with pytest.raises(sp.SparoaError):
            call(**kw)
            raise AssertionError(f"{list(kw)} was taken")
    call()
    ctx.sync()
