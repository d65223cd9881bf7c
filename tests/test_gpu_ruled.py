"""Attention under score rules on the GPU against 64 bits: caps, biases by distance, prefixes, trees of drafts.

Tolerances, as for the attention without rules.  fp32 scores (D 2^-24 of sum |q k|, 1e-4 at most here), a cap
(a few 2^-24 of it, 2e-5 for 50) and a bias (2^-24 of what still counts, 30) move the probabilities by 2^-12
at most; they are rounded to one bf16 where there are many rows: (2^-8 + 2^-12) of sum p |v|.  A result is
rounded once: 2^-8 of its size.  The log of the sum moves with the scores: 2e-4."""
import math
import random

import pytest
import torch

from test_gpu_decoder import _batch, _close, _g

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


def _trees(new, seed):
    """Parents of each sequence's new tokens (-1: none; forests too), and their ancestor bits with noise above."""
    rng = random.Random(seed)
    parents, bits = [], []
    for n in new:
        p, b = [], []
        for i in range(n):
            up = -1 if i == 0 or rng.random() < 0.05 else rng.randint(max(0, i - 6), i - 1)
            p.append(up)
            b.append((b[up] if up >= 0 else 0) | 1 << i)
            noise = (b[i] & ((1 << i) - 1)) | rng.getrandbits(64) >> i << i
            bits.append(noise - (1 << 64) if noise >> 63 else noise)
        parents.append(p)
    return parents, torch.tensor(bits, dtype=torch.int64)


def _reference(q, k, v, table, new, kv, page, scale, causal, window, cap, slopes, prefix, parents):
    T, H, D = q.shape
    KH = k.shape[1]
    G = H // KH
    y, size = torch.zeros(T, H, D, dtype=torch.float64), torch.zeros(T, H, D, dtype=torch.float64)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    row = 0
    for b, (n, L) in enumerate(zip(new, kv)):
        for i in range(n):
            t, p = row + i, L - n + i
            far = {}
            if parents is None:
                for j in range(L):
                    if not causal or j <= p or (prefix is not None and j < prefix[b]):
                        far[j] = p - j
            else:
                chain, a = [], i
                while a >= 0:
                    chain.append(a)
                    a = parents[b][a]
                deep = len(chain) - 1
                for j in range(max(0, L - n)):
                    far[j] = L - n + deep - j
                for d, a in enumerate(chain):
                    if 0 <= L - n + a < L:
                        far[L - n + a] = d
            keys = [j for j, d in far.items() if not window or d < window]
            if not keys:
                continue
            at = torch.tensor(keys)
            pages = table[b][at // page].long()
            kk, vv = k[pages, :, at % page].double(), v[pages, :, at % page].double()  # [keys, KH, D]
            d = torch.tensor([abs(far[j]) for j in keys], dtype=torch.float64)
            for h in range(H):
                s = (kk[:, h // G] @ q[t, h].double()) * scale
                if cap:
                    s = cap * torch.tanh(s / cap)
                if slopes is not None:
                    s = s - slopes[h].double() * d
                lse[t, h] = torch.logsumexp(s, 0)
                w = torch.softmax(s, 0)
                y[t, h], size[t, h] = w @ vv[:, h // G], w @ vv[:, h // G].abs()
        row += n
    return y, lse, size


def _run(sp, ctx, new, kv, H, KH, D, page, causal=True, window=0, cap=0.0, slopes=False, prefix=None, tree=False, seed=0, max_q=None, scale=None,
         loud=1.0):
    cache, batch, k, v, table = _batch(sp, new, kv, page, KH, D, seed)
    if max_q is not None:
        batch = sp.PagedBatch(batch.q_start, batch.kv_len, batch.table, max_q)
    T = sum(new)
    q = (loud * torch.randn(T, H, D, generator=_g(seed + 1))).to(torch.bfloat16)
    scale = D ** -0.5 if scale is None else scale
    sl = torch.exp2(-8.0 * torch.arange(1, H + 1) / H) if slopes else None
    parents, bits = _trees(new, seed) if tree else (None, None)
    rules = sp.ScoreRules(cap=cap, slopes=None if sl is None else sl.cuda(),
                          prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda"),
                          tree=None if bits is None else bits.cuda())
    y = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), 5.0, device="cuda")
    sp.sparoa_ruled_attention(ctx, q.cuda(), y, cache, batch, rules, scale=scale, causal=causal, window=window, lse=lse)
    ctx.sync()
    want, wl, size = _reference(q, k, v, table, new, kv, page, scale, causal, window, cap, sl, prefix, parents)
    got = lse.double().cpu()
    empty = wl == -math.inf
    assert torch.equal(got == -math.inf, empty)
    assert (y.cpu()[empty] == 0).all()
    err = (got - wl)[~empty].abs()
    assert (err <= 2e-4 + 2.0 ** -22 * wl[~empty].abs()).all(), f"lse off by {err.max():.2e}"
    _close(y, want, "y", extra=(2.0 ** -8 + 2.0 ** -12) * size + 1e-30)


HEADS = [(4, 4, 64), (8, 2, 128), (6, 1, 64), (3, 1, 128), (16, 2, 64)]
RULES = [dict(cap=30.0), dict(slopes=True), dict(prefix=1), dict(cap=5.0, slopes=True), dict(cap=20.0, prefix=1, slopes=True), dict()]


def _prefixes(kv, kind):
    return [[0, L, L // 2, 1, L + 50][b % 5] for b, L in enumerate(kv)] if kind else None


@pytest.mark.parametrize("H,KH,D", HEADS)
@pytest.mark.parametrize("rules", RULES)
@pytest.mark.parametrize("new,kv,page", [([1, 1, 1, 1, 1], [1, 17, 128, 129, 300], 16), ([3, 2, 1], [3, 140, 260], 64), ([1], [700], 32)])
@pytest.mark.parametrize("window", [0, 70])
def test_few_rows(sp, ctx, H, KH, D, rules, new, kv, page, window):
    kw = dict(rules)
    kw["prefix"] = _prefixes(kv, kw.get("prefix"))
    _run(sp, ctx, new, kv, H, KH, D, page, window=window, **kw)


@pytest.mark.parametrize("H,KH,D", [(4, 4, 64), (8, 2, 128), (3, 1, 64)])
@pytest.mark.parametrize("rules", RULES)
@pytest.mark.parametrize("new,kv,page", [([33, 1, 100], [33, 150, 260], 16), ([70, 5, 40, 3], [200, 5, 300, 129], 128)])
@pytest.mark.parametrize("window", [0, 90])
def test_chunks(sp, ctx, H, KH, D, rules, new, kv, page, window):
    kw = dict(rules)
    kw["prefix"] = _prefixes(kv, kw.get("prefix"))
    _run(sp, ctx, new, kv, H, KH, D, page, window=window, **kw)


@pytest.mark.parametrize("H,KH,D", HEADS)
@pytest.mark.parametrize("new,kv,page", [([2, 4, 3], [2, 130, 300], 16), ([16, 1, 9], [16, 128, 200], 32), ([64, 63, 33], [64, 191, 400], 64),
                                         ([40, 0, 64], [41, 30, 170], 128)])
@pytest.mark.parametrize("rules", [dict(), dict(slopes=True, cap=20.0), dict(window=5), dict(window=100, slopes=True)])
def test_trees(sp, ctx, H, KH, D, new, kv, page, rules):
    _run(sp, ctx, new, kv, H, KH, D, page, tree=True, seed=len(kv) + page, **rules)


@pytest.mark.parametrize("max_q", [1, 64])
@pytest.mark.parametrize("tree", [False, True])
def test_fewer_cached_than_new(sp, ctx, max_q, tree):
    """Tokens before their sequence's first position see nothing but a prefix; in a tree nothing."""
    _run(sp, ctx, [9, 20, 1], [4, 7, 0], 4, 2, 64, 16, tree=tree, prefix=None if tree else [2, 7, 3], slopes=True, seed=4, max_q=max_q)


@pytest.mark.parametrize("max_q", [1, 200])
def test_not_causal(sp, ctx, max_q):
    _run(sp, ctx, [7, 40], [30, 200], 4, 2, 64, 32, causal=False, cap=10.0, slopes=True, max_q=max_q)
    _run(sp, ctx, [7, 40], [30, 200], 4, 2, 64, 32, causal=False, slopes=True, window=20, max_q=max_q)


@pytest.mark.parametrize("max_q,n", [(1, 1), (50, 50)])
@pytest.mark.parametrize("cap", [0.01, 2.0, 50.0, 1000.0])
def test_caps(sp, ctx, max_q, n, cap):
    """Scores far beyond the cap, at both ends, and far below it."""
    for loud in (0.01, 1.0, 40.0):
        if cap == 1000.0 and loud == 40.0:
            continue  # (scores of hundreds: 1e-4 of them is more than the tolerances take)
        _run(sp, ctx, [n], [280], 4, 2, 64, 32, cap=cap, loud=loud, seed=6, max_q=max_q)


def test_no_rules_are_the_attention_without(sp, ctx):
    """Rules that change nothing leave the same results up to the rounding of the scale's place."""
    for new, kv in (([1, 1], [300, 77]), ([60, 3], [400, 90])):
        cache, batch, *_ = _batch(sp, new, kv, 32, 2, 64, 1)
        q = torch.randn(sum(new), 4, 64, generator=_g(2)).to(torch.bfloat16).cuda()
        y, z = torch.empty_like(q), torch.empty_like(q)
        sp.sparoa_paged_attention(ctx, q, y, cache, batch)
        sp.sparoa_ruled_attention(ctx, q, z, cache, batch, sp.ScoreRules())
        # (two roundings to bf16 of numbers that are 2^-12 apart, probabilities too)
        _close(z, y.double().cpu(), "no rules", rel=2.0 ** -7, extra=2.0 ** -7 * 4)


def test_long_contexts_are_split(sp, ctx):
    """Items that many CTAs share, joined: one token and a tree over 20000 keys, a chunk under a prefix."""
    _run(sp, ctx, [1], [20000], 4, 1, 64, 64, cap=15.0, seed=8)
    _run(sp, ctx, [12], [9000], 8, 2, 64, 64, tree=True, slopes=True, seed=9)
    _run(sp, ctx, [1], [5000], 2, 1, 128, 64, slopes=True, window=3000, seed=3)


def test_rows_of_no_sequence_are_left(sp, ctx):
    for n in (2, 60):
        cache, batch, *_ = _batch(sp, [n], [200], 32, 2, 64, 1)
        start = batch.q_start + 3
        batch = sp.PagedBatch(start, batch.kv_len, batch.table, n)
        q = torch.randn(n + 8, 4, 64, generator=_g(2)).to(torch.bfloat16).cuda()
        y, lse = torch.full_like(q, 9.0), torch.full((n + 8, 4), 9.0, device="cuda")
        tree = torch.zeros(n + 8, dtype=torch.int64, device="cuda")
        for rules in (sp.ScoreRules(cap=30.0), sp.ScoreRules(tree=tree)):
            sp.sparoa_ruled_attention(ctx, q, y, cache, batch, rules, lse=lse)
            ctx.sync()
            for t in (y, lse):
                assert (t[:3] == 9).all() and (t[n + 3:] == 9).all() and (t[3:n + 3] != 9).any()


def test_far_keys_under_steep_slopes(sp, ctx):
    """Keys whose bias is hundreds below the nearest ones' weigh nothing, and nothing of them is left in the
    sums, whatever their values."""
    for n in (1, 40, 300):
        cache, batch, k, v, table = _batch(sp, [n], [1500], 64, 1, 64, 5)
        slopes = torch.tensor([4.0, 0.3, 0.01])
        q = torch.randn(n, 3, 64, generator=_g(6)).to(torch.bfloat16)
        y, lse = torch.empty(n, 3, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 3, device="cuda")
        sp.sparoa_ruled_attention(ctx, q.cuda(), y, cache, batch, sp.ScoreRules(slopes=slopes.cuda()), lse=lse)
        some = sorted({0, n // 2, n - 1})
        kk, vv = (torch.cat([pool[int(table[0, j]), 0] for j in range(24)])[:1500].double() for pool in (k, v))
        for i in some:
            p = 1500 - n + i
            s = torch.einsum("hd,ld->hl", q[i].double(), kk[:p + 1]) / 8 - slopes.double()[:, None] * (p - torch.arange(p + 1))
            w = torch.softmax(s, -1)
            assert ((lse[i].double().cpu() - torch.logsumexp(s, -1)).abs() <= 2e-4).all()
            _close(y[i], w @ vv[:p + 1], f"row {i} of {n}", extra=(2.0 ** -8 + 2.0 ** -12) * (w @ vv[:p + 1].abs()))


def test_a_query_that_is_not_a_number(sp, ctx):
    """gives results that are none, its own only; under caps too."""
    for n in (2, 40):
        cache, batch, *_ = _batch(sp, [n], [200], 32, 2, 64, 1)
        q = torch.randn(n, 4, 64, generator=_g(2)).to(torch.bfloat16)
        q[1, 2, 5] = float("nan")
        y = torch.empty(n, 4, 64, dtype=torch.bfloat16, device="cuda")
        sp.sparoa_ruled_attention(ctx, q.cuda(), y, cache, batch, sp.ScoreRules(cap=30.0))
        bad = y.isnan().cpu()
        assert bad[1, 2].all() and int(bad.sum()) == 64


@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("cap", [0.0, 30.0, 200.0])
def test_a_key_that_is_not_a_number(sp, ctx, n, cap):
    """makes results none wherever it is seen, however far away: a bias does not hide it."""
    cache, batch, k, v, table = _batch(sp, [n], [1500], 64, 1, 64, 5)
    cache.k[int(table[0, 0]), 0, 9, 3] = float("nan")  # the key at position 9
    q = torch.randn(n, 3, 64, generator=_g(6)).to(torch.bfloat16).cuda()
    y, lse = torch.empty_like(q), torch.empty(n, 3, device="cuda")
    slopes = torch.tensor([4.0, 0.3, 0.01], device="cuda")
    for window in (0, 1400):
        sp.sparoa_ruled_attention(ctx, q, y, cache, batch, sp.ScoreRules(cap=cap, slopes=slopes), window=window, lse=lse)
        sees = torch.arange(1500 - n, 1500, device="cuda") < 9 + (window or 1500)
        assert y[sees].isnan().all() and lse[sees].isnan().all()
        assert y[~sees].isfinite().all() and lse[~sees].isfinite().all()


def test_graph_follows_its_lists(sp):
    """Another tree, other lengths and queries than those captured."""
    c = sp.Context(0)
    cache, batch, k, v, table = _batch(sp, [6, 5], [60, 100], 16, 2, 64, 3)
    q = torch.zeros(11, 4, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(q)
    tree = torch.zeros(11, dtype=torch.int64, device="cuda")
    rules = sp.ScoreRules(tree=tree)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.sparoa_ruled_attention(c, q, y, cache, batch, rules)
    for step in range(3):
        parents, bits = _trees([6, 5], step)
        tree.copy_(bits)
        lens = [60 - step, 100 - 7 * step]
        batch.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        x = torch.randn(11, 4, 64, generator=_g(step)).to(torch.bfloat16)
        q.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want, _, size = _reference(x, k, v, table, [6, 5], lens, 16, 64 ** -0.5, True, 0, 0, None, None, parents)
        _close(y, want, f"replay {step}", extra=(2.0 ** -8 + 2.0 ** -12) * size)
    c.close()


def test_a_tree_of_too_many_tokens_is_reported(sp):
    c = sp.Context(0)
    cache, batch, *_ = _batch(sp, [65, 4], [100, 50], 16, 2, 64, 3)
    batch = sp.PagedBatch(batch.q_start, batch.kv_len, batch.table, 64)
    q = torch.zeros(69, 4, 64, dtype=torch.bfloat16, device="cuda")
    for max_q in (1, 64):
        batch = sp.PagedBatch(batch.q_start, batch.kv_len, batch.table, max_q)
        sp.sparoa_ruled_attention(c, q, torch.empty_like(q), cache, batch, sp.ScoreRules(tree=torch.zeros(69, dtype=torch.int64, device="cuda")))
        with pytest.raises(sp.SparoaError) as e:
            c.sync()
        assert e.value.status == sp.ERR_INVALID_ARG
    c.sync()
    c.close()


def test_refusals(sp, ctx):
    cache, batch, *_ = _batch(sp, [1, 1], [20, 20], 16, 2, 64, 8)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(q)
    f4, i2, t2 = torch.zeros(4, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    S = sp.ScoreRules

    def go(rules, batch=batch, **kw):
        sp.sparoa_ruled_attention(ctx, q, y, cache, batch, rules, **kw)

    wide = sp.PagedBatch(batch.q_start, batch.kv_len, batch.table, 65)
    bad = [lambda: go(S(cap=-1.0)), lambda: go(S(cap=math.nan)), lambda: go(S(cap=math.inf)), lambda: go(S(cap=1e-6)), lambda: go(S(slopes=f4[:3])),
           lambda: go(S(prefix=i2[:1])), lambda: go(S(tree=t2[:1])), lambda: go(S(tree=t2, prefix=i2)), lambda: go(S(tree=t2), causal=False),
           lambda: go(S(prefix=i2), causal=False), lambda: go(S(tree=t2), wide), lambda: S(slopes=f4.half()), lambda: S(prefix=t2), lambda: S(tree=i2),
           lambda: S(slopes=f4.cpu()), lambda: go(S(), scale=0.0), lambda: go(S(), window=-1)]
    for i, f in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            f()
            raise AssertionError(f"call {i} was taken")
    go(S(tree=t2))
    ctx.sync()
