"""Decoder operators on the GPU against plain 64-bit implementations: the residual step with its
norms, rotary positions into a paged cache, attention over it.

Tolerances.  A bf16 result is rounded once: at most 2^-8 of the value.  fp32 sums of C
terms add at most C 2^-24 of the terms' sizes, far below that; for values that are small beside
their row (cancellation) an absolute part of 1e-5 of the row's largest is allowed.  Attention of few
rows keeps 16 bits of its probabilities (2^-16 of sum p |v|), and fp32 scores (D 2^-24 of sum |q k|, at
most 1e-4 here) move the probabilities by 1e-4: 2^-9 + 2^-12 of sum p |v| is allowed for both.
Attention of chunks rounds them to one bf16: 2^-8 + 2^-12 of sum p |v|.
The log of the sum moves with the scores: 2e-4."""
import math

import numpy as np
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


def _g(seed):
    return torch.Generator().manual_seed(seed)


def _close(got, ref, what, rel=2.0 ** -8, extra=None):
    got, ref = got.double().cpu(), ref.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    tol = rel * ref.abs() + (extra if extra is not None else 1e-5 * ref.abs().amax(-1, keepdim=True))
    bad = (got - ref).abs() > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got - ref).abs() - tol).max():.3e}"


# ---------------------------------------------------------------------------
# residual step
# ---------------------------------------------------------------------------
def _norm64(v, n, eps):
    if n is None or n[0] == "none":
        return v
    kind, w, b = n
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / ((v * v).mean(-1, keepdim=True) + eps).sqrt()
    if w is not None:
        v = v * w.double()
    return v if b is None else v + b.double()


def _params(kind, C, seed, weight=True, bias=False):
    g = _g(seed)
    return (kind, 1 + 0.2 * torch.randn(C, generator=g) if weight else None, 0.3 * torch.randn(C, generator=g) if bias else None)


NORM_SHAPES = [(1, 8), (3, 64), (5, 256), (4, 264), (7, 512), (2, 520), (9, 1024), (3, 1032), (197, 768), (2, 4096), (1, 8192),
               (2, 8200), (1, 16384), (1000, 128)]


@pytest.mark.parametrize("R,C", NORM_SHAPES)
@pytest.mark.parametrize("res", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("post,pre,gate", [("none", "rms", 0), ("rms", "rms", None), ("layer", "layer", 3), ("rms", "none", 1)])
def test_add_norm(sp, ctx, R, C, res, post, pre, gate):
    g = _g(R * 31 + C)
    x = (3 * torch.randn(R, C, generator=g)).to(res)
    h = (torch.randn(R, C, generator=g) + 0.5).to(torch.bfloat16)
    h[R // 2] = 0  # a row without variance
    n1 = _params(post, C, 1, bias=post == "layer")
    n2 = _params(pre, C, 2, bias=pre == "layer")
    per = gate or 0
    gt = None if gate is None else torch.randn(-(-R // per) if per else 1, C, generator=g)
    y = torch.full((R, C), float("nan"), dtype=torch.bfloat16, device="cuda")
    r = torch.full((R, C), float("nan"), dtype=res, device="cuda")
    dev = [sp.norm(n[0], *(None if t is None else t.cuda() for t in n[1:]), eps=1e-5) for n in (n1, n2)]
    occ = sp.OccupancyBuffer(R, C)
    sp.sparoa_add_norm(ctx, x.cuda(), h.cuda(), r, y, post=dev[0], gate=None if gt is None else gt.cuda(), rows_per_gate=per,
                       scale=0.5, pre=dev[1], y_occ=occ)
    z = 0.5 * _norm64(h.double(), n1, 1e-5)
    if gt is not None:
        z = z * (gt.double().repeat_interleave(per, 0)[:R] if per else gt.double())
    want = x.double() + z
    # fp32 r: a few roundings of its two terms
    _close(r, want, "r", rel=2.0 ** -8 if res == torch.bfloat16 else 2.0 ** -21, extra=1e-5 * want.abs().amax(-1, keepdim=True)
           if res == torch.bfloat16 else 2.0 ** -20 * (x.double().abs() + z.abs() + z.abs().amax(-1, keepdim=True)))
    _close(y, _norm64(want, n2, 1e-5), "y")
    assert occ.to_host()["nnz"] == int((y != 0).sum())


@pytest.mark.parametrize("R,C", [(1221, 200), (1301, 520), (2433, 600), (1217, 768), (1251, 1000), (1219, 1024), (2435, 1024), (1303, 1032)])
@pytest.mark.parametrize("res", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("post,pre,gate", [("none", "layer", 197), ("rms", "rms", None), ("layer", "layer", 0)])
def test_add_norm_many_rows(sp, ctx, R, C, res, post, pre, gate):
    """More rows than CTAs are on the GPU at once, of lengths around those that a warp takes alone; in place too."""
    test_add_norm(sp, ctx, R, C, res, post, pre, gate)
    g = _g(R)
    x = torch.randn(R, C, generator=g).to(res)
    h = torch.randn(R, C, generator=g).to(torch.bfloat16)
    w = _params("rms", C, 3)
    xd, hd = x.cuda(), h.cuda()
    sp.sparoa_add_norm(ctx, xd, hd, xd, hd, pre=sp.norm("rms", w[1].cuda()))
    _close(xd, x.double() + h.double(), "r in place of x")
    _close(hd, _norm64(x.double() + h.double(), w, 1e-6), "y in place of h")


def test_add_norm_parts(sp, ctx):
    """No block output (a first norm), no stream before it, no output asked for, and results in place."""
    R, C = 37, 1000
    g = _g(5)
    x = torch.randn(R, C, generator=g).to(torch.bfloat16)
    h = torch.randn(R, C, generator=g).to(torch.bfloat16)
    w = _params("rms", C, 3)
    n = sp.norm("rms", w[1].cuda())
    y = torch.empty(R, C, dtype=torch.bfloat16, device="cuda")
    sp.sparoa_add_norm(ctx, x.cuda(), None, None, y, pre=n)
    _close(y, _norm64(x.double(), w, 1e-6), "norm of x")
    r = torch.empty(R, C, dtype=torch.float32, device="cuda")
    sp.sparoa_add_norm(ctx, None, h.cuda(), r, None, post=n, scale=-2.0)
    _close(r, -2 * _norm64(h.double(), w, 1e-6), "post norm alone")
    xd, hd = x.cuda(), h.cuda()
    sp.sparoa_add_norm(ctx, xd, hd, xd, hd, pre=n)
    _close(xd, x.double() + h.double(), "r in place of x")
    _close(hd, _norm64(x.double() + h.double(), w, 1e-6), "y in place of h")


def test_add_norm_large_values(sp, ctx):
    """A row whose values are far from zero keeps its variance; rows of huge values stay finite."""
    R, C = 4, 2048
    g = _g(6)
    x = torch.randn(R, C, generator=g) + 1000.0
    x[1] = torch.randn(C, generator=g) * 1e15
    x[2] = torch.randn(C, generator=g) * 1e-15
    y = torch.empty(R, C, dtype=torch.bfloat16, device="cuda")
    sp.sparoa_add_norm(ctx, x.cuda(), None, None, y, pre=sp.norm("layer", eps=0.0))
    _close(y, _norm64(x.double(), ("layer", None, None), 0.0), "layer norm", extra=1.6e-3)  # its mean: 25 roundings of 2^-24 of 1000


def test_add_norm_refusals(sp, ctx):
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    w = torch.ones(65, device="cuda")
    bad = [lambda: sp.sparoa_add_norm(ctx, x[:, :60].contiguous(), None, None, y[:, :60].contiguous()),
           lambda: sp.sparoa_add_norm(ctx, x, None, None, None),
           lambda: sp.sparoa_add_norm(ctx, None, None, x, y),
           lambda: sp.sparoa_add_norm(ctx, x, None, None, y, post=sp.norm("rms")),
           lambda: sp.sparoa_add_norm(ctx, x, x, None, y, gate=w[:64], rows_per_gate=2),
           lambda: sp.sparoa_add_norm(ctx, x, x, None, y, gate=w[:64], rows_per_gate=-1),
           lambda: sp.sparoa_add_norm(ctx, x, None, None, y, pre=sp.norm("rms", w[:63])),
           lambda: sp.sparoa_add_norm(ctx, x, None, None, y, pre=sp.norm("rms", w[1:])),  # off a 16-byte boundary
           lambda: sp.sparoa_add_norm(ctx, x, None, None, y, pre=sp.norm("rms", eps=-1.0)),
           lambda: sp.sparoa_add_norm(ctx, x, x[:2], None, y),
           lambda: sp.sparoa_add_norm(ctx, x.float(), x, torch.empty_like(x), y),
           lambda: sp.sparoa_add_norm(ctx, x.t(), None, None, y),
           lambda: sp.norm("rms", w.double())]
    for k, f in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            f()
            pytest.fail(f"call {k} was taken")
    big = torch.zeros(1, 16392, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sp.SparoaError) as e:
        sp.sparoa_add_norm(ctx, big, None, None, big)
    assert e.value.status == sp.ERR_UNSUPPORTED
    sp.sparoa_add_norm(ctx, x[:0], None, None, y[:0])  # no rows: nothing to do


# ---------------------------------------------------------------------------
# a batch over a paged cache
# ---------------------------------------------------------------------------
def _batch(sp, new, kv, page, KH, D, seed, fill="nan", spare=3):
    """Pools with every sequence's pages in random places; what no token was written to holds `fill`."""
    g = _g(seed)
    need = [-(-max(L, n, 1) // page) for n, L in zip(new, kv)]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(new), max(need)), -7, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    k = torch.full((pages, KH, page, D), float(fill), dtype=torch.bfloat16)
    v = k.clone()
    for b, L in enumerate(kv):
        for j0 in range(0, L, page):
            e = min(page, L - j0)
            p = int(table[b, j0 // page])
            k[p, :, :e] = torch.randn(KH, e, D, generator=g).to(torch.bfloat16)
            v[p, :, :e] = torch.randn(KH, e, D, generator=g).to(torch.bfloat16)
    start = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32)
    cache = sp.KVCache(k.cuda(), v.cuda())
    # (entries that no position needs stay -7: they are not read)
    batch = sp.PagedBatch(start.cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), table.cuda(), max_q=max(new))
    return cache, batch, k, v, table


def _seq(pool, table, b, L, page):
    """[KH, L, D] in 64 bits of sequence b."""
    if L == 0:
        return pool.double()[0][:, :0]
    return torch.cat([pool[int(table[b, j // page])][:, :min(page, L - j)] for j in range(0, L, page)], 1).double()


def _attn64(q, k, v, table, new, kv, page, scale, causal, window):
    """y, log of the sums, and sum p |v| (the size of the rounding of the probabilities)."""
    T, H, D = q.shape
    KH = k.shape[1]
    G = H // KH
    y = torch.zeros(T, H, D, dtype=torch.float64)
    size = torch.zeros_like(y)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    row = 0
    for b, (n, L) in enumerate(zip(new, kv)):
        ks, vs = _seq(k, table, b, L, page), _seq(v, table, b, L, page)
        pos = torch.arange(L - n, L)[:, None]
        j = torch.arange(L)[None]
        keep = torch.ones(n, L, dtype=torch.bool)
        if causal:
            keep &= j <= pos
        if window:
            keep &= j > pos - window
        for h in range(H):
            s = q[row:row + n, h].double() @ ks[h // G].t() * scale
            s = s.masked_fill(~keep, -math.inf)
            some = keep.any(1)
            if some.any():
                lse[row:row + n, h][some] = torch.logsumexp(s[some], 1)
                p = torch.softmax(s[some], 1)
                y[row:row + n, h][some] = p @ vs[h // G]
                size[row:row + n, h][some] = p @ vs[h // G].abs()
        row += n
    return y, lse, size


def _check_attn(sp, ctx, new, kv, H, KH, D, page, causal=True, window=0, seed=0, max_q=None, strided=False, scale=None,
                p_round=2.0 ** -9):
    cache, batch, k, v, table = _batch(sp, new, kv, page, KH, D, seed)
    if max_q is not None:
        batch.desc.max_q = max_q
    T = sum(new)
    q = (1.5 * torch.randn(T, H, D, generator=_g(seed + 1))).to(torch.bfloat16)
    if strided:
        buf = torch.full((T, H + 2 * KH, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        buf[:, :H] = q.cuda()
        qd = buf[:, :H]
    else:
        qd = q.cuda()
    y = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), float("nan"), device="cuda")
    sp.sparoa_paged_attention(ctx, qd, y, cache, batch, scale=scale, causal=causal, window=window, lse=lse)
    ctx.sync()
    want, wl, size = _attn64(q, k, v, table, new, kv, page, scale or D ** -0.5, causal, window)
    what = f"new {new} kv {kv} H{H}/{KH} D{D} page {page} causal {causal} window {window}"
    empty = torch.isinf(wl)
    got = lse.double().cpu()
    assert torch.equal(torch.isinf(got), empty) and not torch.isnan(got).any(), what
    assert ((got - wl)[~empty].abs() <= 2e-4).all(), what
    _close(y, want, what, extra=(p_round + 2.0 ** -12) * size)
    assert (y.cpu()[empty] == 0).all(), what
    return y, lse


LENGTHS = [([1], [1]), ([1], [15]), ([1], [16]), ([1], [17]), ([1], [127]), ([1], [129]), ([1], [3000]),
           ([1, 1, 1], [1, 700, 33]), ([1] * 17, [3 + 41 * i for i in range(17)]),
           ([2, 1, 3], [2, 64, 900]), ([5, 0, 4], [200, 10, 4]), ([1, 1, 2], [0, 130, 1])]


@pytest.mark.parametrize("new,kv", LENGTHS)
@pytest.mark.parametrize("H,KH,D,page", [(4, 4, 64, 16), (8, 2, 128, 64), (3, 1, 64, 32), (6, 2, 128, 128), (20, 1, 128, 16)])
def test_attention_few_rows(sp, ctx, new, kv, H, KH, D, page):
    _check_attn(sp, ctx, new, kv, H, KH, D, page, seed=len(new) + kv[0])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 5, 128, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_masks(sp, ctx, causal, window, D):
    _check_attn(sp, ctx, [3, 1, 7, 2], [400, 129, 7, 1], 4, 2, D, 32, causal=causal, window=window, seed=window)


def test_attention_strides_and_scale(sp, ctx):
    _check_attn(sp, ctx, [4, 1], [50, 300], 8, 4, 64, 16, strided=True, scale=0.03)
    _check_attn(sp, ctx, [1, 2], [500, 300], 4, 2, 128, 64, strided=True, scale=1.5)


CHUNKS = [([17], [17]), ([64], [64]), ([65], [65]), ([33], [500]), ([128], [128]), ([129], [129]), ([300], [300]), ([20], [3000]),
          ([100, 1, 40], [100, 700, 333]), ([16, 1], [16, 257]), ([40, 3], [100, 1000]), ([30, 0, 1, 200], [10, 0, 0, 1025]),
          ([257, 20], [2000, 20])]


@pytest.mark.parametrize("new,kv", CHUNKS)
@pytest.mark.parametrize("H,KH,D,page", [(2, 2, 64, 16), (8, 2, 128, 64), (3, 1, 64, 32), (6, 2, 128, 128), (20, 1, 128, 16)])
def test_attention_chunks(sp, ctx, new, kv, H, KH, D, page):
    _check_attn(sp, ctx, new, kv, H, KH, D, page, seed=len(new) + kv[0], p_round=2.0 ** -8)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 5, 128, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_chunk_masks(sp, ctx, causal, window, D):
    _check_attn(sp, ctx, [70, 1, 7, 150], [400, 129, 7, 1300], 4, 2, D, 32, causal=causal, window=window, seed=window,
                p_round=2.0 ** -8)


def test_attention_chunk_strides_and_scale(sp, ctx):
    _check_attn(sp, ctx, [40, 1], [50, 300], 8, 4, 64, 16, strided=True, scale=0.03, p_round=2.0 ** -8)
    _check_attn(sp, ctx, [1, 90], [500, 300], 4, 2, 128, 64, strided=True, scale=1.5, p_round=2.0 ** -8)
    _check_attn(sp, ctx, [50], [600], 4, 2, 64, 16, scale=20.0, p_round=2.0 ** -8)  # weights below the smallest float


def test_attention_growing_scores(sp, ctx):
    """Every key outweighs all before it by far, and the other way round: the rows' maxima move at
    every unit, or never again."""
    D, n, L, page = 64, 40, 1500, 16
    for sign in (1.0, -1.0):
        cache, batch, k, v, table = _batch(sp, [n], [L], page, 1, D, 5)
        u = torch.ones(D) / D ** 0.5
        for j in range(L):
            k[int(table[0, j // page]), 0, j % page] = (sign * u * j * 0.5).to(torch.bfloat16)
        cache.k.copy_(k)
        q = (torch.randn(n, 2, D, generator=_g(1)) * 0.1 + u).to(torch.bfloat16)
        y = torch.empty(n, 2, D, dtype=torch.bfloat16, device="cuda")
        sp.sparoa_paged_attention(ctx, q.cuda(), y, cache, batch, scale=1.0, causal=False)
        ctx.sync()
        want, _, size = _attn64(q, k, v, table, [n], [L], page, 1.0, False, 0)
        # scores of up to 800 in fp32: 64 2^-24 * 800 move the weights by 3e-3
        _close(y, want, f"growing {sign}", extra=(2.0 ** -8 + 4e-3) * size)


def test_attention_any_max_q(sp, ctx):
    """max_q chooses a kernel, not the result."""
    for mq in (0, 1, 1000):
        _check_attn(sp, ctx, [30, 1, 9], [77, 400, 9], 8, 2, 128, 32, max_q=mq, p_round=2.0 ** -8)
        _check_attn(sp, ctx, [30, 1, 9], [77, 400, 9], 6, 6, 64, 16, max_q=mq, p_round=2.0 ** -8)
        _check_attn(sp, ctx, [700], [700], 4, 1, 64, 16, max_q=mq, p_round=2.0 ** -8)


def test_attention_chunk_split_is_repeatable(sp, ctx):
    """Few tiles over a long context: their units are shared by many CTAs."""
    cache, batch, *_ = _batch(sp, [20], [40000], 64, 2, 128, 3)
    q = torch.randn(20, 8, 128, generator=_g(4)).to(torch.bfloat16).cuda()
    ys = [torch.empty(20, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(10)]
    for y in ys:
        sp.sparoa_paged_attention(ctx, q, y, cache, batch)
    ctx.sync()
    assert all(torch.equal(ys[0], y) for y in ys[1:])
    _check_attn(sp, ctx, [20], [40000], 8, 2, 128, 64, p_round=2.0 ** -8)


def test_attention_chunk_timeout(sp):
    """A wait that runs out: an error, and the context is usable afterwards."""
    c = sp.Context(0)
    cache, batch, *_ = _batch(sp, [64], [3000], 16, 2, 128, 8)
    q = torch.randn(64, 8, 128, generator=_g(1)).to(torch.bfloat16).cuda()
    y, z = torch.empty_like(q), torch.empty_like(q)
    sp.sparoa_paged_attention(c, q, y, cache, batch)
    c.sync()
    c.set_fault(1)
    c.set_wait_limit(2000000)
    sp.sparoa_paged_attention(c, q, z, cache, batch)
    with pytest.raises(sp.SparoaError) as e:
        c.sync()
    assert e.value.status == sp.ERR_TIMEOUT
    c.set_fault(0)
    c.set_wait_limit(0)
    sp.sparoa_paged_attention(c, q, z, cache, batch)
    c.sync()
    assert torch.equal(y, z)
    c.close()


def test_attention_split_is_repeatable(sp, ctx):
    """A sequence split over all SMs: the partial results are joined in one order."""
    cache, batch, *_ = _batch(sp, [1], [40000], 64, 2, 128, 3)
    q = torch.randn(1, 8, 128, generator=_g(4)).to(torch.bfloat16).cuda()
    ys = [torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(20)]
    for y in ys:
        sp.sparoa_paged_attention(ctx, q, y, cache, batch)
    ctx.sync()
    assert all(torch.equal(ys[0], y) for y in ys[1:])
    _check_attn(sp, ctx, [1], [40000], 8, 2, 128, 64)


def test_attention_large_scores(sp, ctx):
    """Scores of hundreds: one key takes all the weight, others fall below the smallest float."""
    _check_attn(sp, ctx, [1, 3], [300, 60], 4, 2, 64, 16, scale=20.0)


@pytest.mark.parametrize("new,kv", [([2, 1], [700, 3000]), ([100, 40], [700, 3000]), ([3, 1], [20, 40])])
def test_attention_nan_query(sp, ctx, new, kv):
    """A query that is not a number gives results that are none, not zeros, and leaves other rows alone."""
    cache, batch, k, v, table = _batch(sp, new, kv, 16, 2, 64, 8)
    T = sum(new)
    q = torch.randn(T, 4, 64, generator=_g(1)).to(torch.bfloat16)
    q[1, 2, 5] = float("nan")
    y = torch.empty(T, 4, 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(T, 4, device="cuda")
    sp.sparoa_paged_attention(ctx, q.cuda(), y, cache, batch, lse=lse)
    ctx.sync()
    assert torch.isnan(y[1, 2]).all() and torch.isnan(lse[1, 2])
    q[1, 2, 5] = 0.0
    want, wl, size = _attn64(q, k, v, table, new, kv, 16, 64 ** -0.5, True, 0)
    keep = torch.ones(T, 4, dtype=torch.bool)
    keep[1, 2] = False
    _close(y[keep], want[keep], "rows beside it", extra=(2.0 ** -8 + 2.0 ** -12) * size[keep])


def test_attention_leaves_other_rows(sp, ctx):
    """Rows past the last sequence's are not touched."""
    cache, batch, *_ = _batch(sp, [2, 1], [20, 40], 16, 2, 64, 8)
    q = torch.randn(6, 4, 64, generator=_g(1)).to(torch.bfloat16).cuda()
    y = torch.full((6, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    sp.sparoa_paged_attention(ctx, q, y, cache, batch)
    ctx.sync()
    assert (y[3:] == 7).all() and (y[:3] != 7).any()


def test_attention_reports_bad_lists(sp, ctx):
    """An entry outside the pool, a length past the table's row, rows past the tensor: an error, no fault."""
    def call(entry=None, length=None, start=None):
        cache, batch, *_ = _batch(sp, [1, 1], [40, 70], 16, 2, 64, 8)
        if entry is not None:
            batch.table[1, 2] = entry
        if length is not None:
            batch.kv_len[1] = length
        if start is not None:
            batch.q_start[2] = start
        q = torch.randn(2, 4, 64, generator=_g(1)).to(torch.bfloat16).cuda()
        sp.sparoa_paged_attention(ctx, q, torch.empty_like(q), cache, batch)
        ctx.sync()
    call()
    for bad in (dict(entry=-1), dict(entry=1000), dict(length=81), dict(length=-1), dict(start=5), dict(start=0)):
        with pytest.raises(sp.SparoaError) as e:
            call(**bad)
        assert e.value.status == sp.ERR_INVALID_ARG, bad
    call()


@pytest.mark.parametrize("n", [1, 2, 40, 300])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention_pages_before_the_window(sp, ctx, n, page):
    """Pages that every new token's window has left are not looked up: their entries may be anything."""
    L, window, H, KH, D = 1000, 150, 4, 2, 64
    cache, batch, k, v, table = _batch(sp, [n, n], [L, L - 3], page, KH, D, 17)
    q = torch.randn(2 * n, H, D, generator=_g(18)).to(torch.bfloat16)
    want, wl, size = _attn64(q, k, v, table, [n, n], [L, L - 3], page, D ** -0.5, True, window)
    for b, kv in enumerate([L, L - 3]):
        first = max(0, kv - n - window + 1)  # the oldest key that the first new token sees
        batch.table[b, :first // page] = -1
        assert first // page > 0
    y = torch.empty(2 * n, H, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(2 * n, H, device="cuda")
    sp.sparoa_paged_attention(ctx, q.cuda(), y, cache, batch, window=window, lse=lse)
    ctx.sync()
    assert ((lse.double().cpu() - wl).abs() <= 2e-4).all()
    _close(y, want, f"n {n} page {page}", extra=(2.0 ** -8 + 2.0 ** -12) * size)


@pytest.mark.parametrize("max_q", [1, 200])
def test_attention_widest_window(sp, ctx, max_q):
    """The widest window hides nothing, from tokens before their sequence's first position neither."""
    for causal in (True, False):
        _check_attn(sp, ctx, [7, 40, 2], [2, 20, 300], 4, 2, 64, 32, causal=causal, window=2 ** 31 - 1, seed=5, max_q=max_q,
                    p_round=2.0 ** -8)


@pytest.mark.parametrize("new,kv", [([1], [300]), ([70, 3], [300, 500]), ([200], [400])])
def test_attention_vanishing_scale(sp, ctx, new, kv):
    """A scale so small that the slack of the running maximum passes the largest float: every key weighs the same."""
    _check_attn(sp, ctx, new, kv, 4, 2, 64, 32, window=40, seed=4, scale=1e-38, p_round=2.0 ** -8)


def test_attention_streams(sp, ctx):
    """Calls of one context on two streams at once: each has partial results of its own."""
    jobs = []
    for i in range(2):
        cache, batch, k, v, table = _batch(sp, [1], [30000], 64, 1, 128, 20 + i)
        q = torch.randn(1, 4, 128, generator=_g(30 + i)).to(torch.bfloat16)
        ref = _attn64(q, k, v, table, [1], [30000], 64, 128 ** -0.5, True, 0)
        jobs.append((cache, batch, q.cuda(), torch.empty(1, 4, 128, dtype=torch.bfloat16, device="cuda"), ref,
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, batch, q, y, ref, st in jobs:
            with torch.cuda.stream(st):
                sp.sparoa_paged_attention(ctx, q, y, cache, batch)
    torch.cuda.synchronize()
    for cache, batch, q, y, ref, st in jobs:
        _close(y, ref[0], "streams", extra=(2.0 ** -9 + 2.0 ** -12) * ref[2])


def test_decoder_calls_under_capture(sp):
    """A first use under capture, replayed with other lengths, pages and queries."""
    c = sp.Context(0)
    H, KH, D, page = 8, 2, 64, 16
    new, kv = [1, 1], [100, 37]
    cache, batch, k, v, table = _batch(sp, new, kv, page, KH, D, 9)
    qkv = torch.zeros(2, (H + 2 * KH) * D, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, H, D, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros_like(q)
    rope = sp.Rope(D)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.sparoa_rope_append(c, qkv, q, cache, batch, rope)
        sp.sparoa_paged_attention(c, q, y, cache, batch)
    for step in range(3):
        lens = [kv[0] + step, kv[1] - 2 * step]
        batch.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        x = torch.randn(2, H + 2 * KH, D, generator=_g(step)).to(torch.bfloat16)
        qkv.copy_(x.view(2, -1))
        graph.replay()
        torch.cuda.synchronize()
        kc, vc = cache.k.cpu(), cache.v.cpu()
        ref, _, size = _attn64(q.cpu(), kc, vc, table, new, lens, page, D ** -0.5, True, 0)
        _close(y, ref, f"replay {step}", extra=(2.0 ** -9 + 2.0 ** -12) * size)
    c.close()


def test_attention_occupancy(sp, ctx):
    cache, batch, *_ = _batch(sp, [3, 2], [3, 0], 16, 2, 64, 8)
    q = torch.randn(5, 4, 64, generator=_g(1)).to(torch.bfloat16).cuda()
    y = torch.empty_like(q)
    occ = sp.OccupancyBuffer(5, 256)
    sp.sparoa_paged_attention(ctx, q, y, cache, batch, y_occ=occ)
    assert occ.to_host()["nnz"] == int((y != 0).sum()) == 3 * 256


def test_attention_refusals(sp, ctx):
    cache, batch, *_ = _batch(sp, [1], [20], 16, 2, 64, 8)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(q)
    go = sp.sparoa_paged_attention
    bad = [lambda: go(ctx, q, y, cache, batch, scale=0.0),
           lambda: go(ctx, q, y, cache, batch, scale=float("nan")),
           lambda: go(ctx, q, y, cache, batch, window=-1),
           lambda: go(ctx, q[:, :3], y[:, :3].contiguous(), cache, batch),     # 3 heads over 2
           lambda: go(ctx, q.transpose(1, 2), y, cache, batch),
           lambda: go(ctx, q.float(), y, cache, batch),
           lambda: go(ctx, q, y.float(), cache, batch),
           lambda: go(ctx, q, y, cache, batch, lse=torch.empty(1, 3, device="cuda")),
           lambda: sp.KVCache(cache.k, cache.v[:1]),
           lambda: sp.PagedBatch(batch.q_start, batch.kv_len, batch.table.long(), 1),
           lambda: sp.PagedBatch(batch.q_start[:1], batch.kv_len, batch.table, 1)]
    for k, f in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            f()
            pytest.fail(f"call {k} was taken")
    for shape in ((2, 2, 16, 96), (2, 2, 24, 64), (2, 2, 256, 64)):
        pool = torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
        x = torch.zeros(1, 4, shape[3], dtype=torch.bfloat16, device="cuda")
        with pytest.raises(sp.SparoaError) as e:
            go(ctx, x, torch.empty_like(x), sp.KVCache(pool, pool), batch)
        assert e.value.status == sp.ERR_UNSUPPORTED, shape
    many = sp.PagedBatch(torch.zeros(1026, dtype=torch.int32, device="cuda"), torch.zeros(1025, dtype=torch.int32, device="cuda"),
                         torch.zeros(1025, 1, dtype=torch.int32, device="cuda"), 1)
    with pytest.raises(sp.SparoaError) as e:
        go(ctx, q, y, cache, many)
    assert e.value.status == sp.ERR_UNSUPPORTED
    go(ctx, q[:0], y[:0], cache, batch)  # no tokens: nothing to do


def test_attention_workspace_failure(sp):
    c = sp.Context(0)
    cache, batch, *_ = _batch(sp, [1], [20], 16, 2, 64, 8)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    c.set_fault(2)
    with pytest.raises(sp.SparoaError) as e:
        sp.sparoa_paged_attention(c, q, torch.empty_like(q), cache, batch)
    assert e.value.status == sp.ERR_OOM
    sp.sparoa_paged_attention(c, q, torch.empty_like(q), cache, batch)
    c.sync()
    c.close()


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def _rope64(x, pos, freq, rot, layout, amp):
    """x [T, heads, D] in 64 bits, turned by pos [T]."""
    ang = pos.double()[:, None] * freq[None]
    cos, sin = (ang.cos() * amp)[:, None], (ang.sin() * amp)[:, None]
    out = x.clone()
    i = torch.arange(rot // 2)
    a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., b] * cos + x[..., a] * sin
    return out


def _freq64(rot, base=10000.0, scaling="none", factor=1.0, context=0.0, low=1.0, high=32.0):
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / max(rot, 1))
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        keep = ((context * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


@pytest.mark.parametrize("new,kv,page", [([1], [1], 16), ([1, 1, 1], [5, 64, 200], 16), ([7, 0, 33], [7, 3, 100], 32),
                                         ([130, 1], [1000, 17], 64), ([5, 4], [3, 4], 16)])
@pytest.mark.parametrize("H,KH,D,rot", [(4, 4, 64, 64), (8, 2, 128, 128), (6, 1, 128, 96), (3, 3, 64, 16), (2, 1, 64, 0)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_append(sp, ctx, new, kv, page, H, KH, D, rot, layout):
    T = sum(new)
    cache, batch, k, v, table = _batch(sp, new, kv, page, KH, D, T, fill=3.0)
    x = torch.randn(T, H + 2 * KH, D, generator=_g(T + D)).to(torch.bfloat16)
    q = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sp.sparoa_rope_append(ctx, x.view(T, -1).cuda(), q, cache, batch, sp.Rope(rot, layout=layout, scale=1.25))
    ctx.sync()
    pos = torch.cat([torch.arange(L - n, L) for n, L in zip(new, kv)])
    want = _rope64(x[:, :H + KH].double(), pos, _freq64(rot), rot, layout, 1.25)
    _close(q, want[:, :H], "q")
    ref = want[:, H:]
    wk, wv, wrote = k.double(), v.double(), torch.zeros(k.shape[0], page, dtype=torch.bool)
    for t, (b, p) in enumerate((b, p) for b, (n, L) in enumerate(zip(new, kv)) for p in range(L - n, L)):
        if p >= 0:
            at = int(table[b, p // page])
            wk[at, :, p % page], wv[at, :, p % page], wrote[at, p % page] = ref[t], x[t, H + KH:].double(), True
    gk, gv = cache.k.cpu(), cache.v.cpu()
    assert torch.equal(gv.double(), wv)
    _close(gk, wk, "keys", extra=1e-5 * wk.abs().amax())
    # what was cached before is as it was
    assert torch.equal(gk.transpose(1, 2)[~wrote], k.transpose(1, 2)[~wrote])


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_rope_far_positions(sp, ctx, scaling):
    """Angles of positions of millions, where a product of two floats is off by whole degrees: values
    of one pair member 0 and the other 1 give the cosines and sines themselves."""
    D = rot = 64
    kw = dict(base=500000.0, scaling=scaling, factor=8.0, context=8192, low=1.0, high=32.0)
    pos = torch.tensor([0, 1, 2, 1000, 131071, 1048575, 16777217, 2000000011, -5], dtype=torch.int32)
    T = pos.numel()
    cache, batch, *_ = _batch(sp, [T], [T], 16, 1, D, 0)
    x = torch.zeros(T, 3, D)
    x[:, :, :rot // 2] = 1.0
    q = torch.empty(T, 1, D, dtype=torch.bfloat16, device="cuda")
    sp.sparoa_rope_append(ctx, x.to(torch.bfloat16).view(T, -1).cuda(), q, cache, batch, sp.Rope(rot, **kw), positions=pos.cuda())
    ctx.sync()
    want = _rope64(x[:, :1].double(), pos, _freq64(rot, **kw), rot, "half", 1.0)
    # the frequency's own 2^-53 grows with the position: 2e9 * 2^-52 < 1e-6
    _close(q, want, scaling, extra=2e-6)


def test_rope_in_place_and_strided(sp, ctx):
    H, KH, D = 4, 2, 64
    new, kv = [3, 2], [10, 2]
    cache, batch, *_ = _batch(sp, new, kv, 16, KH, D, 0)
    other, same, *_ = _batch(sp, new, kv, 16, KH, D, 0)
    x = torch.randn(5, (H + 2 * KH) * D + 8, generator=_g(1)).to(torch.bfloat16).cuda()
    src = x[:, :-8]
    q = torch.empty(5, H, D, dtype=torch.bfloat16, device="cuda")
    rope = sp.Rope(64, layout="interleaved")
    sp.sparoa_rope_append(ctx, src, q, cache, batch, rope)
    sp.sparoa_rope_append(ctx, src, src[:, :H * D], other, same, rope)
    ctx.sync()
    assert torch.equal(src[:, :H * D].reshape(5, H, D), q)
    nan = torch.isnan(cache.k)
    assert torch.equal(nan, torch.isnan(other.k)) and torch.equal(cache.k[~nan], other.k[~nan])


def test_rope_bad_lists_and_refusals(sp, ctx):
    H, KH, D = 4, 2, 64
    x = torch.zeros(2, (H + 2 * KH) * D, dtype=torch.bfloat16, device="cuda")
    q = torch.empty(2, H, D, dtype=torch.bfloat16, device="cuda")
    rope = sp.Rope(32)
    for entry, length in ((-1, None), (500, None), (None, 1000)):
        cache, batch, *_ = _batch(sp, [1, 1], [40, 70], 16, KH, D, 8)
        before = cache.k.clone()
        if entry is not None:
            batch.table[1, 4] = entry
        if length is not None:
            batch.kv_len[1] = length
        sp.sparoa_rope_append(ctx, x, q, cache, batch, rope)
        with pytest.raises(sp.SparoaError) as e:
            ctx.sync()
        assert e.value.status == sp.ERR_INVALID_ARG
        changed = (cache.k.view(torch.int16) != before.view(torch.int16)).any(-1).any(1)
        assert int(changed.sum()) <= 1  # the other sequence's token only
    cache, batch, *_ = _batch(sp, [1, 1], [40, 70], 16, KH, D, 8)
    bad = [lambda: sp.sparoa_rope_append(ctx, x[:, :-8], q, cache, batch, rope),
           lambda: sp.sparoa_rope_append(ctx, x, q, cache, batch, sp.Rope(80)),
           lambda: sp.sparoa_rope_append(ctx, x, q.float(), cache, batch, rope),
           lambda: sp.sparoa_rope_append(ctx, x, q, cache, batch, rope, positions=torch.zeros(1, dtype=torch.int32, device="cuda")),
           lambda: sp.sparoa_rope_append(ctx, x.view(2, 4, -1).transpose(1, 2), q, cache, batch, rope),
           lambda: sp.Rope(24), lambda: sp.Rope(-16), lambda: sp.Rope(32, base=1.0), lambda: sp.Rope(32, scaling="linear", factor=0.5),
           lambda: sp.Rope(32, scaling="parts", factor=2.0, context=0.0),
           lambda: sp.Rope(32, scaling="parts", factor=2.0, context=10.0, low=4.0, high=4.0)]
    for k, f in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            f()
            pytest.fail(f"call {k} was taken")


def test_rope_leaves_other_rows(sp, ctx):
    cache, batch, *_ = _batch(sp, [1, 1], [40, 70], 16, 2, 64, 8)
    x = torch.ones(4, 8 * 64, dtype=torch.bfloat16, device="cuda")
    q = torch.full((4, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    sp.sparoa_rope_append(ctx, x, q, cache, batch, sp.Rope(64))
    ctx.sync()
    assert (q[2:] == 9).all() and (q[:2] != 9).all()
