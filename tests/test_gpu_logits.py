"""Logits to tokens on the GPU against 64 bits.

Tolerances.  A changed logit has five roundings at most, each 2^-24 of a number not above the sum of its
terms' sizes: 2^-21 of that sum.  The best token is that of the logits as stored.  The log of the sum: a
thread adds up to V / 512 weights and 30 joins follow, each 2^-24, a weight is off by 2^-21 and by its
argument's rounding (2^-24 of at most 20 where it counts): 1e-5 up to V = 3e5, and 2^-22 of its size."""
import math

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


def _case(R, V, dtype, seen=0, penalties=False, bias=0, masked=False, seed=0):
    g = torch.Generator().manual_seed(seed * 1009 + R * 17 + V)
    c = {"x": (torch.randn(R, V, generator=g) * 3).to(dtype)}
    if seen:
        lens = [0 if r % 3 == 1 else int(torch.randint(1, seen + 1, (), generator=g)) for r in range(R)]
        c["start"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
        c["seen"] = (torch.rand(sum(lens), generator=g) ** 2 * V).int()
    if penalties:
        p = torch.rand(R, 4, generator=g)
        c["penalties"] = torch.stack([1 + p[:, 0], p[:, 1] - 0.3, p[:, 2], 0.3 + p[:, 3]], 1)
    if bias:
        c["bias"] = torch.randn(R if bias == 2 else 1, V, generator=g)
    if masked:
        c["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (R, (V + 31) // 32), generator=g).int()
    return c


def _want(c):
    """Changed logits in 64 bits, and the sum of the sizes of their terms."""
    x = c["x"].double()
    R, V = x.shape
    rep, presence, frequency, temperature = c["penalties"].double().t()[..., None] if "penalties" in c else torch.tensor([1.0, 0, 0, 1.0])[:, None, None].double()
    size = x.abs()
    if "seen" in c and "penalties" in c:
        count = torch.zeros(R, V, dtype=torch.float64)
        for r in range(R):
            t = c["seen"][c["start"][r]:c["start"][r + 1]].long()
            t = t[(t >= 0) & (t < V)]
            count[r].index_add_(0, t, torch.ones(len(t), dtype=torch.float64))
        less = torch.where(x > 0, x / rep, x * rep) - presence - frequency * count
        size = torch.where(count > 0, x.abs() * rep.clamp_min(1) + presence.abs() + (frequency * count).abs(), size)
        x = torch.where(count > 0, less, x)
    if "bias" in c:
        x, size = x + c["bias"].double(), size + c["bias"].double().abs()
    x, size = x / temperature, size / temperature
    if "allowed" in c:
        v = torch.arange(V)
        on = (c["allowed"][:, v // 32] >> (v % 32)) & 1
        x = torch.where(on == 1, x, -math.inf)
    return x, size


def _rules(sp, c):
    d = {k: c[k].cuda() for k in ("seen", "penalties", "bias", "allowed") if k in c}
    return sp.LogitRules(seen_start=c["start"].cuda() if "start" in c else None, **d)


def _check(y, best, lse, c):
    want, size = _want(c)
    V = want.shape[1]
    if y is not None:
        y = y.cpu()
        masked = want == -math.inf
        assert torch.equal(y == -math.inf, masked)
        assert ((y.double() - want).abs() <= 2.0 ** -21 * size)[~masked].all()
        first = torch.where(y == y.amax(1, keepdim=True), torch.arange(V), V).amin(1)
    else:
        first = want.argmax(1)
    first = torch.where(want.amax(1) > -math.inf, first, -1)
    assert torch.equal(best.cpu().long(), first)
    ref = torch.logsumexp(want, 1)
    got = lse.cpu().double()
    none = ref == -math.inf
    assert torch.equal(got == -math.inf, none)
    assert ((got - ref).abs() <= 1e-5 + 2.0 ** -22 * ref.abs())[~none].all()


def _run(sp, ctx, c, store=True):
    R, V = c["x"].shape
    y = torch.full((R, V), 7.0, device="cuda") if store else None
    best, lse = torch.full((R,), 99, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")
    sp.sparoa_shape_logits(ctx, c["x"].cuda(), _rules(sp, c), y=y, best=best, lse=lse)
    _check(y, best, lse, c)


@pytest.mark.parametrize("R,V", [(1, 1), (1, 31), (2, 33), (3, 512), (1, 4097), (5, 5000), (7, 16387), (2, 32000), (1, 70001), (33, 1003), (700, 257)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rules", [{}, {"seen": 40, "penalties": True}, {"penalties": True, "bias": 1, "masked": True},
                                   {"seen": 3000, "penalties": True, "bias": 2, "masked": True}, {"seen": 5, "bias": 1}])
def test_rules(sp, ctx, R, V, dtype, rules):
    _run(sp, ctx, _case(R, V, dtype, **rules))


@pytest.mark.parametrize("R,V,seen", [(1, 260001, 9000), (2, 500003, 50), (160, 40001, 100), (1, 1000003, 70000)])
def test_large(sp, ctx, R, V, seen):
    """Vocabularies that are counted in several pieces, lists longer than 16 bits hold."""
    _run(sp, ctx, _case(R, V, torch.float32, seen=seen, penalties=True, masked=True))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_without_stored_logits(sp, ctx, dtype):
    c = _case(9, 12345, torch.float32, seen=30, penalties=True, bias=1, masked=True)
    c["x"] = c["x"].to(dtype)
    _run(sp, ctx, c, store=False)


def test_in_place_and_strided(sp, ctx):
    c = _case(6, 1001, torch.float32, seen=30, penalties=True, bias=2)
    wide = torch.full((6, 1100), 5.0, device="cuda")
    x = wide[:, 50:1051]
    x.copy_(c["x"])
    best, lse = torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda")
    sp.sparoa_shape_logits(ctx, x, _rules(sp, c), y=x, best=best, lse=lse)
    _check(x, best, lse, c)
    assert (wide[:, :50] == 5).all() and (wide[:, 1051:] == 5).all()


def test_one_token_many_times(sp, ctx):
    """A list of one token: every count adds up, also beyond 16 bits."""
    c = _case(2, 300, torch.float32, penalties=True)
    c["start"] = torch.tensor([0, 70000, 70000], dtype=torch.int32)
    c["seen"] = torch.full((70000,), 299, dtype=torch.int32)
    c["penalties"][:, 2] = 2.0 ** -10
    _run(sp, ctx, c)


def test_tokens_outside_the_vocabulary(sp, ctx):
    c = _case(3, 500, torch.float32, penalties=True)
    c["start"] = torch.tensor([0, 4, 4, 7], dtype=torch.int32)
    c["seen"] = torch.tensor([-1, 500, 3, 2 ** 31 - 1, -2 ** 31, 0, 0], dtype=torch.int32)
    _run(sp, ctx, c)
    ctx.sync()


def test_masks_and_infinities(sp, ctx):
    """Rows without a token, rows of minus infinity, NaN and infinity in masked places and in open ones."""
    V = 1000
    x = torch.randn(8, V, generator=torch.Generator().manual_seed(1))
    allowed = torch.full((8, 32), -1, dtype=torch.int32)
    allowed[0] = 0
    x[1] = -math.inf
    x[2, 5], x[2, 6] = math.nan, math.inf
    allowed[2, 0] = ~(3 << 5)
    x[3, 999] = math.inf
    x[4, 77] = math.nan
    x[5] = math.nan
    x[6] = -torch.finfo(torch.float32).max
    x[7, 3:] = -math.inf
    y, best, lse = torch.empty(8, V, device="cuda"), torch.empty(8, dtype=torch.int32, device="cuda"), torch.empty(8, device="cuda")
    sp.sparoa_shape_logits(ctx, x.cuda(), sp.LogitRules(allowed=allowed.cuda()), y=y, best=best, lse=lse)
    best, lse, y = best.tolist(), lse.cpu(), y.cpu()
    open4 = x[4].clone()
    open4[77] = -math.inf
    assert best == [-1, -1, int(torch.where(torch.arange(V) // 2 == 10 ** 9, x[2], x[2].masked_fill((torch.arange(V) == 5) | (torch.arange(V) == 6), -math.inf)).argmax()),
                    999, int(open4.argmax()), -1, 0, int(x[7, :3].argmax())]
    assert lse[0] == -math.inf and lse[1] == -math.inf and lse[3] == math.inf and lse[4].isnan() and lse[5].isnan()
    assert (y[0] == -math.inf).all() and y[2, 5] == -math.inf and y[2, 6] == -math.inf
    open2 = x[2].double().masked_fill((torch.arange(V) == 5) | (torch.arange(V) == 6), -math.inf)
    assert abs(lse[2].double() - torch.logsumexp(open2, 0)) <= 1e-5
    assert abs(lse[7].double() - torch.logsumexp(x[7, :3].double(), 0)) <= 1e-5
    assert lse[6] == -torch.finfo(torch.float32).max  # (log 1000 is far below its spacing)


def test_ties_go_to_the_lowest(sp, ctx):
    for V, at in ((64, (9, 40)), (100003, (50, 70000)), (40000, (39999, 39998))):
        x = torch.zeros(2, V)
        for t in at:
            x[:, t] = 3.0
        best = torch.empty(2, dtype=torch.int32, device="cuda")
        sp.sparoa_shape_logits(ctx, x.cuda(), best=best)
        assert best.tolist() == [min(at)] * 2
    x = torch.zeros(1, 5000, device="cuda")
    sp.sparoa_shape_logits(ctx, x, best=best[:1])
    assert best[0] == 0


def test_lists_out_of_bounds_are_reported(sp):
    ctx = sp.Context(0)
    c = _case(4, 300, torch.float32, penalties=True)
    for start in ([0, 9, 3, 3, 3], [-1, 0, 0, 0, 0], [0, 0, 0, 0, 4]):
        c["start"], c["seen"] = torch.tensor(start, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
        y = torch.empty(4, 300, device="cuda")
        sp.sparoa_shape_logits(ctx, c["x"].cuda(), _rules(sp, c), y=y)
        with pytest.raises(sp.SparoaError) as e:
            ctx.sync()
        assert e.value.status == sp.ERR_INVALID_ARG
        assert y.isfinite().all()
    ctx.sync()
    ctx.close()


def test_graph(sp, ctx):
    c = _case(3, 40001, torch.float32, seen=20, penalties=True)
    x, rules = c["x"].cuda(), _rules(sp, c)
    y, best, lse = torch.empty_like(x), torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    sp.sparoa_shape_logits(ctx, x, rules, y=y, best=best, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.sparoa_shape_logits(ctx, x, rules, y=y, best=best, lse=lse)
    c["x"] = c["x"].flip(1)
    x.copy_(c["x"])
    graph.replay()
    torch.cuda.synchronize()
    _check(y, best, lse, c)


def test_refusals(sp, ctx):
    x = torch.zeros(4, 100, device="cuda")
    i4 = torch.zeros(4, dtype=torch.int32, device="cuda")
    L = sp.LogitRules
    bad = [lambda: L(seen=i4), lambda: L(penalties=x), lambda: L(seen_start=i4.long(), seen=i4), lambda: L(bias=x.half()),
           lambda: L(allowed=i4), lambda: sp.sparoa_shape_logits(ctx, x), lambda: sp.sparoa_shape_logits(ctx, x.half(), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x, best=i4[:3]), lambda: sp.sparoa_shape_logits(ctx, x, best=i4.long()),
           lambda: sp.sparoa_shape_logits(ctx, x, y=x[:, :99]), lambda: sp.sparoa_shape_logits(ctx, x.t(), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x, L(bias=x[0, :99].contiguous()), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x, L(bias=x[:3].contiguous()), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x, L(allowed=i4.view(4, 1)), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x, L(penalties=x[:3, :4].contiguous()), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x, L(seen_start=i4, seen=i4), best=i4),
           lambda: sp.sparoa_shape_logits(ctx, x.to(torch.bfloat16), y=x.half()), lambda: sp.sparoa_shape_logits(ctx, x.cpu(), best=i4)]
    for i, f in enumerate(bad):
        with pytest.raises(sp.SparoaError):
            f()
            raise AssertionError(f"call {i} was taken")
    ctx.sync()


def test_division_is_rounded_as_a_division(sp, ctx):
    """z / repetition is the rounded quotient: the bits of the division of two fp32 numbers, for ordinary sizes;
    infinities stay."""
    V = 100000
    g = torch.Generator().manual_seed(12)
    x = torch.randn(4, V, generator=g).abs() * torch.tensor([[1.0], [1e-20], [1e20], [3.0]])
    x[3, 7] = math.inf
    rep = torch.tensor([1.1, 1.3, 0.7, 1.9999999])
    pen = torch.stack([rep, torch.zeros(4), torch.zeros(4), torch.ones(4)], 1)
    start = torch.arange(5, dtype=torch.int32) * V
    seen = torch.arange(V, dtype=torch.int32).repeat(4)
    y = torch.empty(4, V, device="cuda")
    xd = x.cuda()
    sp.sparoa_shape_logits(ctx, xd, sp.LogitRules(seen_start=start.cuda(), seen=seen.cuda(), penalties=pen.cuda()), y=y)
    assert torch.equal(y, xd / rep.cuda()[:, None])
