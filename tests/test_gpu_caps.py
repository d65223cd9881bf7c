"""Capped attention scores on the GPU against 64 bits, over all that a cap and a scale may be: few rows, one tile of
rows, two tiles.

Tolerances.  A raw score q k is off by D 2^-24 of sum |q k|, which a cap passes on by its slope, 1 - tanh^2.  The
capped score is off by 2^-20 of itself: the quotient's, the polynomial's, the tanh's and the product's roundings.  The
log of the sum is off by the mean of its scores' errors, and a result by sum p |v - y| of them; half as much again
is allowed for second orders.  Weights, their sums and the log take 2^-18 more, and probabilities rounded to
one bf16 2^-8 of sum p |v|."""
import math

import pytest
import torch

from test_gpu_decoder import _batch, _close, _g, _seq

pytestmark = pytest.mark.gpu

ROWS = [(1, 300), (40, 500), (300, 700)]  # new and cached tokens; two rows of a key head a token


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


def _check(sp, ctx, q, cache, batch, k, v, table, L, page, cap, scale, slopes=None):
    """One sequence's new tokens q [n, H, D] behind L - n others."""
    n, H, D = q.shape
    rules = sp.ScoreRules(cap=cap, slopes=None if slopes is None else slopes.cuda())
    y, lse = torch.full((n, H, D), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((n, H), 5.0, device="cuda")
    sp.sparoa_ruled_attention(ctx, q.cuda(), y, cache, batch, rules, scale=scale, lse=lse)
    ctx.sync()
    G = H // k.shape[1]
    kk, vv = (_seq(t, table, 0, L, page).repeat_interleave(G, 0) for t in (k, v))
    x = q.double().transpose(0, 1)
    z = torch.tanh(x @ kk.transpose(1, 2) * scale / cap)
    err = 2.0 ** -24 * D * scale * (x.abs() @ kk.abs().transpose(1, 2)) * (1 - z * z) + 2.0 ** -20 * (cap * z).abs()
    s = cap * z
    far = (torch.arange(L - n, L)[:, None] - torch.arange(L)[None]).double()
    if slopes is not None:
        s = s - slopes.double()[:, None, None] * far
        err = err + 2.0 ** -21 * s.abs()
    s = s.masked_fill(far < 0, -math.inf)
    p = torch.softmax(s, -1)
    want, size, off = p @ vv, p @ vv.abs(), 1.5 * (p * err)
    tol = off.sum(-1) + 2.0 ** -18 + 2.0 ** -22 * torch.logsumexp(s, -1).abs()
    got = lse.double().cpu().t()
    assert ((got - torch.logsumexp(s, -1)).abs() <= tol).all(), f"lse off by {((got - torch.logsumexp(s, -1)).abs() - tol).max():.2e}"
    extra = (2.0 ** -8 + 2.0 ** -17) * size + off @ vv.abs() + off.sum(-1)[..., None] * want.abs()
    _close(y, want.transpose(0, 1), "y", extra=extra.transpose(0, 1))


def _inputs(sp, n, L, seed, page=32, D=64, H=4, KH=2):
    cache, batch, k, v, table = _batch(sp, [n], [L], page, KH, D, seed)
    return torch.randn(n, H, D, generator=_g(seed + 1)), cache, batch, k, v, table


@pytest.mark.parametrize("n,L", ROWS)
@pytest.mark.parametrize("cap,scale", [(0.001, 1.4e3), (0.001, 1e6), (1.0, 1e8), (0.001, 2e38), (30.0, 1e-30)])
def test_a_scale_of_any_size(sp, ctx, n, L, cap, scale):
    """Scores that are zero (empty queries) beside a cap that others are far beyond."""
    q, *rest = _inputs(sp, n, L, 11)
    q[::3] = 0
    q[:, 1] = 0
    _check(sp, ctx, q.to(torch.bfloat16), *rest, L, 32, cap, scale)


@pytest.mark.parametrize("n,L", ROWS)
@pytest.mark.parametrize("cap", [1e3, 1e4, 1e6, 1e30, 3e38])
def test_caps_far_above_the_scores(sp, ctx, n, L, cap):
    """leave them as they are, products of more than 1024 too."""
    q, *rest = _inputs(sp, n, L, 12)
    _check(sp, ctx, (100 * q).to(torch.bfloat16), *rest, L, 32, cap, 0.01)


@pytest.mark.parametrize("n,L", ROWS)
@pytest.mark.parametrize("cap", [0.01, 2.0, 50.0, 54.0, 56.0, 1000.0])
@pytest.mark.parametrize("biased", [False, True])
def test_scores_small_and_large_in_turn(sp, ctx, n, L, cap, biased):
    """Every other 128 keys are 40 times as large, and of those every fifth as small as the others."""
    q, cache, batch, k, v, table = _inputs(sp, n, L, 13)
    for j in range(L):
        if j // 128 % 2 and j % 5:
            k[int(table[0, j // 32]), :, j % 32] *= 40
    cache.k.copy_(k)
    slopes = torch.tensor([0.5, 0.1, 0.01, 0.0]) if biased else None
    _check(sp, ctx, q.to(torch.bfloat16), cache, batch, k, v, table, L, 32, cap, 0.125, slopes)


@pytest.mark.parametrize("n", [1, 40, 75, 300])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("heads", [4, 6])
def test_results_know_nothing_of_what_is_not_seen(sp, ctx, n, slopes, heads):
    """The same bits whatever is in places that no token was written to, before the window and behind a token."""
    outs = []
    for fill in ("0", "nan", "inf", "30000"):
        cache, batch, k, v, table = _batch(sp, [n], [700], 64, 2, 64, 14, fill=fill)
        cache.k[int(table[0, 0])] = float(fill)  # before every token's window
        q = torch.randn(n, heads, 64, generator=_g(15)).to(torch.bfloat16).cuda()
        y, lse = torch.empty_like(q), torch.empty(n, heads, device="cuda")
        rules = sp.ScoreRules(cap=30.0, slopes=torch.full((heads,), 0.02, device="cuda") if slopes else None)
        sp.sparoa_ruled_attention(ctx, q, y, cache, batch, rules, window=300, lse=lse)
        ctx.sync()
        outs.append((y.clone(), lse.clone()))
    assert outs[0][0].isfinite().all() and outs[0][1].isfinite().all()
    for y, lse in outs[1:]:
        assert torch.equal(y, outs[0][0]) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("n", [1, 40, 75, 300])
@pytest.mark.parametrize("slopes", [False, True])
def test_results_know_nothing_of_other_sequences(sp, ctx, n, slopes):
    """The same bits whatever the next sequence asks for."""
    outs = []
    for loud in (0.0, 1.0, 1e4, float("nan")):
        cache, batch, *_ = _batch(sp, [n, 70], [700, 300], 64, 2, 64, 16)
        q = torch.randn(n + 70, 4, 64, generator=_g(17))
        q[n:] *= loud
        q = q.to(torch.bfloat16).cuda()
        y, lse = torch.empty_like(q), torch.empty(n + 70, 4, device="cuda")
        rules = sp.ScoreRules(cap=30.0, slopes=torch.full((4,), 0.02, device="cuda") if slopes else None)
        sp.sparoa_ruled_attention(ctx, q, y, cache, batch, rules, lse=lse)
        ctx.sync()
        outs.append((y[:n].clone(), lse[:n].clone()))
    assert outs[0][0].isfinite().all() and outs[0][1].isfinite().all()
    for y, lse in outs[1:]:
        assert torch.equal(y, outs[0][0]) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("cap", [0.01, 5.0, 50.0, 1e4, 1e30])
def test_capped_scores_have_fp32_bits(sp, ctx, n, cap):
    """A row's keys are all alike, so that the log of the sum is its score and the log of their number; off by
    2^-21 of the score and by 2^-20 for the sum's weights (2^-22), the logs and their sum."""
    H, D, L = 8, 64, 700
    cache, batch, k, v, table = _batch(sp, [n], [L], 64, 1, D, 18)
    k[:] = 0
    k[..., 0] = 1
    cache.k.copy_(k)
    q = torch.zeros(n, H, D)
    t = torch.exp(torch.rand(n, H, generator=_g(19)) * math.log(1e5) + math.log(1e-4)).clamp(max=10.0)
    if n == 1:
        t[0] = torch.tensor([1e-3, 0.01, 0.1, 0.3, 0.45, 0.55, 1.0, 3.0])
    q[..., 0] = (t * min(cap, 1e30)).clamp(max=100.0) * torch.where(torch.arange(H) % 3 == 0, -1.0, 1.0)
    q = q.to(torch.bfloat16)
    y, lse = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H, device="cuda")
    sp.sparoa_ruled_attention(ctx, q.cuda(), y, cache, batch, sp.ScoreRules(cap=cap), scale=1.0, lse=lse)
    ctx.sync()
    score = cap * torch.tanh(q[..., 0].double() / cap)
    keys = torch.arange(L - n + 1, L + 1).double().log()[:, None]
    err = (lse.double().cpu() - score - keys).abs()
    tol = 2.0 ** -21 * score.abs() + 2.0 ** -20 * (1 + keys)
    assert (err <= tol).all(), f"off by {(err / tol).max():.2f} of what is allowed"
